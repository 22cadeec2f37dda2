"""Refusals of the calls that write the cache, without a GPU: layers and
entries that share memory, and a commit's pointers when no token is new."""
import pytest

from paper_2605_28283_gb300 import binding as pp
from test_attn_abi import A, append, batch, cache, commit, lib  # noqa: F401


def accepted(status):
    """What a call that passes its checks returns without a GPU."""
    return status in (pp.PP_ERR_CUDA, pp.PP_ERR_UNSUPPORTED)


needs_no_gpu = pytest.mark.skipif("__import__('torch').cuda.is_available()",
                                  reason="made-up addresses would be launched")


@pytest.mark.parametrize("layer_stride", [0, 64, 128, 1024, 16 * 1024, 9 * 16 * 1024])
def test_commit_refuses_layers_that_share_memory(lib, layer_stride):  # noqa: F811
    """0 is the binding's default; the others lay layer 1 over a head, a token or a page of layer 0."""
    assert commit(lib, layers=2, ls=layer_stride) == pp.PP_ERR_INVALID_ARG


@needs_no_gpu
def test_commit_takes_layers_that_lie_apart(lib):  # noqa: F811
    assert accepted(commit(lib, layers=1, ls=0))                   # one layer: no stride needed
    assert accepted(commit(lib, layers=3, ls=10 * 16 * 1024))      # layer by layer
    # the layers of a page side by side, of a token side by side, and head by head
    assert accepted(commit(lib, c=cache(page_stride=2 * 16 * 1024), layers=2, ls=16 * 1024))
    assert accepted(commit(lib, c=cache(page_stride=2 * 16 * 1024, token_stride=2 * 1024), layers=2, ls=1024))
    assert accepted(commit(lib, c=cache(head_stride=16 * 128, token_stride=128), layers=2, ls=10 * 16 * 1024))
    # dimensions of one entry carry any stride
    assert accepted(commit(lib, c=cache(n_pages=1, page_stride=0, n_heads=4, n_kv_heads=1, head_stride=0), layers=2, ls=16 * 1024))


@pytest.mark.parametrize("call", [append, commit])
@pytest.mark.parametrize("kw", [dict(head_stride=0), dict(head_stride=64), dict(token_stride=0), dict(token_stride=512),
                                dict(page_stride=0), dict(page_stride=8 * 1024)])
def test_entries_that_share_memory_are_not_written(lib, call, kw):  # noqa: F811
    assert call(lib, c=cache(**kw)) == pp.PP_ERR_INVALID_ARG


@needs_no_gpu
def test_reading_entries_that_share_memory_is_allowed(lib):  # noqa: F811
    """Attention over one key head under several heads' names."""
    from test_attn_abi import attend
    assert accepted(attend(lib, c=cache(head_stride=0)))


@pytest.mark.parametrize("kw,want", [(dict(q_start=0), pp.PP_ERR_INVALID_ARG), (dict(ctx_len=0), pp.PP_ERR_INVALID_ARG),
                                     (dict(pages=0), pp.PP_ERR_INVALID_ARG), (dict(q_start=A + 2), pp.PP_ERR_ALIGN),
                                     (dict(ctx_len=A + 1), pp.PP_ERR_ALIGN), (dict(pages=A + 2), pp.PP_ERR_ALIGN)])
def test_commit_checks_its_pointers_when_no_token_is_new(lib, kw, want):  # noqa: F811
    """A commit of no new tokens still runs (it writes new_len), so it reads the batch."""
    assert commit(lib, b=batch(n_tokens=0, **kw)) == want


@needs_no_gpu
def test_commit_of_nothing_needs_no_path(lib):  # noqa: F811
    """Paths of length zero, and no sequences: tensors without elements have no address."""
    assert accepted(commit(lib, path=None, mp=0))
    assert accepted(commit(lib, b=batch(n_seqs=0, q_start=0, ctx_len=0, pages=0), path=None, acc=None))
    assert commit(lib, path=None, mp=1) == pp.PP_ERR_INVALID_ARG
    assert commit(lib, path=None, mp=0, acc=None) == pp.PP_ERR_INVALID_ARG


@pytest.mark.gpu
def test_commit_of_nothing_on_the_gpu():
    import torch
    ints = lambda *shape, fill=0: torch.full(shape, fill, dtype=torch.int32, device="cuda")  # noqa: E731
    k = torch.randn(4, 16, 2, 64, device="cuda")
    c = pp.KVCache(k.clone(), k.clone(), 2)
    ws = pp.alloc_attn_workspace(c)
    b = pp.Batch(torch.tensor([0, 3, 3], dtype=torch.int32, device="cuda"), ints(2, fill=5), ints(2, 2), 3)
    new_len = ints(2, fill=-1)
    pp.pp_kv_commit(c, b, ints(2, 0), ints(2), ws, new_len=new_len)
    assert new_len.tolist() == [5, 5] and torch.equal(c.k, k) and torch.equal(c.v, k)
    none = pp.Batch(ints(1), ints(0), ints(0, 1), 0)
    pp.pp_kv_commit(c, none, ints(0, 4), ints(0), ws, new_len=ints(0))
    assert pp.pp_get_device_status(ws) == pp.PP_OK
