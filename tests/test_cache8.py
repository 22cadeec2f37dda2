"""The cache in 8 bits without a GPU: refusals (before any CUDA call, with the
documented status) and the restatement's own rounding against torch's."""
import ctypes

import numpy as np
import pytest

import cache8_ref as ref
from paper_2605_28283_gb300 import binding as pp
from paper_2605_28283_gb300 import build as ppbuild

A = 0x1000000  # an aligned address; nothing dereferences it: every call here is refused
BIG = 1 << 40
PAGE = 32 * 8 * 128


@pytest.fixture(scope="module")
def lib():
    ppbuild.build()
    return pp.load()


def cache(**kw):
    d = dict(dtype=pp.PP_BF16, n_heads=32, n_kv_heads=8, head_dim=128, page_size=32, n_pages=10, block=16, page_stride=PAGE,
             token_stride=1024, head_stride=128, k=A, v=2 * A, k_scale=3 * A, v_scale=4 * A)
    d.update(kw)
    return pp.pp_cache8(*[d[n] for n, _ in pp.pp_cache8._fields_])


def batch(**kw):
    d = dict(n_seqs=2, n_tokens=5, max_pages=4, q_start=A, ctx_len=A, pages=A)
    d.update(kw)
    return pp.pp_batch(*[d[n] for n, _ in pp.pp_batch._fields_])


def r(x):
    return None if x is None else ctypes.byref(x)


C, B = cache(), batch()


def append(lib, c=C, b=B, n=None, rot=None, pos=None, q=5 * A, qs=4096, k=6 * A, ks=1024, v=7 * A, vs=1024, o=8 * A, os_=4096,
           ws=A, size=BIG):
    return lib.pp_kvq_append(r(c), r(b), r(n), r(rot), pos, q, qs, k, ks, v, vs, o, os_, ws, size, None)


def read(lib, c=C, b=B, k=6 * A, ks=1024, v=7 * A, vs=1024, ws=A, size=BIG):
    return lib.pp_kvq_read(r(c), r(b), k, ks, v, vs, ws, size, None)


def attend(lib, c=C, b=B, q=5 * A, qs=4096, mask=None, words=0, scale=0.1, o=8 * A, os_=4096, ws=A, size=BIG):
    return lib.pp_kvq_tree_attention(r(c), r(b), q, qs, mask, words, scale, o, os_, ws, size, None)


def commit(lib, c=C, b=B, layers=1, ls=0, sls=0, path=A, mp=8, acc=2 * A, new=None, ws=A, size=BIG):
    return lib.pp_kvq_commit(r(c), r(b), layers, ls, sls, path, mp, acc, new, ws, size, None)


BAD_CACHES = [(None, pp.PP_ERR_INVALID_ARG), (dict(dtype=5), pp.PP_ERR_DTYPE), (dict(n_heads=0), pp.PP_ERR_SHAPE),
              (dict(n_kv_heads=5), pp.PP_ERR_SHAPE), (dict(n_kv_heads=0), pp.PP_ERR_SHAPE), (dict(head_dim=120), pp.PP_ERR_SHAPE),
              (dict(head_dim=272), pp.PP_ERR_SHAPE), (dict(head_dim=0), pp.PP_ERR_SHAPE), (dict(page_size=24), pp.PP_ERR_SHAPE),
              (dict(page_size=0), pp.PP_ERR_SHAPE), (dict(n_pages=0), pp.PP_ERR_SHAPE), (dict(block=8), pp.PP_ERR_SHAPE),
              (dict(block=0), pp.PP_ERR_SHAPE), (dict(block=64), pp.PP_ERR_SHAPE), (dict(k=0), pp.PP_ERR_INVALID_ARG),
              (dict(v_scale=0), pp.PP_ERR_INVALID_ARG), (dict(k=A + 8), pp.PP_ERR_ALIGN), (dict(k_scale=A + 2), pp.PP_ERR_ALIGN),
              (dict(token_stride=1032), pp.PP_ERR_ALIGN), (dict(head_stride=-16), pp.PP_ERR_INVALID_ARG)]
BAD_BATCHES = [(None, pp.PP_ERR_INVALID_ARG), (dict(n_seqs=-1), pp.PP_ERR_SHAPE), (dict(n_tokens=-1), pp.PP_ERR_SHAPE),
               (dict(max_pages=-1), pp.PP_ERR_SHAPE), (dict(n_tokens=1 << 27), pp.PP_ERR_SHAPE),
               (dict(q_start=0), pp.PP_ERR_INVALID_ARG), (dict(ctx_len=0), pp.PP_ERR_INVALID_ARG),
               (dict(pages=0), pp.PP_ERR_INVALID_ARG), (dict(pages=A + 2), pp.PP_ERR_ALIGN)]


@pytest.mark.parametrize("call", [append, read, attend, commit])
def test_caches_batches_and_workspaces(lib, call):
    for kw, want in BAD_CACHES:
        assert call(lib, c=None if kw is None else cache(**kw)) == want, kw
    for kw, want in BAD_BATCHES:
        assert call(lib, b=None if kw is None else batch(**kw)) == want, kw
    assert call(lib, ws=0) == pp.PP_ERR_WORKSPACE
    assert call(lib, ws=A + 16) == pp.PP_ERR_WORKSPACE
    need = lib.pp_kvq_workspace_size(r(C))
    assert need % 256 == 0 and need > 0
    assert call(lib, size=need - 1) == pp.PP_ERR_WORKSPACE
    assert lib.pp_kvq_workspace_size(None) == 0 and lib.pp_kvq_workspace_size(r(cache(head_dim=8))) == 0


@pytest.mark.parametrize("call", [append, commit])
def test_written_caches_have_entries_apart(lib, call):
    for kw in (dict(head_stride=64), dict(token_stride=512), dict(page_stride=1024), dict(v_scale=3 * A + 64)):
        assert call(lib, c=cache(**kw)) == pp.PP_ERR_INVALID_ARG, kw


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), pp.PP_ERR_INVALID_ARG), (dict(o=None), pp.PP_ERR_INVALID_ARG), (dict(k=0), pp.PP_ERR_INVALID_ARG),
    (dict(v=7 * A + 4), pp.PP_ERR_ALIGN), (dict(qs=4095), pp.PP_ERR_INVALID_ARG), (dict(ks=1028), pp.PP_ERR_ALIGN),
    (dict(o=5 * A + 64), pp.PP_ERR_INVALID_ARG), (dict(o=6 * A), pp.PP_ERR_INVALID_ARG), (dict(pos=A + 1), pp.PP_ERR_ALIGN),
    (dict(n=pp.pp_head_norm(-1.0, None, None)), pp.PP_ERR_INVALID_ARG), (dict(n=pp.pp_head_norm(0.1, A + 4, None)), pp.PP_ERR_ALIGN),
    (dict(rot=pp.pp_rotation(132, 0, 1.0, A)), pp.PP_ERR_SHAPE), (dict(rot=pp.pp_rotation(64, 3, 1.0, A)), pp.PP_ERR_INVALID_ARG)])
def test_append_refusals(lib, kw, want):
    assert append(lib, **kw) == want


@pytest.mark.parametrize("kw,want", [(dict(k=0), pp.PP_ERR_INVALID_ARG), (dict(v=6 * A), pp.PP_ERR_INVALID_ARG),
                                     (dict(ks=1023), pp.PP_ERR_INVALID_ARG), (dict(vs=1028), pp.PP_ERR_ALIGN)])
def test_read_refusals(lib, kw, want):
    assert read(lib, **kw) == want


@pytest.mark.parametrize("kw,want", [(dict(scale=0.0), pp.PP_ERR_INVALID_ARG), (dict(scale=float("nan")), pp.PP_ERR_INVALID_ARG),
                                     (dict(mask=A, words=0), pp.PP_ERR_INVALID_ARG), (dict(mask=A + 2, words=1), pp.PP_ERR_ALIGN),
                                     (dict(o=5 * A), pp.PP_ERR_INVALID_ARG), (dict(q=0), pp.PP_ERR_INVALID_ARG)])
def test_attention_refusals(lib, kw, want):
    assert attend(lib, **kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(layers=0), pp.PP_ERR_SHAPE), (dict(mp=-1), pp.PP_ERR_SHAPE), (dict(layers=2, ls=10 * PAGE, sls=159), pp.PP_ERR_INVALID_ARG),
    (dict(layers=2, ls=10 * PAGE - 16, sls=160), pp.PP_ERR_INVALID_ARG), (dict(layers=2, ls=10 * PAGE + 8, sls=160), pp.PP_ERR_ALIGN),
    (dict(layers=2, ls=10 * PAGE, sls=-1), pp.PP_ERR_INVALID_ARG), (dict(path=None), pp.PP_ERR_INVALID_ARG),
    (dict(acc=None), pp.PP_ERR_INVALID_ARG), (dict(new=2 * A), pp.PP_ERR_INVALID_ARG), (dict(new=3 * A + 1), pp.PP_ERR_ALIGN)])
def test_commit_refusals(lib, kw, want):
    assert commit(lib, **kw) == want


def test_binding_refuses_wrong_tensors(lib):
    import torch
    code = torch.zeros((3, 32, 2, 64), dtype=torch.uint8)
    s = torch.ones((3, 2, 2))
    ok = pp.KVCache8(code, code.clone(), s, s.clone(), 4, torch.bfloat16)
    assert ok.block == 16
    assert pp.KVCache8.empty(3, 32, 4, 2, 64, torch.float32, 32, device="cpu").k_scale.shape == (3, 2, 1)
    for bad in ((code, code[:2], s, s), (code.float(), code.float(), s, s), (code, code, s.double(), s.double()),
                (code, code, s[:, :, :1], s), (code, code, torch.ones(3, 2, 3), torch.ones(3, 2, 3)),
                (code, code, torch.ones(3, 2, 4)[..., ::2], s), (code, code.transpose(1, 2).contiguous().transpose(1, 2), s, s)):
        with pytest.raises(pp.PPError):
            pp.KVCache8(*bad, 4, torch.bfloat16)
    with pytest.raises(pp.PPError):
        pp.KVCache8(code, code, s, s, 4, torch.float16)
    with pytest.raises(pp.PPError):
        pp.KVCache8.empty(3, 30, 4, 2, 64, torch.float32, 16, device="cpu")
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)
    b = pp.Batch(i32(0, 2), i32(5), torch.zeros((1, 2), dtype=torch.int32), 2)
    ws, kv = torch.zeros(256, dtype=torch.uint8), torch.zeros((2, 2, 64), dtype=torch.bfloat16)
    for bad in (kv.float(), kv[:1], kv[:, :1]):
        with pytest.raises(pp.PPError):
            pp.pp_kvq_read(ok, b, bad, kv.clone(), ws, stream=0)
        with pytest.raises(pp.PPError):
            pp.pp_kvq_append(ok, b, None, None, None, None, kv, bad, None, ws, stream=0)
    with pytest.raises(pp.PPError):
        pp.pp_kvq_append(ok, b, pp.HeadNorm(torch.ones(64)), None, None, None, kv, kv, None, ws, stream=0)
    with pytest.raises(pp.PPError):
        pp.pp_kvq_commit(ok, b, i32(0, 1)[None], i32(1, 1), ws, stream=0)


def test_restated_codes_against_torch():
    import torch
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(20000) * np.exp2(rng.uniform(-12, 6, 20000)), ref.VALUES[:127], -ref.VALUES[:127],
                        (ref.VALUES[:126] + ref.VALUES[1:127]) / 2, [0.0, -0.0]])  # halfway between all neighbours
    x = np.clip(x, -448, 448).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ref.codes_of(x), want)
    assert (ref.codes_of(np.array([np.nan, np.inf, -np.inf])) == 0x7f).all()
    for a, e in ((448.0, 0), (448.01, 1), (224.0, -1), (224.1, 0), (0.0, -60), (1e-30, -60), (1.0, -8), (1.75, -8), (1.76, -7)):
        assert ref.scale_for(np.array(a)) == 2.0 ** e, a


def test_restated_append_and_commit():
    """Hand cases: a block that keeps its scale, one that grows, one without cached entries; a path across blocks."""
    code = np.zeros((2, 32, 1, 16), np.uint8)
    scale = np.full((2, 1, 2), 99.0, np.float32)
    c = ref.Cache(code, scale, 16)
    table = [1, 0]
    x = np.ones((20, 1, 16))
    c.append(table, 0, x)
    assert c.scale[1].tolist() == [[2.0 ** -8, 2.0 ** -8]] and (c.entry(table, 19) == 1).all()
    c.append(table, 20, 0.5 * x[:2])
    assert c.scale[1, 0, 1] == 2.0 ** -8 and (c.entry(table, 21) == 0.5).all()
    c.append(table, 22, 4.0 * x[:12])  # entries 22..31, then 32, 33 of the next page
    assert c.scale[1, 0, 1] == 2.0 ** -6 and c.scale[0, 0, 0] == 2.0 ** -6
    assert (c.entry(table, 17) == 1).all() and (c.entry(table, 21) == 0.5).all() and (c.entry(table, 33) == 4).all()
    c.append(table, 20, 0.25 * x[:14])  # a tree of 14 drafts behind 20 entries; 17, 18 stay in the grown block
    assert c.scale[1, 0, 1] == 2.0 ** -6 and c.scale[0, 0, 0] == 2.0 ** -10
    c.commit(table, 20, [0, 12, 13])
    assert [float(c.entry(table, e)[0, 0]) for e in (19, 20, 21, 22)] == [1.0, 0.25, 0.25, 0.25]
    assert c.scale[1, 0, 1] == 2.0 ** -6
