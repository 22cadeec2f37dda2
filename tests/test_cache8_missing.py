"""Calls of the 8-bit cache and of the head norms that leave a tensor or handle out: the binding's own error, with the
documented status (no GPU)."""
import pytest

from paper_2605_28283_gb300 import binding as pp
from paper_2605_28283_gb300 import build as ppbuild


@pytest.fixture(scope="module")
def lib():
    ppbuild.build()
    return pp.load()


def status(call, good, **kw):
    with pytest.raises(pp.PPError) as e:
        call(**{**good, **kw})
    return e.value.status


def heads():
    import torch
    q, k = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    g = torch.ones(64, dtype=torch.bfloat16)
    return dict(norm=pp.HeadNorm(g, g), rot=pp.Rotation(torch.ones(32)), positions=torch.zeros(3, dtype=torch.int32), q=q, k=k, stream=0)


@pytest.mark.parametrize("name", ["norm", "positions", "q", "q_out", "k_out"])
def test_head_norm(lib, name):
    h = heads()
    good = dict(h, q_out=h["q"], k_out=h["k"])
    assert status(pp.pp_head_norm_rope, good, **{name: None}) == pp.PP_ERR_INVALID_ARG


@pytest.mark.parametrize("name", ["norm", "positions", "q", "q_grad", "k_grad", "dq", "dk"])
def test_head_norm_gradients(lib, name):
    h = heads()
    good = dict(h, q_grad=h["q"].clone(), k_grad=h["k"].clone(), dq=h["q"].clone(), dk=h["k"].clone(), dq_gamma=None, dk_gamma=None,
                ws=None)
    assert status(pp.pp_head_norm_rope_grad, good, **{name: None}) == pp.PP_ERR_INVALID_ARG


def steps():
    import torch
    code, scale = torch.zeros((2, 3, 32, 2, 64), dtype=torch.uint8), torch.ones((2, 3, 2, 2))
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)
    kv, q = torch.zeros((2, 2, 64), dtype=torch.bfloat16), torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    base = dict(cache=pp.KVCache8(*code, *scale, 4, torch.bfloat16), ws=torch.zeros(256, dtype=torch.uint8), stream=0,
                batch=pp.Batch(i32(0, 2), i32(5), torch.zeros((1, 2), dtype=torch.int32), 2))
    return {pp.pp_kvq_append: dict(base, norm=None, rot=None, positions=None, q=None, k=kv, v=kv, q_out=None),
            pp.pp_kvq_read: dict(base, k_out=kv, v_out=kv.clone()),
            pp.pp_kvq_tree_attention: dict(base, q=q, mask=None, scale=0.1, out=q.clone()),
            pp.pp_kvq_commit: dict(base, path=i32(0, 1)[None], n_accept=i32(1))}


@pytest.mark.parametrize("call,names", [("pp_kvq_append", "kv"), ("pp_kvq_read", ["k_out", "v_out"]),
                                        ("pp_kvq_tree_attention", ["q", "out"]), ("pp_kvq_commit", ["path", "n_accept"])])
def test_steps_of_the_cache(lib, call, names):
    call = getattr(pp, call)
    good = steps()[call]
    for name in names:
        assert status(call, good, **{name: None}) == pp.PP_ERR_INVALID_ARG, name
    assert status(call, good, ws=None) == pp.PP_ERR_WORKSPACE
