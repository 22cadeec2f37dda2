"""Tensors of several devices: handles and calls of the 8-bit cache and of the head norms refuse them, and tensors on the
CPU, before anything is launched.  No GPU is needed: a tensor that says that it is on another device stands in for one."""
import pytest
import torch

from paper_2605_28283_gb300 import binding as pp
from paper_2605_28283_gb300 import build as ppbuild


class Elsewhere(torch.Tensor):
    def get_device(self):
        return 7


class Here(torch.Tensor):
    def get_device(self):
        return 0


def there(t):
    return t.as_subclass(Elsewhere)


def here(t):
    return t.as_subclass(Here)


@pytest.fixture(scope="module")
def lib():
    ppbuild.build()
    return pp.load()


def refused(call, **kw):
    with pytest.raises(pp.PPError) as e:
        call(**kw)
    assert e.value.status == pp.PP_ERR_INVALID_ARG and "device" in str(e.value), str(e.value)


def parts(make):
    code, scale = torch.zeros((2, 3, 32, 2, 64), dtype=torch.uint8), torch.ones((2, 3, 2, 2))
    return [make(t) for t in (*code, *scale)]


def i32(*v):
    return torch.tensor(v, dtype=torch.int32)


def batch(make=here):
    return pp.Batch(make(i32(0, 2)), make(i32(5)), make(torch.zeros((1, 2), dtype=torch.int32)), 2)


@pytest.mark.parametrize("which", range(4))
def test_a_cache_of_two_devices(which):
    p = parts(here)
    p[which] = there(p[which])
    with pytest.raises(pp.PPError) as e:
        pp.KVCache8(*p, 4, torch.bfloat16)
    assert e.value.status == pp.PP_ERR_INVALID_ARG


def test_weights_of_two_devices():
    g = torch.ones(64, dtype=torch.bfloat16)
    with pytest.raises(pp.PPError) as e:
        pp.HeadNorm(here(g), there(g))
    assert e.value.status == pp.PP_ERR_INVALID_ARG
    assert pp.HeadNorm(None, None).device is None


def norm_call(make):
    g = torch.ones(64, dtype=torch.bfloat16)
    q, k = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    return dict(norm=pp.HeadNorm(make(g), make(g)), rot=pp.Rotation(make(torch.ones(32))), positions=make(i32(1, 2, 3)),
                q=make(q), k=make(k), stream=0)


@pytest.mark.parametrize("name", ["norm", "rot", "positions", "q", "k", "q_out", "k_out"])
def test_head_norm(lib, name):
    make = lambda m: (lambda c: dict(c, q_out=c["q"], k_out=c["k"]))(norm_call(m))
    refused(pp.pp_head_norm_rope, **{**make(here), name: make(there)[name]})
    refused(pp.pp_head_norm_rope, **make(lambda t: t))


@pytest.mark.parametrize("name", ["norm", "rot", "positions", "q", "k", "q_grad", "k_grad", "dq", "dk", "dq_gamma", "dk_gamma", "ws"])
def test_head_norm_gradients(lib, name):
    def make(m):
        c = norm_call(m)
        return dict(c, q_grad=c["q"], k_grad=c["k"], dq=c["q"], dk=c["k"], dq_gamma=m(torch.zeros(64)), dk_gamma=m(torch.zeros(64)),
                    ws=m(torch.zeros(256, dtype=torch.uint8)))
    refused(pp.pp_head_norm_rope_grad, **{**make(here), name: make(there)[name]})
    refused(pp.pp_head_norm_rope_grad, **make(lambda t: t))


def step(call, m):
    kv, q = torch.zeros((2, 2, 64), dtype=torch.bfloat16), torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    c = dict(cache=pp.KVCache8(*parts(m), 4, torch.bfloat16), batch=batch(m), ws=m(torch.zeros(256, dtype=torch.uint8)), stream=0)
    g = torch.ones(64, dtype=torch.bfloat16)
    return dict(c, **{
        "pp_kvq_append": dict(norm=pp.HeadNorm(m(g), None), rot=pp.Rotation(m(torch.ones(32))), positions=m(i32(1, 2)), q=m(q), k=m(kv),
                              v=m(kv), q_out=m(q)),
        "pp_kvq_read": dict(k_out=m(kv), v_out=m(kv.clone())),
        "pp_kvq_tree_attention": dict(q=m(q), mask=m(i32(1, 3)[:, None]), scale=0.1, out=m(q.clone())),
        "pp_kvq_commit": dict(path=m(i32(0, 1)[None]), n_accept=m(i32(1)), new_len=m(i32(0)))}[call])


@pytest.mark.parametrize("call", ["pp_kvq_append", "pp_kvq_read", "pp_kvq_tree_attention", "pp_kvq_commit"])
def test_steps_of_the_cache(lib, call):
    good, other = step(call, here), step(call, there)
    for name in good:
        if name not in ("stream", "scale"):
            refused(getattr(pp, call), **{**good, name: other[name]})
    refused(getattr(pp, call), **step(call, lambda t: t))


def test_a_batch_of_two_devices(lib):
    for i in range(3):
        t = [i32(0, 2), i32(5), torch.zeros((1, 2), dtype=torch.int32)]
        t = [there(x) if n == i else here(x) for n, x in enumerate(t)]
        refused(pp.pp_kvq_read, **{**step("pp_kvq_read", here), "batch": pp.Batch(*t, 2)})
