"""Norms of query and key heads: refusals (before any CUDA call), and the
restated gradient against differences of the restated forward pass."""
import ctypes

import numpy as np
import pytest

import norm_ref
from paper_2605_28283_gb300 import binding as pp
from paper_2605_28283_gb300 import build as ppbuild

A = 0x100000  # an aligned address; nothing dereferences it: every call here is refused
F = dict(T=4, H=4, Hkv=2, D=128)


@pytest.fixture(scope="module")
def lib():
    ppbuild.build()
    return pp.load()


def ref(x):
    return None if x is None else ctypes.byref(x)


def norm(eps=1e-6, qg=A, kg=A):
    return pp.pp_head_norm(eps, qg, kg)


def rot(**kw):
    d = dict(rot_dim=128, layout=0, scale=1.0, inv_freq=A)
    d.update(kw)
    return pp.pp_rotation(*[d[n] for n, _ in pp.pp_rotation._fields_])


def fwd(lib, dtype=pp.PP_BF16, n=norm(), r=rot(), pos=A, T=4, H=4, Hkv=2, D=128, q=A, qs=512, k=2 * A, ks=256, qo=3 * A,
        qos=512, ko=4 * A, kos=256):
    return lib.pp_head_norm_rope(dtype, ref(n), ref(r), pos, T, H, Hkv, D, q, qs, k, ks, qo, qos, ko, kos, None)


def bwd(lib, dtype=pp.PP_BF16, n=norm(), r=rot(), pos=A, T=4, H=4, Hkv=2, D=128, q=A, qs=512, k=2 * A, ks=256, gq=3 * A,
        gqs=512, gk=4 * A, gks=256, dq=5 * A, dqs=512, dk=6 * A, dks=256, dgq=7 * A, dgk=8 * A, ws=9 * A, n_ws=1 << 30):
    return lib.pp_head_norm_rope_grad(dtype, ref(n), ref(r), pos, T, H, Hkv, D, q, qs, k, ks, gq, gqs, gk, gks, dq, dqs,
                                      dk, dks, dgq, dgk, ws, n_ws, None)


COMMON = [(dict(dtype=7), pp.PP_ERR_DTYPE), (dict(H=0), pp.PP_ERR_SHAPE), (dict(Hkv=-1), pp.PP_ERR_SHAPE),
          (dict(T=-1), pp.PP_ERR_SHAPE), (dict(D=260), pp.PP_ERR_SHAPE), (dict(D=132, r=None), pp.PP_ERR_SHAPE),
          (dict(n=None), pp.PP_ERR_INVALID_ARG), (dict(n=norm(eps=-1.0)), pp.PP_ERR_INVALID_ARG),
          (dict(n=norm(eps=float("nan"))), pp.PP_ERR_INVALID_ARG), (dict(n=norm(eps=float("inf"))), pp.PP_ERR_INVALID_ARG),
          (dict(n=norm(qg=A + 8)), pp.PP_ERR_ALIGN), (dict(pos=None), pp.PP_ERR_INVALID_ARG), (dict(pos=A + 2), pp.PP_ERR_ALIGN),
          (dict(r=rot(rot_dim=132)), pp.PP_ERR_SHAPE), (dict(r=rot(layout=4)), pp.PP_ERR_INVALID_ARG),
          (dict(r=rot(inv_freq=0)), pp.PP_ERR_INVALID_ARG), (dict(q=None), pp.PP_ERR_INVALID_ARG),
          (dict(k=None), pp.PP_ERR_INVALID_ARG), (dict(q=A + 4), pp.PP_ERR_ALIGN), (dict(qs=511), pp.PP_ERR_INVALID_ARG),
          (dict(qs=516), pp.PP_ERR_ALIGN), (dict(ks=128), pp.PP_ERR_INVALID_ARG)]


@pytest.mark.parametrize("kw,want", COMMON)
def test_both_directions_refuse(lib, kw, want):
    assert fwd(lib, **kw) == want
    assert bwd(lib, **kw) == want


@pytest.mark.parametrize("kw", [dict(qo=A + 16), dict(qo=2 * A), dict(ko=A), dict(ko=3 * A), dict(ko=2 * A + 128),
                                dict(qo=A, qos=1024)])
def test_forward_refuses_overlaps(lib, kw):
    assert fwd(lib, **kw) == pp.PP_ERR_INVALID_ARG


@pytest.mark.parametrize("kw,want", [(dict(dq=A + 16), pp.PP_ERR_INVALID_ARG), (dict(dq=4 * A), pp.PP_ERR_INVALID_ARG),
                                     (dict(dk=5 * A), pp.PP_ERR_INVALID_ARG), (dict(dk=3 * A), pp.PP_ERR_INVALID_ARG),
                                     (dict(dgq=8 * A), pp.PP_ERR_INVALID_ARG), (dict(dgk=A + 64), pp.PP_ERR_INVALID_ARG),
                                     (dict(dgk=5 * A), pp.PP_ERR_INVALID_ARG), (dict(dgq=9 * A), pp.PP_ERR_INVALID_ARG),
                                     (dict(dgq=7 * A + 2), pp.PP_ERR_ALIGN), (dict(ws=None), pp.PP_ERR_WORKSPACE),
                                     (dict(ws=9 * A + 64), pp.PP_ERR_WORKSPACE), (dict(n_ws=1000), pp.PP_ERR_WORKSPACE)])
def test_backward_refuses(lib, kw, want):
    assert bwd(lib, **kw) == want


def test_workspace_size(lib):
    assert pp.pp_head_norm_workspace_size(128) >= 128 * 4 and pp.pp_head_norm_workspace_size(128) % 256 == 0
    for bad in (0, -4, 6, 260):
        assert pp.pp_head_norm_workspace_size(bad) == 0


def test_binding_refuses_wrong_tensors(lib):
    import torch
    q, k = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    g = torch.ones(64, dtype=torch.bfloat16)
    pos = torch.zeros(3, dtype=torch.int32)
    freq = pp.Rotation(torch.ones(32))
    good = dict(norm=pp.HeadNorm(g, g), rot=freq, positions=pos, q=q, k=k, q_out=q, k_out=k, stream=0)

    def call(**kw):
        with pytest.raises(pp.PPError) as e:
            pp.pp_head_norm_rope(**{**good, **kw})
        return e.value.status
    assert call(norm=pp.HeadNorm(g.float(), None)) == pp.PP_ERR_DTYPE
    assert call(norm=pp.HeadNorm(None, g[:32])) == pp.PP_ERR_SHAPE
    assert call(positions=None) == pp.PP_ERR_INVALID_ARG
    assert call(positions=pos[:2]) == pp.PP_ERR_SHAPE
    assert call(positions=pos.long()) == pp.PP_ERR_DTYPE
    assert call(q=q[0]) == pp.PP_ERR_SHAPE
    assert call(k=k[:2]) == pp.PP_ERR_SHAPE
    assert call(k=k.float()) == pp.PP_ERR_DTYPE
    assert call(q_out=q.transpose(0, 1)) == pp.PP_ERR_SHAPE
    for bad in (torch.ones(2, 64), torch.ones(128)[::2]):
        with pytest.raises(pp.PPError):
            pp.HeadNorm(bad, None)
    with pytest.raises(pp.PPError) as e:
        pp.pp_head_norm_rope_grad(pp.HeadNorm(g, g), freq, pos, q, k, q, k, q.clone(), k.clone(), torch.zeros(64, dtype=torch.bfloat16),
                                  None, torch.zeros(1 << 20, dtype=torch.uint8), stream=0)
    assert e.value.status == pp.PP_ERR_DTYPE


@pytest.mark.parametrize("layout,rot_dim", [("half", 16), ("interleaved", 8), (None, 0)])
def test_restated_gradient_against_differences(layout, rot_dim):
    rng = np.random.default_rng(3)
    T, H, D = 2, 3, 16
    x, dy, gamma = rng.standard_normal((T, H, D)), rng.standard_normal((T, H, D)), 1 + 0.3 * rng.standard_normal(D)
    pos = np.array([5, 70])
    freq = None if layout is None else 100.0 ** (-2.0 * np.arange(rot_dim // 2) / rot_dim)
    args = (1e-5, pos, freq, layout or "half", 1.25)
    dx, dg = norm_ref.backward(x, gamma, *args, dy)
    loss = lambda x, gamma: (norm_ref.forward(x, gamma, *args) * dy).sum()
    for got, which in ((dx, 0), (dg, 1)):
        for _ in range(20):
            v = rng.standard_normal(got.shape)
            h = 1e-5
            hi, lo = (loss(x + s * h * v, gamma) if which == 0 else loss(x, gamma + s * h * v) for s in (1, -1))
            # the second difference's error is h^2 times third derivatives of order 10, and 2^-52 / h of values of order 10
            assert abs((hi - lo) / (2 * h) - (got * v).sum()) < 1e-7
