"""GPU tests of the head norms with rotation and their gradients against the
fp64 restatement (norm_ref) within its derived bounds."""
import numpy as np
import pytest

import norm_ref as ref
from test_gpu_attention import rounded, to_dev
from test_gpu_cache import POSITIONS, freqs
from test_gpu_canaries import Guarded

pytestmark = pytest.mark.gpu

SHAPES = [(1, 0, 8, 8), (3, 1, 64, 64), (2, 2, 64, 16), (5, 5, 80, 20), (2, 1, 128, 128), (4, 2, 96, 12), (32, 8, 128, 64),
          (2, 2, 256, 256), (3, 3, 256, 4), (1, 1, 128, 4), (40, 40, 128, 0), (6, 2, 24, 8), (7, 7, 200, 100)]


class Data:
    def __init__(self, T, H, Hkv, D, rot, dtype, seed=0, gamma=True, pos=None, std=1.7):
        rng = np.random.default_rng(seed)
        self.dtype, self.rot = dtype, rot
        self.x = [rounded(rng.standard_normal((T, n, D)) * std, dtype) for n in (H, Hkv)]
        self.dy = [rounded(rng.standard_normal((T, n, D)), dtype) for n in (H, Hkv)]
        self.gamma = [rounded(1 + 0.3 * rng.standard_normal(D), dtype) if gamma else None for _ in range(2)]
        self.pos = np.array(pos if pos is not None else rng.integers(0, 5000, T), np.int32)
        self.freq = freqs(rot) if rot else None

    def handles(self, pp, layout, scale, eps):
        norm = pp.HeadNorm(*[None if g is None else to_dev(g, self.dtype) for g in self.gamma], eps)
        return norm, pp.Rotation(to_dev(self.freq), layout, scale) if self.rot else None

    def want(self, which, eps, layout, scale):
        a = (self.x[which], self.gamma[which], eps)
        y = ref.forward(*a, self.pos, self.freq, layout, scale)
        return y, ref.forward_bound(*a, self.freq, layout, scale, self.dtype, y)

    def want_grad(self, which, eps, layout, scale, per_thread):
        a = (self.x[which], self.gamma[which], eps)
        dx, dg = ref.backward(*a, self.pos, self.freq, layout, scale, self.dy[which])
        return (dx, dg), ref.backward_bound(*a, self.freq, layout, scale, self.dy[which], self.dtype, dx, per_thread)


def within(got, want, tol):
    got = got.float().cpu().numpy()
    assert np.isfinite(got).all()
    off = np.abs(got - want) - tol
    assert off.max(initial=-1.0) <= 0, (float(off.max()), np.unravel_index(off.argmax(), off.shape))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("H,Hkv,D,rot", SHAPES)
def test_forward(pp, dtype, layout, H, Hkv, D, rot):
    import torch
    d = Data(len(POSITIONS), H, Hkv, D, rot, dtype, seed=D + H, pos=POSITIONS)
    for scale, eps in ((1.0, 1e-6), (1.375, 0.25)):
        norm, r = d.handles(pp, layout, scale, eps)
        q, k = to_dev(d.x[0], dtype), to_dev(d.x[1], dtype) if Hkv else None
        qo, ko = torch.full_like(q, 9.0), None if k is None else torch.full_like(k, 9.0)
        pp.pp_head_norm_rope(norm, r, to_dev(d.pos), q, k, qo, ko)
        for i, got in enumerate((qo, ko)[:1 + (Hkv > 0)]):
            within(got, *d.want(i, eps, layout, scale))
        # in place: the same bits
        pp.pp_head_norm_rope(norm, r, to_dev(d.pos), q, k, q, k)
        assert torch.equal(q.view(torch.uint8), qo.view(torch.uint8))
        assert k is None or torch.equal(k.view(torch.uint8), ko.view(torch.uint8))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("H,Hkv,D,rot", SHAPES)
def test_backward(pp, dtype, layout, H, Hkv, D, rot):
    import torch
    d = Data(len(POSITIONS), H, Hkv, D, rot, dtype, seed=D + H + 1, pos=POSITIONS)
    norm, r = d.handles(pp, layout, 1.375, 1e-5)
    q, k, gq, gk = (to_dev(a, dtype) for a in d.x + d.dy)
    dq, dk = torch.full_like(q, 9.0), torch.full_like(k, 9.0)
    dgq, dgk = (torch.full((D,), 9.0, device="cuda") for _ in range(2))
    ws = pp.alloc_head_norm_workspace(D)
    ws.fill_(0xff)
    args = (norm, r, to_dev(d.pos), q, k if Hkv else None, gq, gk if Hkv else None)
    pp.pp_head_norm_rope_grad(*args, dq, dk if Hkv else None, dgq, dgk, ws)
    for i, (dx, dg) in enumerate(((dq, dgq), (dk, dgk))[:1 + (Hkv > 0)]):
        # a thread has its rows of up to all tokens
        (wx, wg), (tx, tg) = d.want_grad(i, 1e-5, layout, 1.375, len(POSITIONS) * (H, Hkv)[i])
        within(dx, wx, tx)
        within(dg, wg, tg)
    if Hkv == 0:
        assert (dgk == 0).all()
    # the gradients over those that came in, and one weight gradient alone: the same bits
    only = torch.full((D,), 9.0, device="cuda")
    pp.pp_head_norm_rope_grad(*args, gq, gk if Hkv else None, None, only, ws)
    assert torch.equal(gq, dq) and (Hkv == 0 or torch.equal(gk, dk)) and torch.equal(only, dgk)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_tokens_strides_and_no_weights(pp, dtype):
    import torch
    T, H, Hkv, D, rot = 1500, 6, 2, 64, 32
    d = Data(T, H, Hkv, D, rot, dtype, gamma=False)
    norm, r = d.handles(pp, "half", 1.0, 1e-6)
    # the parts of one projection, with other columns behind them
    wide = torch.full((T, H + Hkv + 3, D), 5.0, device="cuda", dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
    wide[:, :H], wide[:, H:H + Hkv] = to_dev(d.x[0], dtype), to_dev(d.x[1], dtype)
    q, k = wide[:, :H], wide[:, H:H + Hkv]
    grads = [to_dev(a, dtype) for a in d.dy]
    dq, dk = (torch.empty_like(g) for g in grads)
    dg = torch.empty(2, D, device="cuda")
    ws = pp.alloc_head_norm_workspace(D)
    pp.pp_head_norm_rope_grad(norm, r, to_dev(d.pos), q, k, *grads, dq, dk, dg[0], dg[1], ws)
    again = torch.empty_like(dg)
    pp.pp_head_norm_rope_grad(norm, r, to_dev(d.pos), q, k, *grads, dq, dk, again[0], again[1], ws)
    assert torch.equal(dg, again)
    for i, (x, g) in enumerate(((dq, dg[0]), (dk, dg[1]))):
        # at least 70 CTAs a tensor: a thread has at most T / 70 tokens, rounded up, of up to 6 heads
        (wx, wg), (tx, tg) = d.want_grad(i, 1e-6, "half", 1.0, (T // 70 + 1) * 6)
        within(x, wx, tx)
        within(g, wg, tg)
    pp.pp_head_norm_rope(norm, r, to_dev(d.pos), q, k, q, k)
    within(q, *d.want(0, 1e-6, "half", 1.0))
    within(k, *d.want(1, 1e-6, "half", 1.0))
    assert (wide[:, H + Hkv:] == 5.0).all()


def test_no_tokens(pp):
    import torch
    norm = pp.HeadNorm(torch.ones(64, device="cuda"), None)
    q, k = torch.empty(0, 4, 64, device="cuda"), torch.empty(0, 2, 64, device="cuda")
    pp.pp_head_norm_rope(norm, None, None, q, k, q, k)
    dg = torch.full((2, 64), 3.0, device="cuda")
    pp.pp_head_norm_rope_grad(norm, None, None, q, k, q, k, q, k, dg[0], dg[1], pp.alloc_head_norm_workspace(64))
    assert (dg == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradient_against_differences(pp, dtype):
    """The kernel's gradients against differences of the restated forward pass in fp64, in random directions: both
    bounds weighted by the direction, and 1e-4 for the difference itself (h^2 times third derivatives of the sum)."""
    import torch
    T, H, Hkv, D, rot = 7, 3, 2, 128, 64
    d = Data(T, H, Hkv, D, rot, dtype, seed=5)
    norm, r = d.handles(pp, "half", 1.0, 1e-5)
    q, k, gq, gk = (to_dev(a, dtype) for a in d.x + d.dy)
    dq, dk = torch.empty_like(q), torch.empty_like(k)
    dg = torch.empty(2, D, device="cuda")
    pp.pp_head_norm_rope_grad(norm, r, to_dev(d.pos), q, k, gq, gk, dq, dk, dg[0], dg[1], pp.alloc_head_norm_workspace(D))
    rng = np.random.default_rng(1)
    for i, (dx, dgi) in enumerate(((dq, dg[0]), (dk, dg[1]))):
        _, (tx, tg) = d.want_grad(i, 1e-5, "half", 1.0, T * 3)
        loss = lambda x, g: (ref.forward(x, g, 1e-5, d.pos, d.freq, "half", 1.0) * d.dy[i]).sum()
        x, g = d.x[i].astype(np.float64), d.gamma[i].astype(np.float64)
        for _ in range(5):
            v, w, h = rng.standard_normal(x.shape), rng.standard_normal(D), 1e-4
            diff = (loss(x + h * v, g) - loss(x - h * v, g)) / (2 * h)
            assert abs(diff - (dx.double().cpu().numpy() * v).sum()) <= (tx * np.abs(v)).sum() + 1e-4
            diff = (loss(x, g + h * w) - loss(x, g - h * w)) / (2 * h)
            assert abs(diff - (dgi.double().cpu().numpy() * w).sum()) <= (tg * np.abs(w)).sum() + 1e-4


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bands_graphs_and_streams(pp, dtype):
    import torch
    T, H, Hkv, D, rot = 5, 4, 1, 80, 40
    d = Data(T, H, Hkv, D, rot, dtype, seed=2)
    norm, r = d.handles(pp, "interleaved", 1.0, 1e-6)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q, k, gq, gk = (to_dev(a, dtype) for a in d.x + d.dy)
    out = [Guarded((T, H, D), dt), Guarded((T, Hkv, D), dt), Guarded((T, H, D), dt), Guarded((T, Hkv, D), dt),
           Guarded((D,), torch.float32), Guarded((D,), torch.float32)]
    ws = Guarded((pp.pp_head_norm_workspace_size(D),), torch.uint8)
    pos = to_dev(d.pos)

    def both(stream=None):
        pp.pp_head_norm_rope(norm, r, pos, q, k, out[0].t, out[1].t, stream=stream)
        pp.pp_head_norm_rope_grad(norm, r, pos, q, k, gq, gk, out[2].t, out[3].t, out[4].t, out[5].t, ws.t, stream=stream)
    both()
    torch.cuda.synchronize()
    assert all(g.bands_intact() for g in out + [ws])
    first = [g.t.clone() for g in out]
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for g in out:
        g.t.zero_()
    torch.cuda.synchronize()
    both(st)
    torch.cuda.synchronize()
    assert all(torch.equal(g.t, f) for g, f in zip(out, first))
    q.copy_(-q)  # the output and dgamma change sign, dq does not
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[0].t, -first[0]) and torch.equal(out[4].t, -first[4])
    assert torch.equal(out[1].t, first[1]) and torch.equal(out[2].t, first[2])
