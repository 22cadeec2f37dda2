"""GPU tests of rotary positions, the append to the paged cache and the commit
of accepted paths, against fp64 restatements (attn_ref) and plain indexing."""
import numpy as np
import pytest

import attn_ref as ref
from test_gpu_attention import rounded, to_dev

pytestmark = pytest.mark.gpu


def freqs(rot, base=10000.0):
    return np.array([base ** (-2.0 * i / rot) for i in range(rot // 2)], np.float32)


POSITIONS = [0, 1, 2, 4095, 4096, 4097, 131071, 1 << 20, (1 << 24) + 1, (1 << 30) + 12345, 2 ** 31 - 1, -1, -70000]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("heads,dim,rot", [(1, 8, 8), (3, 64, 64), (2, 64, 16), (5, 80, 20), (2, 128, 128), (4, 96, 12),
                                           (32, 128, 64), (2, 256, 256), (1, 128, 4)])
@pytest.mark.parametrize("inverse", [False, True])
def test_rope(pp, dtype, layout, heads, dim, rot, inverse):
    import torch
    rng = np.random.default_rng(rot + heads)
    pos = np.array(POSITIONS, np.int32)
    x = rounded(rng.standard_normal((len(pos), heads, dim)), dtype)
    f = freqs(rot)
    for scale in (1.0, 1.375):
        r = pp.Rotation(to_dev(f), layout, scale)
        xd = to_dev(x, dtype)
        y = torch.full_like(xd, 9.0)
        pp.pp_rope(r, to_dev(pos), xd, y, inverse=inverse)
        want = ref.rotate(x, pos, f, layout, scale, inverse)
        tol = ref.rotate_bound(x, f, layout, scale, dtype, want)
        got = y.float().cpu().numpy()
        assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) - tol).max())
        # in place: the same bits
        pp.pp_rope(r, to_dev(pos), xd, xd, inverse=inverse)
        assert torch.equal(xd.view(torch.uint8), y.view(torch.uint8))


def test_rope_many_tokens_and_strides(pp):
    import torch
    T, heads, dim = 1111, 6, 64
    rng = np.random.default_rng(0)
    wide = rounded(rng.standard_normal((T, heads + 3, dim)), "bf16")
    pos = rng.integers(0, 100000, T).astype(np.int32)
    f = freqs(dim)
    buf = to_dev(wide, "bf16")
    y = torch.full((T, heads, dim + 0), 1.0, dtype=torch.bfloat16, device="cuda")
    pp.pp_rope(pp.Rotation(to_dev(f)), to_dev(pos), buf[:, 2:2 + heads], y)
    want = ref.rotate(wide[:, 2:2 + heads], pos, f, "half")
    tol = ref.rotate_bound(wide[:, 2:2 + heads], f, "half", 1.0, "bf16", want)
    assert (np.abs(y.float().cpu().numpy() - want) <= tol).all()
    assert np.array_equal(buf.float().cpu().numpy(), wide)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_gradient(pp, layout):
    """The rotation back is the gradient: against the fp64 formula of L = sum(w . rope(x)) and against central
    differences of the operator itself (the rotation is linear, so a step of 1/2 leaves only fp32 rounding:
    2 * 64 * 2^-24 * |w| * |y| over the sum, below 2e-4 for 64 elements of unit size)."""
    import torch
    rng = np.random.default_rng(4)
    T, H, D, rot, scale = 3, 2, 16, 12, 1.25
    pos = np.array([5, 77, 3000], np.int32)
    f = freqs(rot)
    r = pp.Rotation(to_dev(f), layout, scale)
    x = rng.standard_normal((T, H, D)).astype(np.float32)
    w = rng.standard_normal((T, H, D)).astype(np.float32)
    g = torch.empty((T, H, D), device="cuda")
    pp.pp_rope(r, to_dev(pos), to_dev(w), g, inverse=True)
    g = g.cpu().numpy().astype(np.float64)
    # formula: R^T w, with R written out pair by pair
    want = w.astype(np.float64).copy()
    for t in range(T):
        for i in range(rot // 2):
            a, b = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
            c, s = np.cos(float(pos[t]) * float(f[i])), np.sin(float(pos[t]) * float(f[i]))
            wa, wb = w[t, :, a].astype(np.float64), w[t, :, b].astype(np.float64)
            want[t, :, a], want[t, :, b] = scale * (wa * c + wb * s), scale * (wb * c - wa * s)
    assert (np.abs(g - want) <= ref.rotate_bound(w, f, layout, scale, "f32", want)).all()

    def loss(v):
        y = torch.empty((T, H, D), device="cuda")
        pp.pp_rope(r, to_dev(pos), to_dev(v.astype(np.float32)), y)
        return float((y.cpu().numpy().astype(np.float64) * w).sum())

    for _ in range(12):
        at = tuple(int(rng.integers(0, k)) for k in (T, H, D))
        d = np.zeros_like(x)
        d[at] = 0.5
        assert abs(loss(x + d) - loss(x - d) - g[at]) <= 2e-4


class AppendCase:
    def __init__(self, seqs, heads, kv_heads, dim, page, dtype, rot, layout, order="token", pad=0, seed=0):
        rng = np.random.default_rng(seed)
        self.dtype, self.page, self.heads, self.layout = dtype, page, heads, layout
        n = [s[0] for s in seqs]
        self.ctx = np.array([s[1] for s in seqs], np.int32)
        self.starts = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        self.used = int(self.starts[-1])
        self.T = self.used + pad
        per = [-(-(a + c) // page) for a, c in seqs]
        perm = rng.permutation(sum(per) + 2).astype(np.int32)
        self.pages = np.full((len(seqs), max(per + [1])), -1, np.int32)
        at = 0
        for b, k in enumerate(per):
            self.pages[b, :k] = perm[at:at + k]
            at += k
        shape = (len(perm), page, kv_heads, dim)
        self.k0, self.v0 = (rounded(rng.standard_normal(shape), dtype) for _ in range(2))
        self.q = rounded(rng.standard_normal((self.T, heads, dim)), dtype)
        self.k, self.v = (rounded(rng.standard_normal((self.T, kv_heads, dim)), dtype) for _ in range(2))
        self.freq = freqs(rot) if rot else None
        self.order = order
        self.default_pos = np.concatenate([c + np.arange(a) for a, c in seqs] + [np.zeros(pad, int)]).astype(np.int32)

    def device(self, pp):
        k, v = to_dev(self.k0, self.dtype), to_dev(self.v0, self.dtype)
        if self.order == "head":
            k, v = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in (k, v))
        cache = pp.KVCache(k, v, self.heads)
        batch = pp.Batch(to_dev(self.starts), to_dev(self.ctx), to_dev(self.pages), self.T)
        rot = None if self.freq is None else pp.Rotation(to_dev(self.freq), self.layout)
        return cache, batch, rot

    def want(self, pos):
        """(q_out, keys, values, their bounds) of the whole cache."""
        if self.freq is None:
            q, k = self.q.astype(np.float64), self.k.astype(np.float64)
            tq, tk = np.zeros_like(q), np.zeros_like(k)
        else:
            q, k = (ref.rotate(a, pos, self.freq, self.layout) for a in (self.q, self.k))
            tq, tk = (ref.rotate_bound(a, self.freq, self.layout, 1.0, self.dtype, r)
                      for a, r in ((self.q, q), (self.k, k)))
        kc, vc, tc = self.k0.astype(np.float64), self.v0.astype(np.float64), np.zeros_like(self.k0, np.float64)
        for b in range(len(self.ctx)):
            for i in range(int(self.starts[b + 1] - self.starts[b])):
                j, t = int(self.ctx[b]) + i, int(self.starts[b]) + i
                at = (self.pages[b, j // self.page], j % self.page)
                kc[at], vc[at], tc[at] = k[t], self.v[t], tk[t]
        return q, kc, vc, tq, tc

    def check(self, pp, pos=None):
        import torch
        cache, batch, rot = self.device(pp)
        ws = pp.alloc_attn_workspace(cache)
        q = to_dev(self.q, self.dtype)
        out = torch.full_like(q, 55.0)
        pp.pp_kv_append(cache, batch, rot, None if pos is None else to_dev(pos), q, to_dev(self.k, self.dtype),
                        to_dev(self.v, self.dtype), out, ws)
        torch.cuda.synchronize()
        assert pp.pp_get_device_status(ws) == pp.PP_OK
        wq, wk, wv, tq, tc = self.want(self.default_pos if pos is None else pos)
        gq = out.float().cpu().numpy()
        u = self.used
        assert (np.abs(gq[:u] - wq[:u]) <= tq[:u]).all()
        assert (gq[u:] == 55.0).all(), "padding rows were written"
        assert (np.abs(cache.k.float().cpu().numpy() - wk) <= tc).all()
        assert np.array_equal(cache.v.float().cpu().numpy(), wv)
        return cache, out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout,rot", [("half", 64), ("interleaved", 64), ("half", 20), ("interleaved", 12), ("half", 0)])
@pytest.mark.parametrize("page,order", [(1, "token"), (7, "head"), (16, "token"), (64, "head")])
def test_append(pp, dtype, layout, rot, page, order):
    c = AppendCase([(1, 0), (5, 30), (0, 12), (17, 6), (1, 63)], 6, 2, 64, page, dtype, rot, layout, order, pad=4)
    c.check(pp)
    rng = np.random.default_rng(1)
    c.check(pp, rng.integers(0, 50000, c.T).astype(np.int32))


@pytest.mark.parametrize("heads,kv,dim", [(1, 1, 8), (40, 40, 128), (12, 3, 80), (8, 1, 256)])
def test_append_head_shapes(pp, heads, kv, dim):
    for dtype in ("bf16", "f32"):
        AppendCase([(3, 5), (40, 0)], heads, kv, dim, 16, dtype, dim // 4 * 4, "half").check(pp)


def test_append_many_sequences(pp):
    """The search for a token's sequence: one to thousands of sequences, empty ones among them."""
    rng = np.random.default_rng(2)
    for B in (1, 2, 31, 32, 33, 1023, 1025, 3000):
        seqs = [(int(rng.integers(0, 3)), int(rng.integers(0, 9))) for _ in range(B - 1)] + [(1, 2)]
        AppendCase(seqs, 2, 1, 16, 4, "f32", 16, "half", seed=B).check(pp)


def test_append_without_queries_and_in_place(pp):
    import torch
    c = AppendCase([(3, 5), (4, 0)], 4, 2, 64, 16, "bf16", 64, "half")
    cache, out = c.check(pp)
    other, batch, rot = c.device(pp)
    ws = pp.alloc_attn_workspace(other)
    pp.pp_kv_append(other, batch, rot, None, None, to_dev(c.k, "bf16"), to_dev(c.v, "bf16"), None, ws)
    assert torch.equal(other.k, cache.k) and torch.equal(other.v, cache.v)
    # one fused projection, queries rotated where they lie
    other, batch, rot = c.device(pp)
    qkv = torch.cat([to_dev(a, "bf16").flatten(1) for a in (c.q, c.k, c.v)], 1).contiguous()
    q, k, v = qkv[:, :256], qkv[:, 256:384], qkv[:, 384:]
    pp.pp_kv_append(other, batch, rot, None, q, k, v, q, ws)
    assert torch.equal(other.k, cache.k) and torch.equal(other.v, cache.v)
    assert torch.equal(q, out.flatten(1)) and torch.equal(v, to_dev(c.v, "bf16").flatten(1))


def test_append_bad_lengths_and_pages(pp):
    """What cannot be right is recorded and not written; the other sequences are."""
    import torch
    for how in ("page_high", "page_negative", "ctx_negative", "ctx_long"):
        c = AppendCase([(2, 30), (3, 40), (1, 9)], 4, 2, 64, 16, "f32", 64, "half")
        _, wk, wv, _, tc = c.want(c.default_pos)
        kept = c.pages[1, 2].copy()
        if how == "page_high":
            c.pages[1, 2] = c.k0.shape[0]
        elif how == "page_negative":
            c.pages[1, 2] = -1
        elif how == "ctx_negative":
            c.ctx[1] = -1
        else:
            c.ctx[1] = 16 * c.pages.shape[1] - 2
        wk[kept], wv[kept], tc[kept] = c.k0[kept], c.v0[kept], 0.0
        cache, batch, rot = c.device(pp)
        ws = pp.alloc_attn_workspace(cache)
        q = to_dev(c.q)
        pp.pp_kv_append(cache, batch, rot, None, q, to_dev(c.k), to_dev(c.v), torch.empty_like(q), ws)
        assert pp.pp_get_device_status(ws) == pp.PP_ERR_INVALID_ARG, how
        assert (np.abs(cache.k.cpu().numpy() - wk) <= tc).all(), how
        assert np.array_equal(cache.v.cpu().numpy(), wv), how


def commit_reference(caches, ctx, pages, page, paths):
    """caches [L, n_pages, page, H, D]: entries moved, read before any is written."""
    out = caches.copy()
    for b, path in enumerate(paths):
        for j, p in enumerate(path):
            s, d = int(ctx[b]) + p, int(ctx[b]) + j
            out[:, pages[b, d // page], d % page] = caches[:, pages[b, s // page], s % page]
    return out


@pytest.mark.parametrize("dtype,kv,dim", [("bf16", 8, 128), ("f32", 2, 64), ("bf16", 1, 8), ("f32", 3, 20)])
@pytest.mark.parametrize("page,order", [(1, "token"), (16, "head"), (64, "token")])
@pytest.mark.parametrize("layers", [1, 3])
def test_commit(pp, dtype, kv, dim, page, order, layers):
    import torch
    rng = np.random.default_rng(page + layers)
    n = [12, 1, 0, 100, 7, 9]
    ctx = np.array([5, 0, 3, 14, 64, 15], np.int32)
    # overlapping moves, nothing accepted, everything accepted, a long path
    paths = [[0, 2, 3, 7, 11], [0], [], sorted(rng.choice(100, 75, replace=False).tolist()), [], [1, 2, 3, 4, 5, 6, 7, 8]]
    per = [-(-(a + int(c)) // page) for a, c in zip(n, ctx)]
    perm = rng.permutation(sum(per) + 1).astype(np.int32)
    pages = np.full((len(n), max(per)), -1, np.int32)
    at = 0
    for b, k in enumerate(per):
        pages[b, :k] = perm[at:at + k]
        at += k
    shape = (layers, len(perm), page, kv, dim)
    k0, v0 = (rounded(rng.standard_normal(shape), dtype) for _ in range(2))
    k, v = to_dev(k0, dtype), to_dev(v0, dtype)
    if order == "head":
        k, v = (t.transpose(2, 3).contiguous().transpose(2, 3) for t in (k, v))
    cache = pp.KVCache(k[0], v[0], kv)
    starts = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    batch = pp.Batch(to_dev(starts), to_dev(ctx), to_dev(pages), int(starts[-1]))
    path = np.full((len(n), 75), -9, np.int32)
    for b, p in enumerate(paths):
        path[b, :len(p)] = p
    acc = np.array([len(p) for p in paths], np.int32)
    new_len = torch.full((len(n),), -1, dtype=torch.int32, device="cuda")
    ws = pp.alloc_attn_workspace(cache)
    pp.pp_kv_commit(cache, batch, to_dev(path), to_dev(acc), ws, new_len=new_len, n_layers=layers,
                    layer_stride=k.stride(0))
    assert pp.pp_get_device_status(ws) == pp.PP_OK
    assert np.array_equal(new_len.cpu().numpy(), ctx + acc)
    for t, t0 in ((k, k0), (v, v0)):
        assert np.array_equal(t.float().cpu().numpy(), commit_reference(t0, ctx, pages, page, paths))


def test_commit_refuses_bad_paths_on_the_device(pp):
    import torch
    page, kv, dim = 16, 2, 16
    rng = np.random.default_rng(0)
    for path, acc in (([3, 3, 5], 3), ([4, 2, 5], 3), ([0, 1, 6], 3), ([-1, 1, 2], 3), ([0, 1, 2], 4), ([0, 1, 2], -1)):
        k0 = rounded(rng.standard_normal((4, page, kv, dim)), "f32")
        k, v = to_dev(k0), to_dev(k0 + 1)
        cache = pp.KVCache(k, v, kv)
        ctx = np.array([20, 3], np.int32)
        batch = pp.Batch(to_dev(np.array([0, 6, 12], np.int32)), to_dev(ctx),
                         to_dev(np.array([[2, 0], [1, 3]], np.int32)), 12)
        new_len = torch.full((2,), -1, dtype=torch.int32, device="cuda")
        ws = pp.alloc_attn_workspace(cache)
        pp.pp_kv_commit(cache, batch, to_dev(np.array([path, [1, 2, 4]], np.int32)), to_dev(np.array([acc, 3], np.int32)),
                        ws, new_len=new_len)
        assert pp.pp_get_device_status(ws) == pp.PP_ERR_INVALID_ARG
        assert new_len.tolist() == [20, 6]
        want = commit_reference(k0[None], ctx, np.array([[2, 0], [1, 3]]), page, [[], [1, 2, 4]])[0]
        assert np.array_equal(k.cpu().numpy(), want) and np.array_equal(v.cpu().numpy(), want + np.float32(1))
