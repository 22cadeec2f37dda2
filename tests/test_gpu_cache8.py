"""GPU tests of the 8-bit cache's append, read and commit against the
restatement in cache8_ref: bit for bit where nothing is computed ahead of the
rounding, within half a code's step and the inputs' bounds elsewhere."""
import numpy as np
import pytest

import attn_ref
import cache8_ref as ref
import norm_ref
from test_gpu_attention import rounded, to_dev
from test_gpu_cache import AppendCase, freqs
from test_gpu_canaries import Guarded

pytestmark = pytest.mark.gpu

E4M3_HALF = 2.0 ** -4  # half a step relative to the value; 2^-10 of the scale below 2^-6 of it


class Append8(AppendCase):
    """AppendCase over an 8-bit cache.  sizes: factors of the tokens' magnitudes, in turn."""

    def __init__(self, seqs, heads, kv_heads, dim, page, block, dtype, rot, layout, norm=False, sizes=(1.0,), **kw):
        super().__init__(seqs, heads, kv_heads, dim, page, dtype, rot, layout, **kw)
        f = np.array([sizes[i % len(sizes)] for i in range(self.T)])[:, None, None]
        self.k, self.v = rounded(self.k * f, dtype), rounded(self.v * f[::-1], dtype)
        rng = np.random.default_rng(77)
        # pages as earlier steps leave them; scales that no entry uses hold NaN
        self.kc, self.vc = (ref.quantised(rng.standard_normal(self.k0.shape), block) for _ in range(2))
        for b, (_, c) in enumerate(seqs):
            for j in range(-(-c // block) * block, self.pages.shape[1] * page, block):
                p = self.pages[b, j // page]
                if p >= 0:
                    self.kc.scale[p, :, j % page // block] = self.vc.scale[p, :, j % page // block] = np.nan
        self.block = block
        self.gamma = [rounded(1 + 0.3 * rng.standard_normal(dim), dtype) for _ in range(2)] if norm else None

    def cache8(self, pp):
        import torch
        code = [to_dev(c.code) for c in (self.kc, self.vc)]
        if self.order == "head":
            code = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in code]
        scale = [to_dev(c.scale) for c in (self.kc, self.vc)]
        return pp.KVCache8(*code, *scale, self.heads, torch.bfloat16 if self.dtype == "bf16" else torch.float32)

    def handles(self, pp):
        batch = pp.Batch(to_dev(self.starts), to_dev(self.ctx), to_dev(self.pages), self.T)
        rot = None if self.freq is None else pp.Rotation(to_dev(self.freq), self.layout)
        norm = None if self.gamma is None else pp.HeadNorm(*[to_dev(g, self.dtype) for g in self.gamma], 1e-5)
        return batch, rot, norm

    def heads_done(self, x, gamma, pos, dtype):
        """(values in fp64, bound) of normed and rotated heads, rounded to dtype (None: not rounded)."""
        def bound(w, tol):
            half = {None: 0.0, "bf16": attn_ref.BF16_HALF_ULP, "f32": attn_ref.F32_HALF_ULP}[dtype]
            return tol + half * (np.abs(w) + tol)
        x = x.astype(np.float64)
        if gamma is not None:
            w = norm_ref.forward(x, gamma, 1e-5, pos, self.freq, self.layout, 1.0)
            return w, bound(w, norm_ref.forward_bound(x, gamma, 1e-5, self.freq, self.layout, 1.0, "f32", w))
        if self.freq is None:
            return x, np.zeros_like(x)
        w = attn_ref.rotate(x, pos, self.freq, self.layout)
        t = np.zeros_like(x)
        n = 2 * len(self.freq)
        t[..., :n] = 1e-6 * norm_ref._pair_sum(x, n // 2, self.layout)[..., :n]
        return w, bound(w, t) * (np.arange(x.shape[-1]) < n)

    def compare(self, got, cache, want, tol):
        """One tensor's codes and scales after the append.  want, tol: new entries' values [T, H, D]."""
        code, scale = got
        exact = not tol.any()
        touched = np.zeros(code.shape[:2], bool)
        for b in range(len(self.ctx)):
            n, c, t0 = int(self.starts[b + 1] - self.starts[b]), int(self.ctx[b]), int(self.starts[b])
            if exact:
                cache.append(self.pages[b], c, want[t0:t0 + n])
                continue
            for lo in range(c - c % self.block, c + n, self.block) if n else ():
                p, o, i = cache.at(self.pages[b], lo)
                new = [e for e in range(lo, lo + self.block) if c <= e < c + n]
                x, t = (a[[t0 + e - c for e in new]] for a in (want, tol))
                now = scale[p, :, i].astype(np.float64)
                top, slack = ref.largest(x, (0, 2)), t.max((0, 2))
                lo_s, hi_s = ref.scale_for(np.maximum(top - slack, 0)), ref.scale_for(top + slack)
                if lo < c:
                    old = cache.scale[p, :, i].astype(np.float64)
                    lo_s, hi_s = (np.where(448 * old >= m, old, s) for m, s in ((top - slack, lo_s), (top + slack, hi_s)))
                    for e in range(lo, min(c, lo + self.block)):
                        again = ref.codes_of(ref.VALUES[cache.code[p, e - lo + o]] * (old / now)[:, None])
                        assert np.array_equal(code[p, e - lo + o], np.where((now != old)[:, None], again, cache.code[p, e - lo + o]))
                assert ((now == lo_s) | (now == hi_s)).all()
                for e, row, slop in zip(new, x, t):
                    held = ref.VALUES[code[p, e - lo + o]] * now[:, None]
                    assert (np.abs(held - row) <= np.maximum(E4M3_HALF * (np.abs(row) + slop), now[:, None] * 2.0 ** -10) + slop).all()
                    touched[p, e - lo + o] = True
                cache.scale[p, :, i] = now
                touched[p, o:o + max(0, c - lo)] = True
        if exact:
            assert np.array_equal(code, cache.code)
        else:
            assert np.array_equal(code[~touched], cache.code[~touched])
        assert np.array_equal(scale, cache.scale, equal_nan=True)

    def check(self, pp, pos=None):
        import torch
        cache = self.cache8(pp)
        batch, rot, norm = self.handles(pp)
        ws = pp.alloc_kvq_workspace(cache)
        q = to_dev(self.q, self.dtype)
        out = torch.full_like(q, 55.0)
        pp.pp_kvq_append(cache, batch, norm, rot, None if pos is None else to_dev(pos), q, to_dev(self.k, self.dtype),
                         to_dev(self.v, self.dtype), out, ws)
        torch.cuda.synchronize()
        assert pp.pp_get_device_status(ws) == pp.PP_OK
        pos = self.default_pos if pos is None else pos
        g = self.gamma or (None, None)
        wq, tq = self.heads_done(self.q, g[0], pos, self.dtype)
        got, u = out.float().cpu().numpy(), self.used
        assert (np.abs(got[:u] - wq[:u]) <= tq[:u]).all()
        assert (got[u:] == 55.0).all(), "padding rows were written"
        for code, scale, held, (w, t) in ((cache.k, cache.k_scale, self.kc, self.heads_done(self.k, g[1], pos, None)),
                                          (cache.v, cache.v_scale, self.vc, (self.v.astype(np.float64), np.zeros(self.v.shape)))):
            self.compare((code.cpu().numpy(), scale.cpu().numpy()), held, w, t)
        return cache, batch, ws, out


SEQS = [(1, 0), (5, 30), (0, 12), (17, 6), (1, 63), (1, 64), (40, 100), (2, 15)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout,rot", [("half", 64), ("interleaved", 64), ("half", 20), ("interleaved", 12), ("half", 0)])
@pytest.mark.parametrize("page,block,order", [(16, 16, "token"), (48, 16, "head"), (64, 32, "token"), (64, 64, "head"),
                                              (128, 128, "token")])
def test_append(pp, dtype, layout, rot, page, block, order):
    args = (SEQS, 6, 2, 64, page, block, dtype, rot, layout)
    Append8(*args, order=order, pad=4).check(pp)
    rng = np.random.default_rng(1)
    # magnitudes that make scales grow, and stay
    c = Append8(*args, norm=rot % 8 == 0, sizes=(1.0, 40.0, 1e-4, 0.0), order=order, pad=4, seed=3)
    c.check(pp, rng.integers(0, 50000, c.T).astype(np.int32))


@pytest.mark.parametrize("heads,kv,dim,rot", [(1, 1, 16, 16), (40, 40, 128, 128), (12, 3, 80, 40), (8, 1, 256, 256),
                                              (4, 2, 256, 20), (6, 3, 48, 4), (2, 2, 240, 120), (32, 8, 128, 0)])
@pytest.mark.parametrize("block", [16, 128])
def test_append_head_shapes(pp, heads, kv, dim, rot, block):
    for dtype in ("bf16", "f32"):
        for norm in (False, True):
            Append8([(3, 5), (140, 0), (1, 70)], heads, kv, dim, block, block, dtype, rot, "half", norm=norm).check(pp)


def test_append_many_sequences(pp):
    rng = np.random.default_rng(2)
    for B in (1, 2, 31, 32, 33, 1023, 1025):
        seqs = [(int(rng.integers(0, 3)), int(rng.integers(0, 40))) for _ in range(B - 1)] + [(1, 2)]
        Append8(seqs, 2, 1, 16, 16, 16, "f32", 0, "half", seed=B).check(pp)


def test_append_again_gives_the_same(pp):
    import torch
    c = Append8(SEQS, 6, 2, 64, 32, 16, "bf16", 64, "half", sizes=(1.0, 30.0))
    cache, batch, ws, out = c.check(pp)
    first = [t.clone() for t in (cache.k, cache.v, cache.k_scale.view(torch.int32), cache.v_scale.view(torch.int32), out)]
    _, rot, norm = c.handles(pp)
    pp.pp_kvq_append(cache, batch, norm, rot, None, to_dev(c.q, "bf16"), to_dev(c.k, "bf16"), to_dev(c.v, "bf16"), out, ws)
    again = (cache.k, cache.v, cache.k_scale.view(torch.int32), cache.v_scale.view(torch.int32), out)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_append_without_queries_and_in_place(pp):
    import torch
    c = Append8([(3, 5), (4, 0)], 4, 2, 64, 16, 16, "bf16", 64, "half", norm=True)
    cache, batch, ws, out = c.check(pp)
    batch, rot, norm = c.handles(pp)
    fresh = Append8([(3, 5), (4, 0)], 4, 2, 64, 16, 16, "bf16", 64, "half", norm=True)
    other = fresh.cache8(pp)
    pp.pp_kvq_append(other, batch, norm, rot, None, None, to_dev(c.k, "bf16"), to_dev(c.v, "bf16"), None, ws)
    assert torch.equal(other.k, cache.k) and torch.equal(other.v, cache.v)
    # one fused projection, queries done where they lie
    other = fresh.cache8(pp)
    qkv = torch.cat([to_dev(a, "bf16").flatten(1) for a in (c.q, c.k, c.v)], 1).contiguous()
    q, k, v = qkv[:, :256], qkv[:, 256:384], qkv[:, 384:]
    pp.pp_kvq_append(other, batch, norm, rot, None, q, k, v, q, ws)
    assert torch.equal(other.k, cache.k) and torch.equal(other.v, cache.v)
    assert torch.equal(q, out.flatten(1)) and torch.equal(v, to_dev(c.v, "bf16").flatten(1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_of_what_is_not_finite(pp, dtype):
    """NaN and infinities are held as NaN and do not touch the scale; huge and tiny magnitudes have scales of their own."""
    c = Append8([(20, 3), (4, 40)], 4, 2, 64, 16, 16, dtype, 0, "half")
    c.v[2, 0, 5], c.v[3, 1, 9], c.v[4, 0, 60] = np.nan, np.inf, -np.inf
    big = 3e38 if dtype == "f32" else float(rounded([3e38], "bf16")[0])
    c.k[13:20, 1] = 0.0
    c.k[13, 1, 0], c.k[14, 1, 1], c.k[15, 0] = big, 1.0, np.nan
    c.k[20:, 1] = rounded(c.k[20:, 1] * 1e-30, dtype)
    c.check(pp)


def test_append_bad_lengths_and_pages(pp):
    """What cannot be right is recorded and not written; the other sequences are."""
    import torch
    seqs = [(2, 30), (3, 40), (1, 9)]
    for how in ("page_high", "page_negative", "ctx_negative", "ctx_long", "start_high"):
        c = Append8(seqs, 4, 2, 64, 16, 16, "f32", 0, "half")
        if how == "page_high":
            c.pages[1, 2] = c.kc.code.shape[0]
        elif how == "page_negative":
            c.pages[1, 2] = -1
        elif how == "ctx_negative":
            c.ctx[1] = -1
        elif how == "ctx_long":
            c.ctx[1] = 16 * c.pages.shape[1] - 2
        else:
            c.starts[3] = c.T + 1
        cache = c.cache8(pp)
        batch, rot, norm = c.handles(pp)
        ws = pp.alloc_kvq_workspace(cache)
        q, v = to_dev(c.q), to_dev(c.v)
        out = torch.full_like(q, 55.0)
        pp.pp_kvq_append(cache, batch, norm, rot, None, q, to_dev(c.k), v, out, ws)
        assert pp.pp_get_device_status(ws) == pp.PP_ERR_INVALID_ARG, how
        good = [0, 1] if how == "start_high" else [0, 2]
        for b in good:
            c.vc.append(c.pages[b], int(c.ctx[b]), c.v[c.starts[b]:c.starts[b + 1]].astype(np.float64))
        assert np.array_equal(cache.v.cpu().numpy(), c.vc.code), how
        assert np.array_equal(cache.v_scale.cpu().numpy(), c.vc.scale, equal_nan=True), how
        rows = np.zeros(c.T, bool)
        for b in good + ([1] if how.startswith("page") else []):
            rows[c.starts[b]:c.starts[b + 1]] = True
        got = out.cpu().numpy()
        assert np.array_equal(got[rows], c.q[rows]) and (got[~rows] == 55.0).all(), how


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,dim,page,block,order", [(4, 2, 64, 16, 16, "token"), (40, 40, 128, 96, 32, "head"),
                                                          (3, 1, 80, 128, 128, "token"), (2, 2, 256, 64, 64, "token"),
                                                          (1, 1, 16, 16, 16, "head")])
def test_read(pp, dtype, heads, kv, dim, page, block, order):
    """Parts of sequences, exact for scales that are powers of two; padding rows and other columns stay; entries of a page
    that does not exist are zeros."""
    import torch
    seqs = [(7, 0), (0, 5), (33, 20), (1, 64), (130, 3)]
    c = Append8(seqs, heads, kv, dim, page, block, dtype, 0, "half", order=order, pad=3, seed=dim)
    whole = np.random.default_rng(5).standard_normal(c.kc.code.shape)
    c.kc, c.vc = ref.quantised(whole, block), ref.quantised(whole * 1e3, block)
    c.kc.code[c.pages[2, 0], 0, 0, :8] = 0x7f
    cache = c.cache8(pp)
    bad = c.pages[4, -(-133 // page) - 1]
    c.pages[4, -(-133 // page) - 1] = -1
    batch, _, _ = c.handles(pp)
    ws = pp.alloc_kvq_workspace(cache)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    wide = torch.full((c.T, 2 * kv * dim + 32), 9.0, dtype=dt, device="cuda")
    ko, vo = wide[:, :kv * dim], wide[:, kv * dim + 16:2 * kv * dim + 16]
    pp.pp_kvq_read(cache, batch, ko, vo, ws)
    assert pp.pp_get_device_status(ws) == pp.PP_ERR_INVALID_ARG
    got = wide.float().cpu().numpy()
    assert (got[c.used:] == 9.0).all() and (got[:, kv * dim:kv * dim + 16] == 9.0).all() and (got[:, 2 * kv * dim + 16:] == 9.0).all()
    values = [x.values() for x in (c.kc, c.vc)]
    for b, (n, ctx) in enumerate(seqs):
        for i in range(n):
            p, o, _ = c.kc.at(c.pages[b], ctx + i)
            for v, at in zip(values, (0, kv * dim + 16)):
                want = np.zeros((kv, dim)) if p < 0 else v[p, o]
                assert np.array_equal(got[c.starts[b] + i, at:at + kv * dim], want.reshape(-1).astype(np.float32), equal_nan=True)
    assert bad >= 0


def paths_case(page, block, kv, dim, layers, seed, n, ctx, paths):
    """Caches of `layers` layers, batch arrays and paths; scales differ from block to block by up to 2^6."""
    rng = np.random.default_rng(seed)
    per = [-(-(a + int(c)) // page) for a, c in zip(n, ctx)]
    perm = rng.permutation(sum(per) + 1).astype(np.int32)
    pages = np.full((len(n), max(per)), -1, np.int32)
    at = 0
    for b, k in enumerate(per):
        pages[b, :k] = perm[at:at + k]
        at += k
    caches = []
    for _ in range(2 * layers):
        x = rng.standard_normal((len(perm), page, kv, dim)) * 2.0 ** rng.integers(-3, 4, (len(perm), page, 1, 1))
        x *= np.repeat(2.0 ** rng.integers(-3, 4, (len(perm), page // block, 1, 1)), block, 1)
        caches.append(ref.quantised(x, block))
    path = np.full((len(n), max(map(len, paths)) + 1), -9, np.int32)
    for b, p in enumerate(paths):
        path[b, :len(p)] = p
    return pages, caches[:layers], caches[layers:], path


@pytest.mark.parametrize("dtype,kv,dim", [("bf16", 8, 128), ("f32", 2, 64), ("bf16", 1, 16), ("f32", 3, 80), ("bf16", 2, 256)])
@pytest.mark.parametrize("page,block,order", [(16, 16, "token"), (48, 16, "head"), (64, 64, "token"), (128, 128, "token")])
@pytest.mark.parametrize("layers", [1, 3])
def test_commit(pp, dtype, kv, dim, page, block, order, layers):
    import torch
    rng = np.random.default_rng(page + layers)
    n = [12, 1, 0, 100, 7, 9, 200]
    ctx = np.array([5, 0, 3, 14, 64, 15, 37], np.int32)
    # overlapping moves, nothing accepted, everything accepted, long paths, one that begins in its place
    paths = [[0, 2, 3, 7, 11], [0], [], sorted(rng.choice(100, 75, replace=False).tolist()), [], [1, 2, 3, 4, 5, 6, 7, 8],
             [0, 1, 2] + sorted((3 + rng.choice(197, 140, replace=False)).tolist())]
    pages, ks, vs, path = paths_case(page, block, kv, dim, layers, page + layers, n, ctx, paths)
    code = [to_dev(np.stack([c.code for c in x])) for x in (ks, vs)]
    if order == "head":
        code = [t.transpose(2, 3).contiguous().transpose(2, 3) for t in code]
    scale = [to_dev(np.stack([c.scale for c in x])) for x in (ks, vs)]
    cache = pp.KVCache8(code[0][0], code[1][0], scale[0][0], scale[1][0], kv, torch.bfloat16 if dtype == "bf16" else torch.float32)
    starts = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    batch = pp.Batch(to_dev(starts), to_dev(ctx), to_dev(pages), int(starts[-1]))
    acc = np.array([len(p) for p in paths], np.int32)
    new_len = torch.full((len(n),), -1, dtype=torch.int32, device="cuda")
    ws = pp.alloc_kvq_workspace(cache)
    pp.pp_kvq_commit(cache, batch, to_dev(path), to_dev(acc), ws, new_len=new_len, n_layers=layers,
                     layer_stride=code[0].stride(0), scale_layer_stride=scale[0].stride(0))
    assert pp.pp_get_device_status(ws) == pp.PP_OK
    assert np.array_equal(new_len.cpu().numpy(), ctx + acc)
    for x, c, s in ((ks, code[0], scale[0]), (vs, code[1], scale[1])):
        for layer, held in enumerate(x):
            for b, p in enumerate(paths):
                held.commit(pages[b], int(ctx[b]), p)
            assert np.array_equal(s[layer].cpu().numpy(), held.scale)
            assert np.array_equal(c[layer].cpu().numpy(), held.code)


def test_commit_refuses_bad_paths_on_the_device(pp):
    import torch
    for path, acc in (([3, 3, 5], 3), ([4, 2, 5], 3), ([0, 1, 6], 3), ([-1, 1, 2], 3), ([0, 1, 2], 4), ([0, 1, 2], -1)):
        ctx = np.array([20, 3], np.int32)
        pages, (k,), (v,), _ = paths_case(16, 16, 2, 32, 1, 0, [6, 6], ctx, [[], []])
        cache = pp.KVCache8(*[to_dev(a) for a in (k.code, v.code, k.scale, v.scale)], 2, torch.float32)
        batch = pp.Batch(to_dev(np.array([0, 6, 12], np.int32)), to_dev(ctx), to_dev(pages), 12)
        new_len = torch.full((2,), -1, dtype=torch.int32, device="cuda")
        ws = pp.alloc_kvq_workspace(cache)
        pp.pp_kvq_commit(cache, batch, to_dev(np.array([path, [1, 2, 4]], np.int32)), to_dev(np.array([acc, 3], np.int32)), ws,
                         new_len=new_len)
        assert pp.pp_get_device_status(ws) == pp.PP_ERR_INVALID_ARG
        assert new_len.tolist() == [20, 6]
        k.commit(pages[1], 3, [1, 2, 4])
        assert np.array_equal(cache.k.cpu().numpy(), k.code) and np.array_equal(cache.k_scale.cpu().numpy(), k.scale)


def test_nothing_to_do(pp):
    import torch
    cache = pp.KVCache8.empty(2, 16, 4, 2, 64, torch.bfloat16)
    ws = pp.alloc_kvq_workspace(cache)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    for B, q_start in ((0, i32(1)), (2, i32(3))):
        batch = pp.Batch(q_start, i32(B), i32(B, 1), 0)
        e = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
        pp.pp_kvq_append(cache, batch, None, None, None, None, e, e, None, ws)
        pp.pp_kvq_read(cache, batch, e, e.clone(), ws)
        pp.pp_kvq_commit(cache, batch, i32(B, 1), i32(B), ws)
    assert pp.pp_get_device_status(ws) == pp.PP_OK
    assert int(cache.k.sum()) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bands_and_graphs(pp, dtype):
    """Sentinel bands around every tensor that is written; replays of a captured append and read follow the lengths."""
    import torch
    c = Append8([(3, 30), (1, 5), (20, 0)], 4, 2, 64, 32, 16, dtype, 64, "half", norm=True)
    want = c.cache8(pp)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = [Guarded(tuple(t.shape), t.dtype) for t in (want.k, want.v, want.k_scale, want.v_scale)]
    g += [Guarded((c.T, 4, 64), dt), Guarded((c.T, 2, 64), dt), Guarded((c.T, 2, 64), dt)]
    for a, t in zip(g, (want.k, want.v, want.k_scale, want.v_scale)):
        a.t.copy_(t)
    cache = pp.KVCache8(*[a.t for a in g[:4]], 4, dt)
    batch, rot, norm = c.handles(pp)
    ws = pp.alloc_kvq_workspace(cache)
    q, k, v = to_dev(c.q, dtype), to_dev(c.k, dtype), to_dev(c.v, dtype)

    def step(cache, out, ko, vo):
        pp.pp_kvq_append(cache, batch, norm, rot, None, q, k, v, out, ws)
        pp.pp_kvq_read(cache, batch, ko, vo, ws)
    fresh = [torch.empty_like(a.t) for a in g[4:]]
    step(want, *fresh)
    step(cache, *[a.t for a in g[4:]])
    torch.cuda.synchronize()
    assert all(a.bands_intact() for a in g)
    same = lambda: all(torch.equal(a.t.view(torch.uint8), t.view(torch.uint8))
                       for a, t in zip(g, [want.k, want.v, want.k_scale, want.v_scale] + fresh))
    assert same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(cache, *[a.t for a in g[4:]])
    batch.ctx_len.copy_(torch.tensor([33, 6, 20], dtype=torch.int32))
    graph.replay()
    step(want, *fresh)
    torch.cuda.synchronize()
    assert same() and all(a.bands_intact() for a in g)
    assert pp.pp_get_device_status(ws) == pp.PP_ERR_INVALID_ARG  # 20 + 20 entries, one page of 32
