"""GPU tests of attention over the 8-bit cache against the fp64 definition over
code * scale, within the bound that attn_ref.attend derives."""
import numpy as np
import pytest

import attn_ref
import cache8_ref as ref
from test_gpu_attention import Case, to_dev
from test_gpu_canaries import Guarded

pytestmark = pytest.mark.gpu


class Case8(Case):
    """Case over an 8-bit cache: the same random entries, held in codes.  spread: blocks' magnitudes differ by up to
    2^spread both ways.  What no sequence uses holds NaN codes; scales that none uses hold NaN."""

    def __init__(self, seqs, heads, kv_heads, dim, page, block, dtype, spread=0, stale=np.nan, **kw):
        super().__init__(seqs, heads, kv_heads, dim, page, dtype, stale=np.nan, **kw)
        rng = np.random.default_rng(9)
        self.block = block
        self.held = []
        for x in (self.k, self.v):
            if spread:
                x = x * np.repeat(2.0 ** rng.integers(-spread, spread + 1, (len(x), page // block, 1, 1)), block, 1)
            used = np.isfinite(x)
            c = ref.quantised(np.where(used, x, np.nan), block)
            none = ~used.reshape(len(x), page // block, -1).any(2)
            c.scale[none[:, None, :].repeat(kv_heads, 1)] = np.nan
            self.held.append(c)
        if stale == 0.0:
            for c in self.held:
                c.code[np.isnan(ref.VALUES[c.code])] = 0
                c.scale[np.isnan(c.scale)] = 1.0
        self.refresh()

    def refresh(self):
        """The values that the definition reads."""
        self.k, self.v = (c.values() for c in self.held)

    def device(self, pp):
        import torch
        code = [to_dev(c.code) for c in self.held]
        if self.order == "head":
            code = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in code]
        cache = pp.KVCache8(*code, *[to_dev(c.scale) for c in self.held], self.heads,
                            torch.bfloat16 if self.dtype == "bf16" else torch.float32)
        batch = pp.Batch(to_dev(self.starts), to_dev(self.ctx), to_dev(self.pages), self.T)
        mask = None if self.mask is None else to_dev(self.mask.view(np.int32))
        q = to_dev(self.q, self.dtype)
        return cache, batch, q, mask, torch.full_like(q, 77.0)

    def run(self, pp, stream=None):
        import torch
        cache, batch, q, mask, out = self.device(pp)
        ws = pp.alloc_kvq_workspace(cache)
        pp.pp_kvq_tree_attention(cache, batch, q, mask, self.scale, out, ws, stream)
        torch.cuda.synchronize()
        return out.float().cpu().numpy(), pp.pp_get_device_status(ws), ws

    def want(self):
        return attn_ref.attend(self.q, self.k, self.v, self.starts, self.ctx, self.pages, self.mask, self.scale, self.dtype)


EDGE = [(1, 0), (1, 1), (1, 62), (1, 63), (1, 64), (1, 127), (1, 128), (1, 300)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,dim", [(4, 4, 128), (8, 2, 128), (6, 2, 64), (4, 1, 80), (8, 1, 256), (16, 1, 64),
                                          (3, 3, 16), (2, 2, 144), (16, 1, 128), (17, 1, 128), (32, 1, 128)])
def test_single_tokens(pp, dtype, heads, kv, dim):
    Case8(EDGE, heads, kv, dim, 16, 16, dtype).check(pp)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page,block", [(16, 16), (48, 16), (32, 32), (64, 64), (256, 128), (96, 32), (384, 64)])
@pytest.mark.parametrize("order", ["token", "head"])
def test_pages_blocks_and_orders(pp, dtype, page, block, order):
    Case8([(3, 130), (1, 7), (5, 0), (2, 65), (1, 500)], 4, 2, 64, page, block, dtype, order=order, seed=page).check(pp)
    Case8([(1, 130), (1, 7), (1, 0), (1, 655)], 8, 2, 128, page, block, dtype, order=order, seed=page, spread=4).check(pp)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", ["tree", "random", "none"])
@pytest.mark.parametrize("heads,kv,dim", [(4, 4, 64), (8, 2, 128), (5, 1, 128), (2, 2, 256)])
def test_masks(pp, dtype, mask, heads, kv, dim):
    Case8([(13, 40), (1, 0), (33, 127), (7, 0), (64, 5), (40, 256)], heads, kv, dim, 16, 16, dtype, mask=mask, seed=heads).check(pp)
    Case8([(3, 40), (1, 0), (4, 127), (2, 0)], heads, kv, dim, 32, 32, dtype, mask=mask, seed=heads).check(pp)


def test_rows_that_see_nothing_are_zero(pp):
    for dtype in ("bf16", "f32"):
        for heads in (2, 4):
            c = Case8([(5, 0), (3, 10), (4, 0)], heads, 2, 64, 16, 16, dtype, mask="none")
            got = c.check(pp)
            assert (got[:5] == 0).all() and (got[8:] == 0).all() and (got[5:8] != 0).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv", [(64, 1), (48, 2), (40, 1), (7, 7)])
def test_large_and_odd_groups(pp, dtype, heads, kv):
    Case8([(1, 150), (3, 20), (7, 0)], heads, kv, 64, 16, 16, dtype).check(pp)
    Case8([(5, 130), (9, 1)], heads, kv, 64, 16, 16, dtype, mask="tree").check(pp)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,dim", [(8, 2, 128), (2, 2, 64), (4, 1, 256)])
def test_long_and_split_items(pp, dtype, heads, kv, dim):
    Case8([(1, 5000), (1, 17), (1, 3000)], heads, kv, dim, 64, 16, dtype, spread=2).check(pp)
    Case8([(9, 3000), (1, 900), (2, 1)], heads, kv, dim, 16, 16, dtype, mask="tree").check(pp)


@pytest.mark.parametrize("kv,order", [(8, "token"), (6, "token"), (8, "head"), (3, "token")])
def test_many_heads_over_long_ragged_contexts(pp, kv, order):
    """Stretches of many tiles: heads taken side by side (8: in fours, 6: in twos), items that count more than their tiles,
    short and empty sequences among long ones."""
    seqs = [(1, 9000), (1, 3), (1, 0), (0, 50), (1, 6001), (1, 130), (1, 7777), (2, 4000), (1, 128), (1, 5000), (1, 64)]
    Case8(seqs * 2, 2 * kv, kv, 128, 64, 16, "bf16", order=order, spread=2, seed=kv).check(pp)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompts_and_padding(pp, dtype):
    Case8([(200, 90), (129, 3), (300, 0)], 4, 2, 64, 32, 16, dtype, pad=5).check(pp)
    Case8([(1, 90), (1, 3)], 4, 2, 128, 32, 16, dtype, pad=5).check(pp)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", ["chain", "tree"])
@pytest.mark.parametrize("n,heads,ctx,page", [(3, 4, 70, 16), (16, 1, 300, 64), (20, 4, 500, 48), (150, 2, 40, 16), (300, 1, 0, 16)])
def test_hidden_and_seen_nan(pp, dtype, mask, n, heads, ctx, page):
    """NaN codes in keys and values of new tokens: rows that do not see the token keep their bound, rows that do get NaN
    (of a value: in its element; of a key: everywhere)."""
    for where in ("value", "key"):
        c = Case8([(n, ctx), (2, 33)], heads, 1, 64, page, 16, dtype, mask=mask, seed=n, stale=0.0)
        want, tol = c.want()
        j = ctx + n // 2
        c.held[where == "value"].code[c.pages[0, j // page], j % page, :, 3] = 0xff
        see = attn_ref.visible(n, ctx, c.mask, 0)[:, j]
        got, status, _ = c.run(pp)
        assert status == pp.PP_OK and see.any() and not see.all()
        ok = np.abs(got - want) <= tol
        assert ok[:n][~see].all() and ok[n:].all()
        bad = got[:n][see]
        if where == "key":
            assert np.isnan(bad).all()
        else:
            assert np.isnan(bad[..., 3]).all()
            ok[:n, :, 3] = True
            assert ok.all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 5, 40])
def test_scales_far_apart(pp, dtype, n):
    """Blocks whose scales differ by 2^30: zero blocks at the smallest scale, tiny and huge values."""
    c = Case8([(n, 200), (n, 17)], 4, 2, 64, 16, 16, dtype, seed=n)
    v = c.held[1]
    rng = np.random.default_rng(n)
    for p in range(len(v.scale)):
        kind = rng.integers(0, 4)
        if kind == 0:
            v.code[p][~np.isnan(ref.VALUES[v.code[p]])] = 0
            v.scale[p] = 2.0 ** -60
        elif kind < 3:
            v.scale[p] = v.scale[p] * 2.0 ** (-20 if kind == 1 else 10)
    c.refresh()
    c.check(pp)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales_that_are_no_powers_of_two(pp, dtype):
    """A cache filled elsewhere.  bf16: code * scale rounded to bf16 moves a score by 2^-8 of sum |q k| and a value by
    2^-8 of itself."""
    for seqs in ([(1, 300), (1, 40)], [(7, 100), (33, 20)]):
        c = Case8(seqs, 4, 2, 64, 32, 16, dtype)
        rng = np.random.default_rng(3)
        for h in c.held:
            h.scale *= rng.uniform(0.6, 1.9, h.scale.shape).astype(np.float32)
        c.refresh()
        want, tol = c.want()
        if dtype == "bf16":
            for b, (n, ctx) in enumerate(seqs):
                k = np.abs(attn_ref.gather(c.k, c.pages[b], ctx + n))
                v = np.abs(attn_ref.gather(c.v, c.pages[b], ctx + n))
                for i in range(int(c.starts[b]), int(c.starts[b]) + n):
                    for h in range(4):
                        ds = 2.0 ** -8 * c.scale * (k[:, h // 2] @ np.abs(c.q[i, h])).max()
                        tol[i, h] += (np.expm1(2 * ds) + 2.0 ** -8) * v[:, h // 2].max(0)
        got, status, _ = c.run(pp)
        assert status == pp.PP_OK and (np.abs(got - want) <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 20])
def test_bits_streams_bands_and_graphs(pp, dtype, n):
    import torch
    c = Case8([(n, 2000), (1, 300), (n, 17)], 8, 2, 128, 16, 16, dtype, mask="tree")
    a = c.run(pp)[0]
    assert np.array_equal(a, c.run(pp)[0])
    cache, batch, q, mask, _ = c.device(pp)
    ws = pp.alloc_kvq_workspace(cache)
    out = Guarded(tuple(q.shape), q.dtype)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        late = torch.empty_like(q)
        busy = torch.randn(2048, 2048, device="cuda")
        for _ in range(20):
            busy = busy @ busy * 1e-3
        late.copy_(q)
        pp.pp_kvq_tree_attention(cache, batch, late, mask, c.scale, out.t, ws)
    torch.cuda.synchronize()
    assert np.array_equal(a, out.t.float().cpu().numpy()) and out.bands_intact()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pp.pp_kvq_tree_attention(cache, batch, q, mask, c.scale, out.t, ws)
    c.ctx = np.array([777, 300, 0], np.int32)
    batch.ctx_len.copy_(to_dev(c.ctx))
    graph.replay()
    torch.cuda.synchronize()
    want, tol = c.want()
    assert (np.abs(out.t.float().cpu().numpy() - want) <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 30])
def test_bad_lengths_and_pages_are_reported(pp, dtype, n):
    good = Case8([(n, 30), (n, 40), (1, 9)], 4, 2, 64, 16, 16, dtype)
    want, tol = good.want()
    for how in ("page_high", "page_negative", "ctx_negative", "ctx_long"):
        c = Case8([(n, 30), (n, 40), (1, 9)], 4, 2, 64, 16, 16, dtype)
        if how == "page_high":
            c.pages[1, 1] = len(c.held[0].code)
        elif how == "page_negative":
            c.pages[1, 0] = -1
        elif how == "ctx_negative":
            c.ctx[1] = -1
        else:
            c.ctx[1] = 16 * c.pages.shape[1] - n + 1
        got, status, _ = c.run(pp)
        assert status == pp.PP_ERR_INVALID_ARG, how
        for rows in (slice(0, n), slice(2 * n, 2 * n + 1)):
            assert (np.abs(got[rows] - want[rows]) <= tol[rows]).all(), how
        if how.startswith("ctx"):
            assert (got[n:2 * n] == 77.0).all(), how


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_tokens(pp, dtype):
    import torch
    for seqs in ([(1, 90), (1, 4)], [(3, 90), (17, 4)], [(30, 90), (40, 4)]):
        c = Case8(seqs, 4, 2, 64, 16, 16, dtype, mask="tree")
        cache, batch, q, mask, _ = c.device(pp)
        ws = pp.alloc_kvq_workspace(cache)
        wide = torch.full((c.T, 8 * 64), 3.0, dtype=q.dtype, device="cuda")
        wide[:, 128:384] = q.flatten(1)
        wout = torch.full((c.T, 300 + 20), 5.0, dtype=q.dtype, device="cuda")
        pp.pp_kvq_tree_attention(cache, batch, wide[:, 128:384], mask, c.scale, wout[:, 32:288], ws)
        want, tol = c.want()
        got = wout.float().cpu().numpy()
        assert (np.abs(got[:, 32:288].reshape(want.shape) - want) <= tol).all()
        assert (got[:, :32] == 5.0).all() and (got[:, 288:] == 5.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_steps_of_a_decode_loop(pp, dtype):
    """Append, attend, read and commit as a drafting loop calls them, one workspace: trees that are appended, attended
    and cut to a path, then single tokens; attention within its bound over what the cache then holds."""
    import torch
    heads, kv, dim, page, block, B = 8, 2, 64, 32, 16, 3
    rng = np.random.default_rng(0)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    cache = pp.KVCache8.empty(3 * 8, page, heads, kv, dim, dt, block)
    table = rng.permutation(24).astype(np.int32).reshape(B, 8)
    ws = pp.alloc_kvq_workspace(cache)
    rot = pp.Rotation.make(dim)
    gamma = torch.ones(dim, dtype=dt, device="cuda")
    norm = pp.HeadNorm(gamma, gamma)
    ctx = np.zeros(B, np.int32)
    for step, new in enumerate(([20, 1, 33], [9, 12, 5], [1, 1, 1], [13, 2, 7], [1, 1, 1])):
        starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        T = int(starts[-1])
        parents = [[int(rng.integers(max(-1, i - 4), i)) for i in range(n)] for n in new]
        chain = step == 0 or max(new) == 1
        if chain:
            parents = [list(range(-1, n - 1)) for n in new]
        mask, depth = attn_ref.tree_mask(parents, 2)
        qkv = torch.from_numpy(rng.standard_normal((T, (heads + 2 * kv) * dim)).astype(np.float32)).to(dt).cuda()
        q, k, v = qkv[:, :heads * dim], qkv[:, heads * dim:(heads + kv) * dim], qkv[:, (heads + kv) * dim:]
        batch = pp.Batch(to_dev(starts), to_dev(ctx), to_dev(table), T)
        pos = to_dev((np.repeat(ctx, new) + depth).astype(np.int32))
        pp.pp_kvq_append(cache, batch, norm, rot, pos, q, k, v, q, ws)
        out = torch.empty((T, heads, dim), dtype=dt, device="cuda")
        pp.pp_kvq_tree_attention(cache, batch, q, None if chain else to_dev(mask.view(np.int32)), dim ** -0.5, out, ws)
        kr, vr = (torch.empty((T, kv, dim), dtype=dt, device="cuda") for _ in range(2))
        pp.pp_kvq_read(cache, batch, kr, vr, ws)
        held = [ref.Cache(c.cpu().numpy(), s.cpu().numpy(), block) for c, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale))]
        values = [h.values() for h in held]
        want, tol = attn_ref.attend(q.float().cpu().numpy().reshape(T, heads, dim), *values, starts, ctx, table,
                                    None if chain else mask, float(np.float32(dim ** -0.5)), dtype)
        assert (np.abs(out.float().cpu().numpy() - want) <= tol).all()
        for b in range(B):
            j = ctx[b] + np.arange(new[b])
            at = slice(int(starts[b]), int(starts[b + 1]))
            for got, val in zip((kr, vr), values):
                assert np.array_equal(got[at].float().cpu().numpy(), val[table[b, j // page], j % page].astype(np.float32))
        paths = [list(range(n)) if chain else sorted(rng.choice(n, max(1, n // 2), replace=False).tolist()) for n in new]
        path = np.full((B, max(new)), -1, np.int32)
        for b, p in enumerate(paths):
            path[b, :len(p)] = p
        acc = np.array([len(p) for p in paths], np.int32)
        new_len = torch.empty(B, dtype=torch.int32, device="cuda")
        pp.pp_kvq_commit(cache, batch, to_dev(path), to_dev(acc), ws, new_len=new_len)
        for b, p in enumerate(paths):
            for h in held:
                h.commit(table[b], int(ctx[b]), p)
        for (c, s), h in zip(((cache.k, cache.k_scale), (cache.v, cache.v_scale)), held):
            assert np.array_equal(c.cpu().numpy(), h.code) and np.array_equal(s.cpu().numpy(), h.scale)
        ctx = ctx + acc
        assert np.array_equal(new_len.cpu().numpy(), ctx)
    assert pp.pp_get_device_status(ws) == pp.PP_OK


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("kv", [8, 16])
def test_every_code_alone(pp, kv, dim):
    # one visible entry a sequence: a weight of one, so that the result is code * scale, rounded once
    scales = np.array([1.0, 2.0 ** -60, 2.0 ** 8, 2.0 ** 119, 1.5, 1 + 2.0 ** -15, 0.75 * 2.0 ** -30, 2.0 ** 100], np.float32)
    c = Case8([(40, 1)] * (256 // dim) + [(200, 1)], 2 * kv if kv == 16 else kv, kv, dim, 16, 16, "bf16", mask="random")
    c.mask[:] = 0
    held = c.held[1]
    for b in range(len(c.ctx)):
        page = int(c.pages[b][0])
        held.code[page, 0] = (dim * b + np.arange(dim)) % 256
        held.scale[page, :, 0] = np.resize(scales, kv)
    c.refresh()
    got, status, _ = c.run(pp)
    assert status == 0
    for b in range(len(c.ctx)):
        code = (dim * b + np.arange(dim)) % 256
        want = ref.VALUES[code][None] * np.resize(scales, kv)[:, None].astype(np.float64)
        want = np.repeat(want, c.heads // kv, 0).astype(np.float32)
        import torch
        want = torch.from_numpy(want).to(torch.bfloat16).float().numpy()
        rows = got[c.starts[b]:c.starts[b + 1]].reshape(-1, c.heads, dim)
        np.testing.assert_array_equal(rows, np.broadcast_to(want, rows.shape))
