"""GPU tests of tree attention over the paged cache against the fp64
definition (attn_ref.attend), at the lengths, head shapes, page sizes, masks
and layouts where it can go wrong.  Every tolerance is the per-element bound
that attn_ref derives."""
import numpy as np
import pytest

import attn_ref as ref

pytestmark = pytest.mark.gpu


def to_dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a))
    if dtype == "bf16":
        t = t.to(torch.bfloat16)
    return t.cuda()


def rounded(a, dtype):
    """The fp32 values a tensor of this type holds."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32))
    return (t.to(torch.bfloat16).float() if dtype == "bf16" else t).numpy()


class Case:
    """Random inputs of one call.  seqs: [(new tokens, cached tokens)]."""

    def __init__(self, seqs, heads, kv_heads, dim, page, dtype, mask="chain", order="token", seed=0, stale=np.nan,
                 pad=0, words=None, std=1.0):
        rng = np.random.default_rng(seed)
        self.dtype, self.page, self.heads = dtype, page, heads
        n = [s[0] for s in seqs]
        self.ctx = np.array([s[1] for s in seqs], np.int32)
        self.starts = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        used = int(self.starts[-1])
        self.T = used + pad
        per = [-(-(a + c) // page) for a, c in seqs]
        n_pages = sum(per) + 3
        perm = rng.permutation(n_pages).astype(np.int32)
        self.pages = np.full((len(seqs), max(per) + 1), -7, np.int32)
        at = 0
        for b, k in enumerate(per):
            self.pages[b, :k] = perm[at:at + k]
            at += k
        # everything past a sequence's entries holds `stale`
        self.k = np.full((n_pages, page, kv_heads, dim), stale, np.float32)
        self.v = np.full((n_pages, page, kv_heads, dim), stale, np.float32)
        for b, (a, c) in enumerate(seqs):
            j = np.arange(a + c)
            shape = (a + c, kv_heads, dim)
            self.k[self.pages[b, j // page], j % page] = rounded(rng.standard_normal(shape), dtype)
            self.v[self.pages[b, j // page], j % page] = rounded(rng.standard_normal(shape) + 0.5, dtype)
        self.q = rounded(rng.standard_normal((self.T, heads, dim)) * std, dtype)
        self.scale = float(np.float32(dim ** -0.5))
        self.mask = None
        if mask != "chain":
            words = words or max(1, -(-max(n) // 32))
            if mask == "tree":
                parents = [[int(rng.integers(max(-1, i - 6), i)) for i in range(a)] for a in n]
                self.mask = ref.tree_mask(parents, words)[0]
            elif mask == "random":  # any bits, bits past the sequence's tokens among them
                self.mask = rng.integers(0, 1 << 32, size=(used, words), dtype=np.uint32)
            elif mask == "none":    # no new token sees any new token
                self.mask = np.zeros((used, words), np.uint32)
            if pad:
                self.mask = np.concatenate([self.mask, np.full((pad, words), 0xffffffff, np.uint32)])
        self.order = order

    def device(self, pp):
        import torch
        k, v = to_dev(self.k, self.dtype), to_dev(self.v, self.dtype)
        if self.order == "head":  # pages stored head by head
            k, v = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in (k, v))
        cache = pp.KVCache(k, v, self.heads)
        batch = pp.Batch(to_dev(self.starts), to_dev(self.ctx), to_dev(self.pages), self.T)
        mask = None if self.mask is None else to_dev(self.mask.view(np.int32))
        q = to_dev(self.q, self.dtype)
        return cache, batch, q, mask, torch.full_like(q, 77.0)

    def run(self, pp, stream=None):
        import torch
        cache, batch, q, mask, out = self.device(pp)
        ws = pp.alloc_attn_workspace(cache)
        pp.pp_tree_attention(cache, batch, q, mask, self.scale, out, ws, stream)
        torch.cuda.synchronize()
        return out.float().cpu().numpy(), pp.pp_get_device_status(ws), ws

    def check(self, pp):
        got, status, ws = self.run(pp)
        assert status == pp.PP_OK
        want, tol = ref.attend(self.q, self.k, self.v, self.starts, self.ctx, self.pages, self.mask, self.scale, self.dtype)
        used = int(self.starts[-1])
        assert np.isfinite(got[:used]).all()
        off = np.abs(got[:used] - want[:used]) - tol[:used]
        assert off.max(initial=-1.0) <= 0, (float(off.max()), np.unravel_index(off.argmax(), off.shape))
        assert (got[used:] == 77.0).all(), "padding rows were written"
        # the counters of split items are back at rest
        assert int(ws[1280:1280 + 4 * 608].sum()) == 0
        return got


EDGE = [(1, 0), (1, 1), (1, 62), (1, 63), (1, 64), (1, 127), (1, 128), (1, 300)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,dim", [(4, 4, 128), (8, 2, 128), (6, 2, 64), (4, 1, 80), (8, 1, 256), (16, 1, 64),
                                          (3, 3, 8), (2, 2, 136)])
def test_single_tokens(pp, dtype, heads, kv, dim):
    Case(EDGE, heads, kv, dim, 16, dtype).check(pp)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [1, 7, 16, 64, 200])
@pytest.mark.parametrize("order", ["token", "head"])
def test_page_sizes_and_orders(pp, dtype, page, order):
    Case([(3, 130), (1, 7), (5, 0), (2, 65)], 4, 2, 64, page, dtype, order=order, seed=page).check(pp)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", ["tree", "random", "none"])
@pytest.mark.parametrize("heads,kv,dim", [(4, 4, 64), (8, 2, 128), (5, 1, 128)])
def test_masks(pp, dtype, mask, heads, kv, dim):
    # (n, 0) under "none": tokens that see nothing give zeros
    Case([(13, 40), (1, 0), (33, 127), (7, 0), (64, 5), (40, 256)], heads, kv, dim, 16, dtype, mask=mask,
         seed=heads).check(pp)


@pytest.mark.parametrize("page", [8, 128, 256, 384])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_pages_around_the_key_tile(pp, page, dim):
    """Pages of part of a key tile, of one and of several (bf16: boxes of one page; 384 is no multiple of 256)."""
    Case([(2, 127), (1, 128), (3, 390), (1, 0), (40, 700)], 4, 2, dim, page, "bf16", seed=page + dim).check(pp)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv", [(64, 1), (48, 2), (40, 1), (7, 7)])
def test_large_and_odd_groups(pp, dtype, heads, kv):
    """Groups of more heads than a row tile's quarter holds, and groups that do not divide it."""
    Case([(1, 150), (3, 20), (7, 0)], heads, kv, 64, 16, dtype).check(pp)
    Case([(5, 130), (9, 1)], heads, kv, 64, 16, dtype, mask="tree").check(pp)


@pytest.mark.parametrize("mask", ["chain", "tree", "random"])
def test_two_row_tiles_with_hidden_values(pp, mask):
    """More than 128 query rows a key head, a non-finite value that some rows do not see, items that are split."""
    c = Case([(200, 900), (129, 3)], 4, 2, 64, 16, "bf16", mask=mask, seed=8)
    clean = Case([(200, 900), (129, 3)], 4, 2, 64, 16, "bf16", mask=mask, seed=8)
    blind = np.zeros(c.T, bool)
    for b in range(2):
        n, ctx = int(c.starts[b + 1] - c.starts[b]), int(c.ctx[b])
        j = ctx + 70
        c.v[c.pages[b, j // 16], j % 16, :, 5] = np.inf
        blind[c.starts[b]:c.starts[b + 1]] = ~ref.visible(n, ctx, c.mask, int(c.starts[b]))[:, j]
    want, tol = ref.attend(clean.q, clean.k, clean.v, clean.starts, clean.ctx, clean.pages, clean.mask, clean.scale, "bf16")
    got, status, _ = c.run(pp)
    assert status == pp.PP_OK and blind.any() and not blind.all()
    assert (np.abs(got - want)[blind] <= tol[blind]).all()
    assert not np.isfinite(got[~blind][..., 5]).any()


def test_rows_that_see_nothing_are_zero(pp):
    for dtype in ("bf16", "f32"):
        c = Case([(5, 0), (3, 10), (40, 0)], 4, 2, 64, 16, dtype, mask="none")
        got = c.check(pp)
        assert (got[:5] == 0).all() and (got[8:] == 0).all() and (got[5:8] != 0).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_mask_narrower_than_the_tree(pp, dtype):
    """Tokens past 32 * mask_words are not seen."""
    Case([(70, 20), (5, 3)], 4, 4, 64, 16, dtype, mask="random", words=1).check(pp)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,dim,seqs", [
    (4, 4, 64, [(127, 0), (128, 0), (129, 3)]),
    (8, 2, 128, [(31, 0), (33, 100), (65, 1), (200, 0)]),
    (6, 2, 128, [(43, 17), (171, 0)]),
    (3, 1, 64, [(300, 129)]),
    (2, 1, 256, [(130, 70)]),
])
def test_prompts(pp, dtype, heads, kv, dim, seqs):
    Case(seqs, heads, kv, dim, 32, dtype, seed=dim).check(pp)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_ragged_sequences(pp, dtype):
    rng = np.random.default_rng(3)
    seqs = [(int(rng.integers(0, 3)), int(rng.integers(0, 200))) for _ in range(300)] + [(0, 0), (0, 50), (1, 0)]
    Case(seqs, 4, 2, 64, 16, dtype).check(pp)


@pytest.mark.parametrize("dtype,kv", [("bf16", 1), ("f32", 1), ("bf16", 2)])
def test_one_long_sequence_is_split(pp, dtype, kv):
    """One item over most of the CTAs: the parts are joined."""
    Case([(1, 20011)], 8, kv, 64, 64, dtype).check(pp)
    Case([(9, 9001)], 8, kv, 128, 64, dtype, mask="tree").check(pp)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_unseen_entries_may_hold_anything(pp, dtype, bad):
    """Non-finite keys and values in another branch of the tree, or later in the prompt, reach only the tokens that
    see them; so does what the pages hold past the sequence."""
    c = Case([(20, 50), (30, 0)], 4, 2, 64, 16, dtype, mask="tree", seed=5, stale=bad)
    blind = np.zeros(c.T, bool)
    for b in range(2):
        n, ctx = int(c.starts[b + 1] - c.starts[b]), int(c.ctx[b])
        node = n // 2
        j = ctx + node
        c.k[c.pages[b, j // 16], j % 16] = bad
        c.v[c.pages[b, j // 16], j % 16] = bad
        see = ref.visible(n, ctx, c.mask, int(c.starts[b]))
        blind[c.starts[b]:c.starts[b + 1]] = ~see[:, j]
    clean = Case([(20, 50), (30, 0)], 4, 2, 64, 16, dtype, mask="tree", seed=5, stale=0.0)
    want, tol = ref.attend(clean.q, clean.k, clean.v, clean.starts, clean.ctx, clean.pages, clean.mask, clean.scale, dtype)
    got, status, _ = c.run(pp)
    assert status == pp.PP_OK and blind.any() and not blind.all()
    assert (np.abs(got - want)[blind] <= tol[blind]).all()
    if np.isnan(bad):
        assert np.isnan(got[~blind]).all()
    # the same in a prompt: the tokens before the bad one do not see it
    c = Case([(150, 9)], 4, 2, 64, 16, dtype, seed=6, stale=bad)
    clean = Case([(150, 9)], 4, 2, 64, 16, dtype, seed=6, stale=0.0)
    j = 9 + 100
    c.v[c.pages[0, j // 16], j % 16] = bad
    want, tol = ref.attend(clean.q, clean.k, clean.v, clean.starts, clean.ctx, clean.pages, None, clean.scale, dtype)
    got, status, _ = c.run(pp)
    assert (np.abs(got - want)[:100] <= tol[:100]).all() and not np.isfinite(got[100:]).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(pp, dtype):
    """Scores of hundreds in both directions: the running maximum moves from tile to tile."""
    Case([(3, 700), (40, 300)], 4, 2, 64, 16, dtype, std=40.0, seed=11).check(pp)
    c = Case([(1, 600)], 2, 1, 64, 16, dtype, seed=12)
    # keys that grow along the sequence, so that every tile raises the maximum
    for j in range(601):
        c.k[c.pages[0, j // 16], j % 16] = rounded(c.q[0, :1] * (j / 40.0), dtype)
    c.check(pp)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_padding_tokens_and_empty_batches(pp, dtype):
    import torch
    Case([(2, 5), (3, 70)], 4, 2, 64, 16, dtype, pad=6).check(pp)
    Case([(2, 5), (3, 70)], 4, 2, 64, 16, dtype, pad=6, mask="tree").check(pp)
    c = Case([(0, 5), (0, 0)], 4, 2, 64, 16, dtype, pad=3)
    got, status, _ = c.run(pp)
    assert status == pp.PP_OK and (got == 77.0).all()
    cache, _, _, _, _ = c.device(pp)
    ws = pp.alloc_attn_workspace(cache)
    none = pp.Batch(torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"),
                    torch.zeros((0, 1), dtype=torch.int32, device="cuda"), 0)
    e = torch.empty((0, 4, 64), dtype=cache.k.dtype, device="cuda")
    pp.pp_tree_attention(cache, none, e, None, 1.0, torch.empty_like(e), ws)
    assert pp.pp_get_device_status(ws) == pp.PP_OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_same_bits_every_time(pp, dtype):
    import torch
    c = Case([(9, 5000), (1, 3000), (20, 17), (1, 1)], 8, 2, 128, 16, dtype, mask="tree")
    a = c.run(pp)[0]
    for _ in range(3):
        assert np.array_equal(a, c.run(pp)[0])
    # and on another stream, behind work that is still running there
    cache, batch, q, mask, out = c.device(pp)
    ws = pp.alloc_attn_workspace(cache)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        late = torch.empty_like(q)
        busy = torch.randn(2048, 2048, device="cuda")
        for _ in range(20):
            busy = busy @ busy * 1e-3
        late.copy_(q)
        pp.pp_tree_attention(cache, batch, late, mask, c.scale, out, ws)
        got = out.float().cpu().numpy()
    assert np.array_equal(a, got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_graph_replay_follows_the_lengths(pp, dtype):
    """A captured call reads the lengths, pages and tokens of the replay."""
    import torch
    c = Case([(1, 400), (1, 20)], 4, 2, 64, 16, dtype)
    cache, batch, q, mask, out = c.device(pp)
    ws = pp.alloc_attn_workspace(cache)
    pp.pp_tree_attention(cache, batch, q, mask, c.scale, out, ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pp.pp_tree_attention(cache, batch, q, mask, c.scale, out, ws)
    c.ctx = np.array([123, 20], np.int32)
    batch.ctx_len.copy_(to_dev(c.ctx))
    out.fill_(77.0)
    g.replay()
    torch.cuda.synchronize()
    want, tol = ref.attend(c.q, c.k, c.v, c.starts, c.ctx, c.pages, None, c.scale, dtype)
    assert (np.abs(out.float().cpu().numpy() - want) <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_tokens(pp, dtype):
    """q and out as parts of wider rows; the rest of the rows stays."""
    import torch
    c = Case([(3, 90), (17, 4)], 4, 2, 64, 16, dtype, mask="tree")
    cache, batch, q, mask, _ = c.device(pp)
    ws = pp.alloc_attn_workspace(cache)
    wide = torch.full((c.T, 8 * 64), 3.0, dtype=q.dtype, device="cuda")
    wide[:, 128:384] = q.flatten(1)
    wout = torch.full((c.T, 300 + 20), 5.0, dtype=q.dtype, device="cuda")
    pp.pp_tree_attention(cache, batch, wide[:, 128:384], mask, c.scale, wout[:, 32:288], ws)
    want, tol = ref.attend(c.q, c.k, c.v, c.starts, c.ctx, c.pages, c.mask, c.scale, dtype)
    got = wout.float().cpu().numpy()
    assert (np.abs(got[:, 32:288].reshape(want.shape) - want) <= tol).all()
    assert (got[:, :32] == 5.0).all() and (got[:, 288:] == 5.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_beyond_32_bit_offsets(pp, dtype):
    """Pages whose byte and element offsets pass 2^32."""
    import torch
    kv, dim, page, far = 2, 64, 16, 40
    esz = 2 if dtype == "bf16" else 4
    stride = (5 << 30) // far // 16 * 16  # elements between pages: 40 pages span 5 Gi elements
    if torch.cuda.mem_get_info()[0] < 2 * 5 * (1 << 30) * esz + (4 << 30):
        pytest.skip("not enough free device memory")
    base = torch.empty(stride * (far - 1) + page * kv * dim, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32,
                       device="cuda")
    c = Case([(1, 200), (2, 30)], 4, kv, dim, page, dtype)
    n = c.k.shape[0]
    views = []
    for part, src in ((0, c.k), (page * kv * dim, c.v)):
        if part:
            base2 = torch.empty_like(base)
        t = torch.as_strided(base if not part else base2, (far, page, kv, dim), (stride, kv * dim, dim, 1))
        t[far - n:] = to_dev(src, dtype)
        views.append(t)
    cache = pp.KVCache(views[0], views[1], c.heads)
    pages = np.where(c.pages >= 0, c.pages + far - n, -1).astype(np.int32)
    batch = pp.Batch(to_dev(c.starts), to_dev(c.ctx), to_dev(pages), c.T)
    q = to_dev(c.q, dtype)
    out = torch.empty_like(q)
    ws = pp.alloc_attn_workspace(cache)
    pp.pp_tree_attention(cache, batch, q, None, c.scale, out, ws)
    want, tol = ref.attend(c.q, c.k, c.v, c.starts, c.ctx, c.pages, None, c.scale, dtype)
    assert (np.abs(out.float().cpu().numpy() - want) <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bad_lengths_and_pages_are_reported(pp, dtype):
    """Lengths and page numbers that cannot be right are recorded, nothing is read past the pages, and the other
    sequences come out right."""
    good = Case([(2, 30), (3, 40), (1, 9)], 4, 2, 64, 16, dtype)
    want, tol = ref.attend(good.q, good.k, good.v, good.starts, good.ctx, good.pages, None, good.scale, dtype)
    for how in ("page_high", "page_negative", "ctx_negative", "ctx_long"):
        c = Case([(2, 30), (3, 40), (1, 9)], 4, 2, 64, 16, dtype)
        if how == "page_high":
            c.pages[1, 1] = c.k.shape[0]
        elif how == "page_negative":
            c.pages[1, 0] = -1
        elif how == "ctx_negative":
            c.ctx[1] = -1
        else:
            c.ctx[1] = 16 * c.pages.shape[1] - 2
        got, status, _ = c.run(pp)
        assert status == pp.PP_ERR_INVALID_ARG, how
        for rows in (slice(0, 2), slice(5, 6)):
            assert (np.abs(got[rows] - want[rows]) <= tol[rows]).all(), how
        if how.startswith("ctx"):
            assert (got[2:5] == 77.0).all(), how


def test_outputs_stay_in_bounds(pp):
    """Sentinel bands around out, before and after (and between rows: test_strided_tokens)."""
    import torch
    from test_gpu_canaries import Guarded
    for dtype in ("bf16", "f32"):
        for seqs, mask in (([(1, 100), (1, 3)], "chain"), ([(33, 260), (7, 2)], "tree"), ([(150, 0)], "chain")):
            c = Case(seqs, 4, 2, 64, 16, dtype, mask=mask)
            cache, batch, q, m, _ = c.device(pp)
            g = Guarded(tuple(q.shape), q.dtype)
            ws = pp.alloc_attn_workspace(cache)
            pp.pp_tree_attention(cache, batch, q, m, c.scale, g.t, ws)
            torch.cuda.synchronize()
            assert g.bands_intact()
