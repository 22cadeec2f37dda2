"""GPU tests of tree attention as a serving loop calls it: batches of other
lengths one after the other on one workspace, as calls and as replays of one
graph.  Each call is compared with the fp64 definition within its derived
bound (attn_ref.attend), with sentinel bands around its output."""
import numpy as np
import pytest

import attn_ref as ref
from test_gpu_attention import Case, to_dev
from test_gpu_canaries import Guarded

pytestmark = pytest.mark.gpu

# (sequences, mask) of successive steps: long and empty contexts, growing and shrinking batches, and items of few
# rows, of 33 to 128 and of more than 128 rows a key head (4 query heads share one)
STEPS = [([(32, 4000)], "tree"), ([(32, 0)], "tree"), ([(9, 100)], "tree"), ([(20, 5000), (12, 700)], "tree"),
         ([(12, 5050)], "chain"), ([(1, 3000), (1, 3001)], "chain"), ([(32, 4100)], "tree"), ([(200, 900)], "chain"),
         ([(31, 2)], "chain"), ([(9, 2500), (30, 17), (25, 1300)], "tree"), ([(9, 2)], "tree")]


def step(pp, case, ws, what):
    """One call on the workspace, checked."""
    import torch
    cache, batch, q, mask, _ = case.device(pp)
    g = Guarded(tuple(q.shape), q.dtype)
    g.t.fill_(77.0)
    pp.pp_tree_attention(cache, batch, q, mask, case.scale, g.t, ws)
    torch.cuda.synchronize()
    want, tol = ref.attend(case.q, case.k, case.v, case.starts, case.ctx, case.pages, case.mask, case.scale, case.dtype)
    off = np.abs(g.t.float().cpu().numpy() - want) - tol
    assert off.max() <= 0, (what, float(off.max()), np.unravel_index(off.argmax(), off.shape))
    assert g.bands_intact(), what
    assert pp.pp_get_device_status(ws) == pp.PP_OK


@pytest.mark.parametrize("dtype,dim", [("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 64), ("f32", 128)])
def test_batches_of_other_lengths_on_one_workspace(pp, dtype, dim):
    first = Case(STEPS[0][0], 4, 1, dim, 16, dtype, mask=STEPS[0][1], stale=0.0)
    ws = pp.alloc_attn_workspace(first.device(pp)[0])
    for i, (seqs, mask) in enumerate(STEPS):
        step(pp, Case(seqs, 4, 1, dim, 16, dtype, mask=mask, seed=i), ws, (i, seqs))


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_steps_with_and_without_split_items(pp, dim):
    """Every key head's item split, then none split, then fewer tokens (records of the earlier call past the end)."""
    ws = None
    for i, seqs in enumerate([[(40, 4000)], [(40, 0)], [(33, 0)], [(40, 4100)], [(33, 50)], [(40, 3900), (35, 10)]]):
        c = Case(seqs, 4, 4, dim, 32, "bf16", mask="tree", seed=20 + i)
        ws = pp.alloc_attn_workspace(c.device(pp)[0]) if ws is None else ws
        step(pp, c, ws, (i, seqs))


@pytest.mark.parametrize("dtype,dim", [("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 64)])
@pytest.mark.parametrize("heads,kv", [(2, 2), (8, 1)])
def test_graph_replays_follow_moving_contexts(pp, dtype, dim, heads, kv):
    """One captured call of 40-row and 320-row items over contexts that grow and shrink."""
    import torch
    c = Case([(40, 4200), (40, 600)], heads, kv, dim, 16, dtype, mask="tree", seed=dim + heads, stale=0.0)
    cache, batch, q, mask, _ = c.device(pp)
    g = Guarded(tuple(q.shape), q.dtype)
    ws = pp.alloc_attn_workspace(cache)
    pp.pp_tree_attention(cache, batch, q, mask, c.scale, g.t, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pp.pp_tree_attention(cache, batch, q, mask, c.scale, g.t, ws)
    for ctx in ([4200, 600], [0, 0], [4100, 599], [60, 600], [2000, 0], [4200, 1]):
        c.ctx = np.array(ctx, np.int32)
        batch.ctx_len.copy_(to_dev(c.ctx))
        g.t.fill_(77.0)
        graph.replay()
        torch.cuda.synchronize()
        want, tol = ref.attend(c.q, c.k, c.v, c.starts, c.ctx, c.pages, c.mask, c.scale, dtype)
        assert (np.abs(g.t.float().cpu().numpy() - want) <= tol).all(), ctx
        assert g.bands_intact() and pp.pp_get_device_status(ws) == pp.PP_OK


def test_example_steps_split_items_in_bf16(pp):
    """The decoding example's layer stack in bf16 with a context long enough that tree steps split their items: the
    logits of a step computed on a workspace that earlier steps used are the bits of a fresh workspace."""
    import os
    import sys
    import torch
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import tree_decode as td
    model = td.TreeDecoder(dtype="bf16", heads=4, kv_heads=1, max_tokens=2048)
    text = [(7 * i) % 23 for i in range(1400)]
    for i in range(0, 1200, 60):
        model.forward(text[i:i + 60])
        model.commit(list(range(60)))
    lengths = [31, 12, 24, 9]
    for i, n in enumerate(lengths):
        nodes = [(text[1200 + i], -1)] + [(text[j], (5 * j + 3) % j) for j in range(1, n)]
        depths, mask = td.tree_tensors(nodes)
        tokens = [t for t, _ in nodes]
        used = model.forward(tokens, depths, mask)
        kept, model.ws = model.ws, pp.alloc_attn_workspace(model.caches[0])
        fresh = model.forward(tokens, depths, mask)
        model.ws = kept
        assert torch.equal(used, fresh), n
        model.commit([0])
    model.check()


def test_a_recorded_error_does_not_end_long_waits(pp):
    """A bad length beside a sequence whose items take several ms: warps wait that long for one another, and the
    recorded error must not end the waits.  152 key heads of 8 over 262144 entries, which are 512 different ones 512
    times over, so that the definition has 512 + n distinct entries with known multiplicities."""
    import torch
    H, D, page, uniq, times, n = 152, 8, 128, 512, 512, 300
    ctx = uniq * times
    rng = np.random.default_rng(0)

    def bf16(a):
        return torch.from_numpy(a.astype(np.float32)).to(torch.bfloat16).float().numpy()

    n_pages = uniq // page + 3
    k, v = (bf16(rng.standard_normal((n_pages, page, H, D)) + shift) for shift in (0.0, 0.5))
    q = bf16(rng.standard_normal((n + 1, H, D)))
    table = np.full((2, ctx // page + 3), -1, np.int32)
    table[0, :ctx // page] = np.tile(np.arange(uniq // page), times)
    table[0, ctx // page:] = uniq // page + np.arange(3)
    cache = pp.KVCache(to_dev(k, "bf16"), to_dev(v, "bf16"), H)
    batch = pp.Batch(to_dev(np.array([0, n, n + 1], np.int32)), to_dev(np.array([ctx, -1], np.int32)), to_dev(table), n + 1)
    out = torch.full((n + 1, H, D), 77.0, dtype=torch.bfloat16, device="cuda")
    ws = pp.alloc_attn_workspace(cache)
    scale = float(np.float32(D ** -0.5))
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    qd = to_dev(q, "bf16")
    torch.cuda.synchronize()
    begin.record()
    pp.pp_tree_attention(cache, batch, qd, None, scale, out, ws)
    end.record()
    assert pp.pp_get_device_status(ws) == pp.PP_ERR_INVALID_ARG
    # the items of a key head (256 and 44 rows) take about half of it each: waits over 1 ms
    assert begin.elapsed_time(end) > 4.0
    got = out.float().cpu().numpy()
    assert (got[n] == 77.0).all()
    kk, vv = (a.reshape(-1, H, D).astype(np.float64)[:uniq + n] for a in (k, v))
    weight = np.concatenate([np.full(uniq, float(times)), np.ones(n)])
    see = np.concatenate([np.ones((n, uniq), bool), np.tril(np.ones((n, n), bool))], 1)
    for h in range(0, H, 7):
        s = scale * (q[:n, h].astype(np.float64) @ kk[:, h].T)
        top = np.where(see, s, -np.inf).max(1, keepdims=True)
        p = np.where(see, weight * np.exp(s - top), 0.0)
        p /= p.sum(1, keepdims=True)
        want, a = p @ vv[:, h], p @ np.abs(vv[:, h])
        # attn_ref.attend's bound, the sums over all ctx + n entries
        eps = ref.F32_HALF_ULP * ((D + 4) * scale * (np.abs(q[:n, h]) @ np.abs(kk[:, h]).T).max(1, keepdims=True)
                                  + 4 * np.abs(s).max(1, keepdims=True))
        t = (2 * np.expm1(2 * eps) + 2.0 ** -20 + 2 * ref.F32_HALF_ULP * ((ctx + n) / 32 + 32) + 2 * ref.BF16_HALF_ULP) * a
        tol = t + ref.BF16_HALF_ULP * (np.abs(want) + t)
        assert (np.abs(got[:n, h] - want) <= tol).all(), h


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,heads", [(5, 4), (40, 2), (90, 4)])
def test_pages_that_do_not_exist_read_as_zeros_beside_hidden_values(pp, dtype, n, heads):
    """A page number out of range in the context of rows that do not see a NaN: its entries are zeros for them too."""
    c = Case([(n, 100), (2, 9)], heads, 1, 64, 16, dtype, mask="tree", seed=n, stale=0.0)
    j = 100 + n // 2
    blind = ~ref.visible(n, 100, c.mask, 0)[:, j]
    k, v = (np.concatenate([a, np.zeros_like(a[:1])]) for a in (c.k, c.v))
    c.pages[0, 2] = c.k.shape[0]
    want, tol = ref.attend(c.q, k, v, c.starts, c.ctx, c.pages, c.mask, c.scale, dtype)
    c.v[c.pages[0, j // 16], j % 16, :, 3] = np.nan
    got, status, _ = c.run(pp)
    assert status == pp.PP_ERR_INVALID_ARG and blind.any() and not blind.all()
    ok = np.abs(got - want) <= tol
    assert ok[:n][blind].all() and ok[n:].all()
    ok[:n, :, 3] = True
    assert ok.all() and np.isnan(got[:n][~blind][..., 3]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", ["chain", "tree"])
@pytest.mark.parametrize("n,heads,ctx,page", [(3, 4, 70, 16), (20, 4, 500, 7), (40, 1, 300, 64), (150, 2, 40, 16), (300, 1, 0, 16)])
def test_non_finite_values_reach_the_rows_that_see_them(pp, dtype, mask, n, heads, ctx, page):
    """NaN and infinities of both signs in elements of several new tokens' values, a tile's edges among them: an
    element is what the definition gives (an infinity of a seen value, NaN where both signs or a NaN are seen), every
    other element and row stays within the bound."""
    c = Case([(n, ctx), (4, 33)], heads, 1, 64, page, dtype, mask=mask, seed=n, stale=0.0)
    want, tol = ref.attend(c.q, c.k, c.v, c.starts, c.ctx, c.pages, c.mask, c.scale, dtype)
    see = ref.visible(n, ctx, c.mask, 0)
    hit = np.zeros((n, 64))
    places = {(node, elem): bad for node, elem, bad in  # where two meet, the last stays
              [(0, 0, np.nan), (n // 2, 9, np.inf), (n - 1, 17, -np.inf), (n // 3, 63, np.inf), (n // 2, 63, -np.inf),
               (min(n - 1, 127), 31, np.inf), (min(n - 1, 128), 32, -np.inf)]}
    for (node, elem), bad in places.items():
        j = ctx + node
        c.v[c.pages[0, j // page], j % page, :, elem] = bad
        with np.errstate(invalid="ignore"):
            hit[see[:, j], elem] += bad
    got, status, _ = c.run(pp)
    assert status == pp.PP_OK
    fine = np.isfinite(hit)
    assert fine.any() and not fine.all()
    for h in range(heads):
        assert (np.abs(got[:n, h] - want[:n, h]) <= tol[:n, h])[fine].all()
        assert not np.isfinite(got[:n, h][~fine]).any()
        assert np.isnan(got[:n, h][np.isnan(hit)]).all()
    assert (np.abs(got[n:] - want[n:]) <= tol[n:]).all()


@pytest.mark.parametrize("heads", [1, 4])
def test_a_non_finite_value_costs_no_pass_over_the_context(pp, heads):
    """Rows that see a NaN of a drafted token, over a long context: at most 4 times the time without it."""
    import torch
    times = []
    for bad in (0.0, np.nan):
        c = Case([(40, 150000)], heads, 1, 128, 64, "bf16", mask="tree", seed=1, stale=0.0)
        for j in range(150000, 150040):
            c.v[c.pages[0, j // 64], j % 64, :, 0] = bad
        cache, batch, q, mask, out = c.device(pp)
        ws = pp.alloc_attn_workspace(cache)
        best = 1e9
        for _ in range(6):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            pp.pp_tree_attention(cache, batch, q, mask, c.scale, out, ws)
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b))
        times.append(best)
        assert pp.pp_get_device_status(ws) == pp.PP_OK
    assert torch.isnan(out[..., 0]).all() and torch.isfinite(out[..., 1:]).all()
    assert times[1] <= 4 * times[0], times


@pytest.mark.parametrize("n,heads", [(300, 152), (20, 456)])
def test_waits_that_give_up_end_the_call(pp, n, heads):
    """Waits over 1 ms give up on a workspace that has a timeout recorded: the call returns with that status, writes
    nothing beside its output, and leaves the GPU usable; on the workspace initialised anew it comes out right."""
    import torch
    D, page, uniq, times = 8, 128, 512, 1024
    ctx = uniq * times
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((uniq // page + 3, page, heads, D), generator=g, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn((n, heads, D), generator=g, device="cuda").bfloat16()
    table = torch.cat([torch.arange(uniq // page).repeat(times), uniq // page + torch.arange(3)]).int()[None].cuda()
    cache = pp.KVCache(k, v, heads)
    batch = pp.Batch(torch.tensor([0, n], dtype=torch.int32, device="cuda"),
                     torch.tensor([ctx], dtype=torch.int32, device="cuda"), table, n)
    ws = pp.alloc_attn_workspace(cache)
    out = Guarded((n, heads, D), torch.bfloat16)
    pp.pp_debug_wait_timeout(ws, 1000)
    pp.pp_tree_attention(cache, batch, q, None, D ** -0.5, out.t, ws)
    assert pp.pp_get_device_status(ws) == pp.PP_ERR_TIMEOUT
    assert out.bands_intact()
    pp.pp_workspace_init(ws)
    pp.pp_tree_attention(cache, batch, q, None, D ** -0.5, out.t, ws)
    assert pp.pp_get_device_status(ws) == pp.PP_OK and out.bands_intact()
    fresh = torch.empty_like(out.t)
    pp.pp_tree_attention(cache, batch, q, None, D ** -0.5, fresh, pp.alloc_attn_workspace(cache))
    assert torch.equal(out.t, fresh) and torch.isfinite(fresh).all()
    # every cached entry counts `times` times; the first head in fp64
    kk, vv = (a.reshape(-1, heads, D)[:uniq + n, 0].double() for a in (k, v))
    s = q[:, 0].double() @ kk.T * D ** -0.5
    s[:, uniq:].masked_fill_(torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1), float("-inf"))
    p = torch.softmax(s + torch.cat([torch.full((uniq,), np.log(times)), torch.zeros(n)]).cuda().double(), -1)
    want, a = p @ vv, p @ vv.abs()
    # two roundings to bf16 of the weights and one of the output, sums of ctx + n terms (attn_ref.attend's bound)
    rel = 3 * ref.BF16_HALF_ULP + 2.0 ** -20 + 2 * ref.F32_HALF_ULP * ((ctx + n) / 32 + 32) + 1e-4
    assert ((fresh[:, 0].double() - want).abs() <= rel * a).all()
