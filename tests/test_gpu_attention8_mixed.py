"""GPU tests of batches over the 8-bit cache whose sequences go to two kernels: long ones beside single tokens.  Every row
is written, once, by one of them, within the bound of attn_ref.attend; padding and skipped sequences stay as they were."""
import numpy as np
import pytest

import attn_ref
from test_gpu_attention import to_dev
from test_gpu_attention8 import Case8

pytestmark = pytest.mark.gpu

SINGLES = [(1, c) for c in (0, 1, 40, 127, 128, 300, 17, 5, 250, 64)]


def shares(c, kv):
    """Whether the case is one that the two kernels share: at most 16 rows a key head on average, above 512 of one sequence."""
    g, n = c.heads // kv, len(c.ctx)
    return -(-c.T * g // n) <= 16 and (c.T - n + 1) * g > 512


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,dim,page,block,mask", [(8, 2, 64, 16, 16, "chain"), (4, 1, 128, 48, 16, "tree"),
                                                         (8, 8, 128, 64, 64, "chain"), (16, 2, 64, 32, 32, "random"),
                                                         (4, 2, 256, 16, 16, "chain")])
def test_a_prompt_beside_single_tokens(pp, dtype, heads, kv, dim, page, block, mask):
    g = heads // kv
    long = 515 // g + 1
    around = [(16 // g, 33), (16 // g + 1, 20), (0, 9), (2, 0)]  # at the rows that divide the two
    seqs = (SINGLES * 20)[:long * g // 8] + [(long, 90)] + around + SINGLES
    c = Case8(seqs, heads, kv, dim, page, block, dtype, mask=mask, seed=heads, pad=3)
    assert shares(c, kv)
    c.check(pp)


def test_all_tokens_of_one_sequence(pp):
    """One long sequence among empty ones: no mean tells, the result is the same."""
    c = Case8([(0, 5)] * 30 + [(300, 60)] + [(0, 0)] * 299, 4, 1, 64, 16, 16, "bf16")
    c.check(pp)
    c = Case8([(0, 5)] * 30 + [(300, 60)] + [(0, 0)] * 100, 4, 1, 64, 16, 16, "bf16", mask="tree")
    assert shares(c, 1)
    c.check(pp)


def test_bits_graphs_and_bad_sequences(pp):
    """The same bits every time and from a graph, whose sequences change sides between replays; a bad sequence of either
    side leaves the others' results."""
    import torch
    n = [1] * 60 + [140] + [1] * 30
    c = Case8([(a, 100 + 7 * i) for i, a in enumerate(n)], 4, 1, 128, 16, 16, "bf16")
    assert shares(c, 1)
    first = c.run(pp)[0]
    assert np.array_equal(first, c.run(pp)[0])
    cache, batch, q, mask, out = c.device(pp)
    ws = pp.alloc_kvq_workspace(cache)
    pp.pp_kvq_tree_attention(cache, batch, q, mask, c.scale, out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pp.pp_kvq_tree_attention(cache, batch, q, mask, c.scale, out, ws)
    out.fill_(77.0)
    graph.replay()
    torch.cuda.synchronize()
    assert np.array_equal(out.float().cpu().numpy(), first)
    # the prompt's first tokens given to the sequence before it, which then has few rows, or many (the entries are there)
    for split in (5, 139):
        starts = c.starts.copy()
        starts[60] += split
        batch.q_start.copy_(to_dev(starts))
        ctx = c.ctx.copy()
        ctx[59:61] = 20
        batch.ctx_len.copy_(to_dev(ctx))
        out.fill_(77.0)
        graph.replay()
        torch.cuda.synchronize()
        want, tol = attn_ref.attend(c.q, c.k, c.v, starts, ctx, c.pages, None, c.scale, "bf16")
        assert (np.abs(out.float().cpu().numpy() - want) <= tol).all()
    assert pp.pp_get_device_status(ws) == pp.PP_OK
    for b in (3, 60):
        d = Case8([(a, 100 + 7 * i) for i, a in enumerate(n)], 4, 1, 128, 16, 16, "bf16")
        d.ctx[b] = -1
        got, status, _ = d.run(pp)
        assert status == pp.PP_ERR_INVALID_ARG
        mine = np.zeros(c.T, bool)
        mine[c.starts[b]:c.starts[b + 1]] = True
        assert (got[mine] == 77.0).all()
        want, tol = c.want()
        assert (np.abs(got - want)[~mine] <= tol[~mine]).all()
