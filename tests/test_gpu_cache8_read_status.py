"""GPU test of the status that pp_kvq_read leaves: none for an intact table, PP_ERR_INVALID_ARG for a page that does not
exist; and the rows that were zeros for want of it are the held values once it is there."""
import numpy as np
import pytest

import cache8_ref as ref
from test_gpu_attention import to_dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("missing", [-1, 9, 2 ** 31 - 1])
@pytest.mark.parametrize("page,block", [(16, 16), (64, 32)])
def test_status_of_a_read(pp, dtype, missing, page, block):
    import torch
    kv, dim, dt = 2, 64, torch.bfloat16 if dtype == "bf16" else torch.float32
    held = [ref.quantised(np.random.default_rng(i).standard_normal((9, page, kv, dim)), block) for i in range(2)]
    cache = pp.KVCache8(*[to_dev(c.code) for c in held], *[to_dev(c.scale) for c in held], kv, dt)
    table = np.random.default_rng(2).permutation(9)[:6].astype(np.int32).reshape(2, 3)
    n = 2 * page + 5  # tokens of each sequence, the third page in part
    starts, ctx = np.array([0, n, 2 * n], np.int32), np.array([0, 3], np.int32)

    def read(table):
        ws = pp.alloc_kvq_workspace(cache)
        out = [torch.full((2 * n, kv, dim), 9.0, dtype=dt, device="cuda") for _ in range(2)]
        pp.pp_kvq_read(cache, pp.Batch(to_dev(starts), to_dev(ctx), to_dev(table), 2 * n), *out, ws)
        return pp.pp_get_device_status(ws), [o.float().cpu().numpy() for o in out]

    status, whole = read(table)
    assert status == pp.PP_OK
    cut = table.copy()
    cut[1, 1] = missing
    status, got = read(cut)
    assert status == pp.PP_ERR_INVALID_ARG
    gone = np.zeros(2 * n, bool)
    gone[n + page - 3:n + 2 * page - 3] = True  # entries page .. 2 page - 1 of the second sequence
    for x, y, c in zip(whole, got, held):
        want = np.concatenate([c.values()[table[b, (ctx[b] + np.arange(n)) // page], (ctx[b] + np.arange(n)) % page] for b in range(2)])
        assert np.array_equal(x, want.astype(np.float32))
        assert (y[gone] == 0).all() and np.array_equal(y[~gone], x[~gone]) and (x[gone] != 0).any()
