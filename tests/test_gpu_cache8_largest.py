"""GPU tests of the 8-bit cache at the upper end of the numbers: what is finite comes back finite.  At the scale 2^120 the
code 256 would be 2^128, so that magnitudes from 248 * 2^120 on become 240 * 2^120, the largest value held."""
import numpy as np
import pytest

import cache8_ref as ref
from test_gpu_attention import rounded, to_dev

pytestmark = pytest.mark.gpu

TOP = 240.0 * 2.0 ** 120
ROWS = [255.0 * 2.0 ** 120, -255.0 * 2.0 ** 120, 248.0 * 2.0 ** 120, 247.0 * 2.0 ** 120, 232.0 * 2.0 ** 120, 1.0]


def held(x, now):
    """What x (finite) is held as at the scales `now`: the nearest code's value, 240 * 2^120 at most."""
    y = ref.VALUES[ref.codes_of(np.clip(x / now, -448, 448))] * now
    return np.where(np.abs(y) > TOP, np.sign(y) * TOP, y)


def setup(pp, dtype, dim, block, lengths, layers=1):
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    kv, page, per = 3, block, 4
    code = torch.zeros((2, layers, per * len(lengths), page, kv, dim), dtype=torch.uint8, device="cuda")
    scale = torch.ones((2, layers, per * len(lengths), kv, 1), dtype=torch.float32, device="cuda")
    cache = pp.KVCache8(code[0, 0], code[1, 0], scale[0, 0], scale[1, 0], kv, dt)
    table = np.arange(per * len(lengths), dtype=np.int32).reshape(len(lengths), per)
    return dt, kv, code, scale, cache, table, pp.alloc_kvq_workspace(cache)


def batch(pp, new, ctx, table):
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    return pp.Batch(to_dev(starts), to_dev(np.array(ctx, np.int32)), to_dev(table), int(starts[-1]))


def read(pp, cache, b, kv, dim, dt, ws):
    import torch
    out = [torch.empty((b.n_tokens, kv, dim), dtype=dt, device="cuda") for _ in range(2)]
    pp.pp_kvq_read(cache, b, *out, ws)
    return [o.float().cpu().numpy() for o in out]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,block", [(16, 16), (128, 16), (256, 128), (80, 64)])
def test_largest_numbers_come_back_finite(pp, dtype, dim, block):
    """New blocks, and blocks whose scale grows to the largest one under cached entries."""
    import torch
    dt, kv, code, scale, cache, table, ws = setup(pp, dtype, dim, block, [0, 0])
    rng = np.random.default_rng(dim)
    first = rng.standard_normal((2, 3, kv, dim))          # three entries of each sequence, of ordinary size
    first[1] *= 2.0 ** 111                                 # the second's: something is left of them at the scale 2^120
    first = rounded(first, dtype)
    x = to_dev(first.reshape(6, kv, dim), dtype)
    pp.pp_kvq_append(cache, batch(pp, [3, 3], [0, 0], table), None, None, None, None, x, x, None, ws)
    last = rounded(np.resize(ROWS, (2, 2, kv, dim)), dtype)
    if dtype == "f32":
        last[:, 1, :, 5] = np.finfo(np.float32).max
    x = to_dev(last.reshape(4, kv, dim), dtype)
    pp.pp_kvq_append(cache, batch(pp, [2, 2], [3, 3], table), None, None, None, None, x, x, None, ws)
    whole = batch(pp, [5, 5], [0, 0], table)
    assert np.isfinite(last).all()
    assert (scale[:, 0, [0, 4]] == 2.0 ** 120).all()
    old = [np.array(ref.scale_for(ref.largest(f.astype(np.float64), (0, 2)))) for f in first]
    for got in read(pp, cache, whole, kv, dim, dt, ws):
        got = got.reshape(2, 5, kv, dim).astype(np.float64)
        assert np.isfinite(got).all()
        for b in range(2):
            cached = held(first[b].astype(np.float64), old[b][:, None])
            assert np.array_equal(got[b, :3], held(cached, 2.0 ** 120))
            assert np.array_equal(got[b, 3:], held(last[b].astype(np.float64), 2.0 ** 120))
    # one visible entry: its values, rounded once
    out = torch.empty((4, kv, dim), dtype=dt, device="cuda")
    mask = torch.tensor([1, 2, 1, 2], dtype=torch.int32, device="cuda")[:, None]
    pp.pp_kvq_append(cache, batch(pp, [2, 2], [0, 0], table), None, None, None, None, to_dev(np.zeros((4, kv, dim), np.float32), dtype), x,
                     None, ws)
    pp.pp_kvq_tree_attention(cache, batch(pp, [2, 2], [0, 0], table), x * 0, mask, 1.0, out, ws)
    got = out.float().cpu().numpy().reshape(2, 2, kv, dim)
    assert np.array_equal(got, held(last.astype(np.float64), 2.0 ** 120).astype(np.float32))
    assert pp.pp_get_device_status(ws) == pp.PP_OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales_filled_elsewhere(pp, dtype):
    """A cached block's scale that is kept, of no power of two: the codes of new entries stay at finite values too."""
    dt, kv, code, scale, cache, table, ws = setup(pp, dtype, 64, 16, [0, 0])
    for s in (0.75 * 2.0 ** 120, 2.0 ** 125, 1.7 * 2.0 ** 119):
        scale.fill_(s)
        x = to_dev(np.resize(ROWS, (2, kv, 64)).astype(np.float32), dtype)
        pp.pp_kvq_append(cache, batch(pp, [1, 1], [3, 3], table), None, None, None, None, x, x, None, ws)
        assert (scale[:, 0, [0, 4]] == s).all()
        for got in read(pp, cache, batch(pp, [1, 1], [3, 3], table), kv, 64, dt, ws):
            f = x.float().cpu().numpy().astype(np.float64)
            assert np.isfinite(got).all()
            # half a code's step, and what lies past the largest code below infinity: a step of 1/8
            assert (np.abs(got - f) <= np.where(np.abs(f) > 200 * 2.0 ** 120, 0.125, 2.0 ** -4 + 2.0 ** -8) * np.abs(f)
                    + s * 2.0 ** -10).all()


@pytest.mark.parametrize("block", [16, 128])
def test_commit_to_the_largest_scale(pp, block):
    """Accepted entries of the largest scale move into blocks with smaller ones, and back to finite numbers."""
    dt, kv, code, scale, cache, table, ws = setup(pp, "f32", 64, block, [0, 0])
    rng = np.random.default_rng(0)
    small = (rng.standard_normal((2, 3, kv, 64)) * 2.0 ** 112).astype(np.float32)
    draft = (rng.standard_normal((2, block + 4, kv, 64)) * 2.0 ** 112).astype(np.float32)
    draft[:, block] = np.resize(ROWS, (kv, 64))
    draft[:, block, :, 7] = np.finfo(np.float32).max
    for x, ctx in ((small, 0), (draft, 3)):
        t = to_dev(x.reshape(-1, kv, 64))
        pp.pp_kvq_append(cache, batch(pp, [x.shape[1]] * 2, [ctx] * 2, table), None, None, None, None, t, t, None, ws)
    b = batch(pp, [block + 4] * 2, [3, 3], table)
    before = [r.reshape(2, block + 4, kv, 64) for r in read(pp, cache, b, kv, 64, dt, ws)]
    pp.pp_kvq_commit(cache, b, to_dev(np.full((2, 1), block, np.int32)), to_dev(np.ones(2, np.int32)), ws)
    after = read(pp, cache, batch(pp, [1, 1], [3, 3], table), kv, 64, dt, ws)
    for x, y in zip(before, after):
        assert np.isfinite(x).all() and np.array_equal(x[:, block], y)
    assert pp.pp_get_device_status(ws) == pp.PP_OK
