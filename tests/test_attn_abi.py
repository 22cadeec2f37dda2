"""Checks of the attention-side entry points that need no GPU: refusals (before
any CUDA call, with the documented status) and the frequency tables of
scaled rotary positions against their formulas."""
import ctypes
import math

import numpy as np
import pytest

from paper_2605_28283_gb300 import binding as pp
from paper_2605_28283_gb300 import build as ppbuild

A = 0x10000  # an aligned address; nothing dereferences it
BIG = 1 << 40
NO_GPU = (pp.PP_ERR_CUDA, pp.PP_ERR_UNSUPPORTED, pp.PP_OK)


@pytest.fixture(scope="module")
def lib():
    ppbuild.build()
    return pp.load()


def cache(**kw):
    d = dict(dtype=pp.PP_BF16, n_heads=32, n_kv_heads=8, head_dim=128, page_size=16, n_pages=10, page_stride=16 * 1024,
             token_stride=1024, head_stride=128, k=A, v=A)
    d.update(kw)
    return pp.pp_cache(*[d[n] for n, _ in pp.pp_cache._fields_])


def batch(**kw):
    d = dict(n_seqs=2, n_tokens=5, max_pages=4, q_start=A, ctx_len=A, pages=A)
    d.update(kw)
    return pp.pp_batch(*[d[n] for n, _ in pp.pp_batch._fields_])


def rotation(**kw):
    d = dict(rot_dim=128, layout=pp.PP_ROPE_HALF, scale=1.0, inv_freq=A)
    d.update(kw)
    return pp.pp_rotation(*[d[n] for n, _ in pp.pp_rotation._fields_])


def ref_or_none(x):
    return None if x is None else ctypes.byref(x)


def append(lib, c=None, b=None, r=None, pos=None, q=A, qs=4096, k=2 * A, ks=1024, v=3 * A, vs=1024, o=A * 16, os_=4096,
           ws=A, n=BIG):
    return lib.pp_kv_append(ref_or_none(c or cache()), ref_or_none(b or batch()), ref_or_none(r), pos, q, qs, k, ks, v,
                            vs, o, os_, ws, n, None)


def attend(lib, c=None, b=None, q=A, qs=4096, mask=None, words=0, scale=0.1, o=A * 16, os_=4096, ws=A, n=BIG):
    return lib.pp_tree_attention(ref_or_none(c or cache()), ref_or_none(b or batch()), q, qs, mask, words, scale, o, os_,
                                 ws, n, None)


def commit(lib, c=None, b=None, layers=1, ls=0, path=A, mp=8, acc=2 * A, new=None, ws=A, n=BIG):
    return lib.pp_kv_commit(ref_or_none(c or cache()), ref_or_none(b or batch()), layers, ls, path, mp, acc, new, ws, n,
                            None)


BAD_CACHES = [(dict(dtype=5), pp.PP_ERR_DTYPE), (dict(n_heads=0), pp.PP_ERR_SHAPE), (dict(n_heads=2048), pp.PP_ERR_SHAPE),
              (dict(n_kv_heads=5), pp.PP_ERR_SHAPE), (dict(n_kv_heads=0), pp.PP_ERR_SHAPE),
              (dict(head_dim=0), pp.PP_ERR_SHAPE), (dict(head_dim=12), pp.PP_ERR_SHAPE),
              (dict(head_dim=264), pp.PP_ERR_SHAPE), (dict(page_size=0), pp.PP_ERR_SHAPE),
              (dict(n_pages=0), pp.PP_ERR_SHAPE), (dict(k=0), pp.PP_ERR_INVALID_ARG), (dict(v=A + 8), pp.PP_ERR_ALIGN),
              (dict(token_stride=1020), pp.PP_ERR_ALIGN), (dict(head_stride=-8), pp.PP_ERR_INVALID_ARG)]
BAD_BATCHES = [(dict(n_seqs=-1), pp.PP_ERR_SHAPE), (dict(n_tokens=-1), pp.PP_ERR_SHAPE), (dict(max_pages=-1), pp.PP_ERR_SHAPE),
               (dict(n_tokens=1 << 27), pp.PP_ERR_SHAPE), (dict(q_start=0), pp.PP_ERR_INVALID_ARG),
               (dict(ctx_len=0), pp.PP_ERR_INVALID_ARG), (dict(pages=0), pp.PP_ERR_INVALID_ARG),
               (dict(pages=A + 2), pp.PP_ERR_ALIGN)]


@pytest.mark.parametrize("call", [append, attend, commit])
def test_caches_batches_and_workspaces_are_checked(lib, call):
    assert call(lib) in NO_GPU[:2] or __import__("torch").cuda.is_available()
    for kw, want in BAD_CACHES:
        assert call(lib, c=cache(**kw)) == want, kw
    for kw, want in BAD_BATCHES:
        assert call(lib, b=batch(**kw)) == want, kw
    assert call(lib, ws=0) == pp.PP_ERR_WORKSPACE
    assert call(lib, ws=A + 16) == pp.PP_ERR_WORKSPACE
    need = lib.pp_attn_workspace_size(ctypes.byref(cache()))
    assert need % 256 == 0 and need > 0
    assert call(lib, n=need - 1) == pp.PP_ERR_WORKSPACE
    assert call.__name__ == "commit" or call(lib, qs=4095) == pp.PP_ERR_INVALID_ARG
    assert call.__name__ == "commit" or call(lib, qs=4100) == pp.PP_ERR_ALIGN


def test_null_structs(lib):
    c, b = cache(), batch()
    assert lib.pp_kv_append(None, ctypes.byref(b), None, None, A, 4096, A, 1024, A, 1024, A, 4096, A, BIG, None) == pp.PP_ERR_INVALID_ARG
    assert lib.pp_tree_attention(ctypes.byref(c), None, A, 4096, None, 0, 1.0, A, 4096, A, BIG, None) == pp.PP_ERR_INVALID_ARG
    assert lib.pp_kv_commit(None, None, 1, 0, A, 1, A, None, A, BIG, None) == pp.PP_ERR_INVALID_ARG
    assert lib.pp_attn_workspace_size(None) == 0
    assert lib.pp_attn_workspace_size(ctypes.byref(cache(n_kv_heads=3))) == 0


def test_append_refusals(lib):
    assert append(lib, k=0) == pp.PP_ERR_INVALID_ARG
    assert append(lib, v=3 * A + 4) == pp.PP_ERR_ALIGN
    assert append(lib, q=None) == pp.PP_ERR_INVALID_ARG      # q without q_out
    assert append(lib, o=None) == pp.PP_ERR_INVALID_ARG
    assert append(lib, q=A, o=A + 64) == pp.PP_ERR_INVALID_ARG  # overlapping, not in place
    assert append(lib, k=16 * A) == pp.PP_ERR_INVALID_ARG    # q_out over k
    assert append(lib, pos=A + 1) == pp.PP_ERR_ALIGN
    for kw, want in [(dict(rot_dim=2), pp.PP_ERR_SHAPE), (dict(rot_dim=6), pp.PP_ERR_SHAPE), (dict(rot_dim=132), pp.PP_ERR_SHAPE),
                     (dict(layout=2), pp.PP_ERR_INVALID_ARG), (dict(scale=float("nan")), pp.PP_ERR_INVALID_ARG),
                     (dict(inv_freq=0), pp.PP_ERR_INVALID_ARG)]:
        assert append(lib, r=rotation(**kw)) == want, kw
    # the parts of one fused projection, queries rotated in place, are not an overlap
    row = 4096 + 2048
    assert append(lib, q=A, qs=row, o=A, os_=row, k=A + 8192, ks=row, v=A + 10240, vs=row) in NO_GPU[:2] or \
        __import__("torch").cuda.is_available()


def test_attend_refusals(lib):
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert attend(lib, scale=scale) == pp.PP_ERR_INVALID_ARG
    assert attend(lib, mask=A, words=0) == pp.PP_ERR_INVALID_ARG
    assert attend(lib, mask=A + 2, words=1) == pp.PP_ERR_ALIGN
    assert attend(lib, o=A) == pp.PP_ERR_INVALID_ARG
    assert attend(lib, q=0) == pp.PP_ERR_INVALID_ARG


def test_commit_refusals(lib):
    assert commit(lib, layers=0) == pp.PP_ERR_SHAPE
    assert commit(lib, mp=-1) == pp.PP_ERR_SHAPE
    assert commit(lib, layers=2, ls=-8) == pp.PP_ERR_INVALID_ARG
    assert commit(lib, layers=2, ls=12) == pp.PP_ERR_ALIGN
    assert commit(lib, path=None) == pp.PP_ERR_INVALID_ARG
    assert commit(lib, acc=None) == pp.PP_ERR_INVALID_ARG
    assert commit(lib, new=2 * A) == pp.PP_ERR_INVALID_ARG  # over n_accept
    assert commit(lib, new=3 * A + 1) == pp.PP_ERR_ALIGN


def test_rope_refusals(lib):
    def rope(dtype=pp.PP_F32, r=None, pos=A, T=4, H=2, D=128, x=A, xs=256, y=A * 4, ys=256):
        return lib.pp_rope(dtype, ref_or_none(r or rotation()), pos, T, H, D, x, xs, y, ys, 0, None)
    assert rope() in NO_GPU[:2] or __import__("torch").cuda.is_available()
    assert rope(y=A) in NO_GPU[:2] or __import__("torch").cuda.is_available()
    assert rope(dtype=3) == pp.PP_ERR_DTYPE
    assert rope(T=-1) == pp.PP_ERR_SHAPE
    assert rope(H=0) == pp.PP_ERR_SHAPE
    assert rope(D=126, r=rotation(rot_dim=64)) == pp.PP_ERR_SHAPE
    assert rope(D=64) == pp.PP_ERR_SHAPE  # rot_dim past the head
    assert rope(x=None) == pp.PP_ERR_INVALID_ARG
    assert rope(pos=None) == pp.PP_ERR_INVALID_ARG
    assert rope(xs=255) == pp.PP_ERR_INVALID_ARG
    assert rope(xs=258) == pp.PP_ERR_ALIGN
    assert rope(y=A + 16) == pp.PP_ERR_INVALID_ARG
    assert lib.pp_rope(pp.PP_F32, None, A, 1, 1, 128, A, 128, A, 128, 0, None) == pp.PP_ERR_INVALID_ARG


def test_binding_refuses_wrong_tensors(lib):
    import torch
    k = torch.zeros((3, 16, 2, 64), dtype=torch.bfloat16)
    cache_ = pp.KVCache(k, k.clone(), 4)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)
    b = pp.Batch(i32(0, 2), i32(5), torch.zeros((1, 2), dtype=torch.int32), 2)
    ws = torch.zeros(256, dtype=torch.uint8)
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    for bad in (q.float(), q[:1], torch.zeros((2, 64, 4), dtype=torch.bfloat16).transpose(1, 2), q[:, :3]):
        with pytest.raises(pp.PPError):
            pp.pp_tree_attention(cache_, b, bad, None, 1.0, torch.empty_like(q), ws, stream=0)
    with pytest.raises(pp.PPError):
        pp.pp_tree_attention(cache_, b, q, torch.zeros((2, 1), dtype=torch.int64), 1.0, torch.empty_like(q), ws, stream=0)
    with pytest.raises(pp.PPError):
        pp.KVCache(k.half(), k.half(), 4)
    with pytest.raises(pp.PPError):
        pp.KVCache(k, k.transpose(0, 1).contiguous().transpose(0, 1), 4)
    with pytest.raises(pp.PPError):
        pp.Batch(i32(0, 2, 3), i32(5), torch.zeros((1, 2), dtype=torch.int32), 2)
    with pytest.raises(pp.PPError):
        pp.Batch(torch.tensor([0, 2]), i32(5), torch.zeros((1, 2), dtype=torch.int32), 2)
    with pytest.raises(pp.PPError):
        pp.Rotation(torch.zeros(4, dtype=torch.float64))


# ------------------------------------------------------------------ frequencies
R, BASE = 64, 10000.0


def plain():
    return [BASE ** (-2.0 * i / R) for i in range(R // 2)]


def test_frequencies_plain_linear_ntk(lib):
    f, s = pp.pp_rope_frequencies("none", R, BASE)
    assert s == 1.0 and np.array_equal(f, np.array(plain(), np.float32))
    f, s = pp.pp_rope_frequencies("linear", R, BASE, 8.0)
    assert s == 1.0 and np.array_equal(f, np.array([x / 8.0 for x in plain()], np.float32))
    f, s = pp.pp_rope_frequencies("ntk", R, BASE, 8.0)
    # the fastest pair keeps its frequency, the slowest is slowed by the factor
    assert f[0] == 1.0 and math.isclose(f[-1], plain()[-1] / 8.0, rel_tol=1e-6)
    want = [(BASE * 8.0 ** (R / (R - 2))) ** (-2.0 * i / R) for i in range(R // 2)]
    assert np.allclose(f, want, rtol=1e-7, atol=0)


def test_frequencies_banded(lib):
    low, high, n = 1.0, 4.0, 8192
    f, s = pp.pp_rope_frequencies("banded", R, BASE, 8.0, low, high, n)
    seen = set()
    for got, x in zip(f, plain()):
        wave = 2 * math.pi / x
        if wave < n / high:
            want, kind = x, 0
        elif wave > n / low:
            want, kind = x / 8.0, 1
        else:
            w = (n / wave - low) / (high - low)
            want, kind = (1 - w) * x / 8.0 + w * x, 2
        seen.add(kind)
        assert math.isclose(got, want, rel_tol=1e-6)
    assert seen == {0, 1, 2} and s == 1.0


def test_frequencies_yarn(lib):
    slow, fast, n, factor = 1.0, 32.0, 4096, 16.0
    f, s = pp.pp_rope_frequencies("yarn", R, BASE, factor, slow, fast, n)
    assert math.isclose(s, 0.1 * math.log(factor) + 1.0, rel_tol=1e-6)
    pair = lambda turns: R * math.log(n / (turns * 2 * math.pi)) / (2 * math.log(BASE))
    lo, hi = max(math.floor(pair(fast)), 0), min(math.ceil(pair(slow)), R - 1)
    assert 0 < lo < hi < R // 2
    for i, (got, x) in enumerate(zip(f, plain())):
        ramp = min(max((i - lo) / (hi - lo), 0.0), 1.0)
        assert math.isclose(got, x * (1 - ramp) + x / factor * ramp, rel_tol=1e-6)
    assert pp.pp_rope_frequencies("yarn", R, BASE, 1.0, slow, fast, n)[1] == 1.0


def test_frequencies_refusals(lib):
    for args, want in [(("none", 6), pp.PP_ERR_SHAPE), (("none", 0), pp.PP_ERR_SHAPE), (("none", 260), pp.PP_ERR_SHAPE),
                       ((9, 64), pp.PP_ERR_INVALID_ARG), (("none", 64, 0.0), pp.PP_ERR_INVALID_ARG),
                       (("none", 64, float("nan")), pp.PP_ERR_INVALID_ARG),
                       (("linear", 64, 1e4, 0.0), pp.PP_ERR_INVALID_ARG),
                       (("banded", 64, 1e4, 8.0, 4.0, 1.0, 8192), pp.PP_ERR_INVALID_ARG),
                       (("yarn", 64, 1e4, 8.0, 1.0, 32.0, 0), pp.PP_ERR_INVALID_ARG),
                       (("yarn", 64, 1.0, 8.0, 1.0, 32.0, 4096), pp.PP_ERR_INVALID_ARG)]:
        with pytest.raises(pp.PPError) as e:
            pp.pp_rope_frequencies(*args)
        assert e.value.status == want, args
