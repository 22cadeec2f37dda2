"""fp64 restatement (numpy) of the attention-side operators, and error bounds.

Written from the definitions, one token and one head at a time where that is
affordable; used by the GPU tests of rotary positions, the paged cache and
tree attention.
"""
import numpy as np

BF16_HALF_ULP = 2.0 ** -8     # relative rounding of fp32 -> bf16 (8 significant bits)
F32_HALF_ULP = 2.0 ** -24


def rotate(x, pos, freq, layout, scale=1.0, inverse=False):
    """x [T, H, D] (any float type) rotated in fp64."""
    x = np.asarray(x, np.float64)
    y = x.copy()
    n = len(freq)
    ang = np.asarray(pos, np.float64)[:, None] * np.asarray(freq, np.float64)[None, :]
    c, s = (scale * np.cos(ang))[:, None, :], (scale * np.sin(ang))[:, None, :]
    if inverse:
        s = -s
    ia, ib = (np.arange(n), np.arange(n) + n) if layout == "half" else (2 * np.arange(n), 2 * np.arange(n) + 1)
    y[..., ia] = x[..., ia] * c - x[..., ib] * s
    y[..., ib] = x[..., ib] * c + x[..., ia] * s
    return y


def rotate_bound(x, freq, layout, scale, dtype, ref):
    """Largest |error| of a correct kernel.  The angle, reduced to turns in [-1/2, 1/2], takes up to three fp32
    roundings of at most 2^-25 turns; sine and cosine are good to 2 ulp, the products and the sum to 3 half ulps:
    together below 1e-6 of |a| + |b|.  Then one rounding to the type.  Elements past the rotated ones are copies."""
    n = len(freq)
    x = np.abs(np.asarray(x, np.float64))
    m = np.zeros_like(x)
    ia, ib = (np.arange(n), np.arange(n) + n) if layout == "half" else (2 * np.arange(n), 2 * np.arange(n) + 1)
    m[..., ia] = m[..., ib] = x[..., ia] + x[..., ib]
    tol = 1e-6 * abs(scale) * m
    tol[..., :2 * n] += (BF16_HALF_ULP if dtype == "bf16" else F32_HALF_ULP) * (np.abs(ref[..., :2 * n]) + tol[..., :2 * n])
    return tol


def gather(cache, pages, n):
    """Entries 0..n-1 of a sequence: cache [n_pages, page, H, D], pages [max_pages]."""
    page = cache.shape[1]
    j = np.arange(n)
    return cache[pages[j // page], j % page]


def visible(n, ctx, mask, q0):
    """[n, ctx + n] truth values; mask None (chain) or uint32 [T, words]."""
    see = np.zeros((n, ctx + n), bool)
    see[:, :ctx] = True
    for i in range(n):
        for j in range(n):
            if mask is None:
                see[i, ctx + j] = j <= i
            else:
                see[i, ctx + j] = j < 32 * mask.shape[1] and bool(int(mask[q0 + i, j // 32]) >> (j % 32) & 1)
    return see


def attend(q, k_cache, v_cache, starts, ctx, pages, mask, scale, dtype):
    """(out, bound) in fp64 for q [T, Hq, D]; caches [n_pages, page, Hkv, D].  Unseen entries never enter a sum.

    The bound on |out_gpu - out|, per element, with A = sum_j p_j |v_j|:
      scores: D + 4 fp32 roundings of the products' absolute sum, and the rounding of scale * log2(e) and of the
      exponent's argument, together eps_s; a weight is then off by a factor exp(2 eps_s), plus 2^-21 for exp2;
      sums of N terms in fp32: N / 32 + 32 roundings (tiles are summed apart);
      bf16 only: weights rounded to bf16 in numerator and denominator, 2 * 2^-8; the output's rounding, 2^-8 |out|.
    """
    T, Hq, D = q.shape
    Hkv = k_cache.shape[2]
    g = Hq // Hkv
    out = np.zeros((T, Hq, D))
    tol = np.zeros((T, Hq, D))
    q = np.asarray(q, np.float64)
    for b in range(len(ctx)):
        q0, n, c = int(starts[b]), int(starts[b + 1] - starts[b]), int(ctx[b])
        if n == 0:
            continue
        k = np.asarray(gather(k_cache, pages[b], c + n), np.float64)
        v = np.asarray(gather(v_cache, pages[b], c + n), np.float64)
        see = visible(n, c, mask, q0)
        for h in range(Hq):
            kh, vh = k[:, h // g], v[:, h // g]
            for i in range(n):
                j = np.nonzero(see[i])[0]
                if len(j) == 0:
                    continue
                s = scale * (kh[j] @ q[q0 + i, h])
                p = np.exp(s - s.max())
                p /= p.sum()
                o = p @ vh[j]
                a = p @ np.abs(vh[j])
                eps_s = F32_HALF_ULP * ((D + 4) * scale * (np.abs(kh[j]) @ np.abs(q[q0 + i, h])).max()
                                        + 4 * np.abs(s).max())
                rel = 2 * np.expm1(2 * eps_s) + 2.0 ** -20 + 2 * F32_HALF_ULP * (len(j) / 32 + 32)
                if dtype == "bf16":
                    rel += 2 * BF16_HALF_ULP
                out[q0 + i, h] = o
                t = rel * a
                tol[q0 + i, h] = t + (BF16_HALF_ULP if dtype == "bf16" else F32_HALF_ULP) * (np.abs(o) + t)
    return out, tol


def tree_mask(parents_by_seq, words):
    """uint32 [T, words]: each node sees its ancestors and itself."""
    rows, depth = [], []
    for parents in parents_by_seq:
        vis, dep = [], []
        for i, p in enumerate(parents):
            vis.append((vis[p] if p >= 0 else 0) | 1 << i)
            dep.append(dep[p] + 1 if p >= 0 else 0)
        rows += [[(x >> (32 * w)) & 0xffffffff for w in range(words)] for x in vis]
        depth += dep
    return np.array(rows, np.uint32).reshape(-1, words), np.array(depth, np.int32)
