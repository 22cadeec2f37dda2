"""fp64 restatement (numpy) of the head norms with rotation, their gradients, and error bounds."""
import numpy as np

import attn_ref as ref

EPS32 = 2.0 ** -24


def forward(x, gamma, eps, pos, freq, layout, scale):
    x = np.asarray(x, np.float64)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1.0 if gamma is None else np.asarray(gamma, np.float64))
    return y if freq is None else ref.rotate(y, pos, freq, layout, scale)


def backward(x, gamma, eps, pos, freq, layout, scale, dy):
    """(dx, dgamma) from dy: dx = r (u - x r^2 mean(u x)), u = g gamma, g = dy rotated back."""
    x = np.asarray(x, np.float64)
    g = np.asarray(dy, np.float64) if freq is None else ref.rotate(dy, pos, freq, layout, scale, inverse=True)
    gam = 1.0 if gamma is None else np.asarray(gamma, np.float64)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    u = g * gam
    return r * (u - x * r * r * (u * x).mean(-1, keepdims=True)), (g * x * r).sum((0, 1))


def _pair_sum(x, n, layout):
    """|a| + |b| of each rotated element's pair, zero elsewhere."""
    m = np.zeros_like(x)
    ia, ib = (np.arange(n), np.arange(n) + n) if layout == "half" else (2 * np.arange(n), 2 * np.arange(n) + 1)
    m[..., ia] = m[..., ib] = np.abs(x[..., ia]) + np.abs(x[..., ib])
    return m


def forward_bound(x, gamma, eps, freq, layout, scale, dtype, want):
    """Largest |error| of a correct kernel.  The sum of squares: a lane adds up to 16 products, the group 5 partial
    sums: 21 roundings, times 1 / D (rounded) plus eps: 2, half of these felt in the root; a reciprocal root good to 2
    ulp: 4; two products: 2; together 17.5 * 2^-24 < 1.1e-6 of the normed value w.  The rotation: 1e-6 of |a| + |b| (attn_ref) and w's own error, which
    1.1e-6 (|a| + |b|) covers.  Then one rounding to the type."""
    w = forward(x, gamma, eps, None, None, layout, 1.0)
    tol = 1.1e-6 * np.abs(w)
    if freq is not None:
        n = len(freq)
        tol[..., :2 * n] = 2.1e-6 * abs(scale) * _pair_sum(w, n, layout)[..., :2 * n]
    half = ref.BF16_HALF_ULP if dtype == "bf16" else EPS32
    return tol + half * (np.abs(want) + tol)


def backward_bound(x, gamma, eps, freq, layout, scale, dy, dtype, dx, per_thread):
    """Bounds of (dx, dgamma).  g is off by 1e-6 of its pair's |a| + |b| (e_g).  S = sum u x over the row: its terms'
    errors and 21 roundings of the absolute sum (e_s).  dx = r (u - x r^2 S / D): the terms' errors, r's 15.5 *
    2^-24 (three times in the second) and 6 roundings: 5e-6 of both terms covers these.  dgamma: each term g x r is off by
    e_g |x| r + 1e-6 |g x r|; sums of at most per_thread terms in a thread, then 64 groups, 20 parts and 32 rows of parts,
    as many roundings of the absolute sum."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    D = x.shape[-1]
    gam = np.ones(D) if gamma is None else np.abs(np.asarray(gamma, np.float64))
    g = np.abs(dy)
    e_g = np.zeros_like(g)
    if freq is not None:
        n = len(freq)
        pair = abs(scale) * _pair_sum(dy, n, layout)
        g[..., :2 * n] = pair[..., :2 * n]  # at least |g|
        e_g = 1e-6 * pair
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    u, e_u = g * gam, e_g * gam + EPS32 * g * gam
    s = (u * np.abs(x)).sum(-1, keepdims=True)
    e_s = (e_u * np.abs(x)).sum(-1, keepdims=True) + 21 * EPS32 * s
    tol = r * (e_u + np.abs(x) * r * r / D * e_s) + 5e-6 * r * (u + np.abs(x) * r * r / D * s)
    half = ref.BF16_HALF_ULP if dtype == "bf16" else EPS32
    t = g * np.abs(x) * r
    tol_gamma = (e_g * np.abs(x) * r + 1e-6 * t + (per_thread + 116) * EPS32 * t).sum((0, 1))
    return tol + half * (np.abs(dx) + tol), tol_gamma
