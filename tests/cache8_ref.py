"""Restatement (numpy) of the cache in 8 bits: codes, scales, append, commit."""
import numpy as np

LEAST = -60


def e4m3_values():
    """fp64 value of each byte: sign, 4 bits of exponent (bias 7), 3 of fraction; exponent and fraction all ones: NaN."""
    v = np.zeros(256)
    for c in range(256):
        e, f = c >> 3 & 15, c & 7
        m = (1 + f / 8) * 2.0 ** (e - 7) if e else f * 2.0 ** -9
        v[c] = np.nan if c & 127 == 127 else (-m if c & 128 else m)
    return v


VALUES = e4m3_values()


def codes_of(x):
    """Bytes of x (magnitudes up to 448) to nearest, ties to the even code; not finite: 0x7f."""
    x = np.asarray(x, np.float64)
    fin = np.isfinite(x)
    a = np.abs(np.where(fin, x, 0.0))
    assert (a <= 448).all()
    e = np.maximum(np.floor(np.log2(np.maximum(a, 1e-300))), -6)
    step = 2.0 ** (e - 3)
    m = np.rint(a / step) * step
    pos = np.searchsorted(VALUES[:127], m)  # the codes 0..126 ascend
    assert (VALUES[pos] == m).all()
    return np.where(fin, pos + 128 * np.signbit(x), 0x7f).astype(np.uint8)


def scale_for(amax):
    """The smallest power of two s >= 2^-60 with 448 s >= amax."""
    amax = np.asarray(amax, np.float64)
    s = np.full(amax.shape, 2.0 ** LEAST)
    while (448 * s < amax).any():
        s = np.where(448 * s < amax, 2 * s, s)
    return s


def largest(x, axis):
    return np.where(np.isfinite(x), np.abs(x), 0.0).max(axis, initial=0.0)


class Cache:
    """Codes [n_pages, page, H, D] and scales [n_pages, H, page / block] of keys or values."""

    def __init__(self, code, scale, block):
        self.code, self.scale, self.block, self.page = code, scale, block, code.shape[1]

    def at(self, table, e):
        p = table[e // self.page]
        return p, e % self.page, e % self.page // self.block

    def entry(self, table, e):
        p, o, i = self.at(table, e)
        return VALUES[self.code[p, o]] * self.scale[p, :, i][:, None].astype(np.float64)

    def values(self):
        return VALUES[self.code] * np.repeat(self.scale, self.block, 2).transpose(0, 2, 1)[..., None].astype(np.float64)

    def fill(self, table, ctx, entries, x, stay=()):
        """Entries (ascending) become x [n, H, D]; those before ctx, and those in `stay`, stay."""
        i = 0
        while i < len(entries):
            lo = entries[i] - entries[i] % self.block
            k = i
            while k < len(entries) and entries[k] < lo + self.block:
                k += 1
            kept = list(range(lo, min(ctx, lo + self.block))) + [e for e in stay if lo <= e < lo + self.block]
            self._fill_block(table, lo, kept, entries[i:k], x[i:k])
            i = k

    def _fill_block(self, table, lo, kept, entries, x):
        p, o, i = self.at(table, lo)
        amax = largest(x, (0, 2))
        now = scale_for(amax)
        if kept:
            old = self.scale[p, :, i].astype(np.float64)
            grow = amax > 448 * old
            now = np.where(grow, now, old)
            for e in kept:
                v = VALUES[self.code[p, o + e - lo]] * (old / now)[:, None]
                self.code[p, o + e - lo][grow] = codes_of(v)[grow]
        self.scale[p, :, i] = now
        for e, row in zip(entries, x):
            self.code[p, o + e - lo] = codes_of(row / now[:, None])

    def append(self, table, ctx, x):
        self.fill(table, ctx, list(range(ctx, ctx + len(x))), x)

    def commit(self, table, ctx, path):
        moved = [(j, p) for j, p in enumerate(path) if p != j]
        rows = [self.entry(table, ctx + p) for _, p in moved]
        self.fill(table, ctx, [ctx + j for j, _ in moved], np.array(rows).reshape(len(rows), *self.code.shape[2:]),
                  [ctx + j for j, p in enumerate(path) if p == j])


def quantised(x, block):
    """A cache of pages that hold x [n_pages, page, H, D] (whole blocks at a time)."""
    n, page, H, D = x.shape
    s = scale_for(largest(x.reshape(n, page // block, block, H, D), (2, 4)))  # [n, blocks, H]
    c = codes_of(x / np.repeat(s, block, 1)[..., None])
    return Cache(c, np.ascontiguousarray(s.transpose(0, 2, 1)).astype(np.float32), block)
