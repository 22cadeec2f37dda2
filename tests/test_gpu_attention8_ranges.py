"""GPU tests of attention over the 8-bit cache where weights, scales and queries span wide ranges: what holds little of a
row's weight, or lies in blocks of small scales, may be all that an element's result consists of.

The bound is that of attn_ref.attend.  Where the weights are multiplied as e4m3 numbers (few rows, bf16), a weight times
its block's value scale may besides be off by 2^-41 of the largest such product of its row: `floor` below, the sum of that
over the row's keys times their codes' magnitudes."""
import numpy as np
import pytest

import attn_ref
import cache8_ref as ref
from test_gpu_attention8 import Case8

pytestmark = pytest.mark.gpu


def floor(c):
    """[T, heads, dim]: sum over the visible keys j of 2^-41 max_i(p_i vs_i) |code_j|."""
    out = np.zeros((c.T, c.heads, c.q.shape[2]))
    g = c.heads // c.k.shape[2]
    code, scale = np.abs(ref.VALUES[c.held[1].code]), c.held[1].scale.astype(np.float64)
    for b in range(len(c.ctx)):
        q0, n, ctx = int(c.starts[b]), int(c.starts[b + 1] - c.starts[b]), int(c.ctx[b])
        j = np.arange(ctx + n)
        page, off = c.pages[b][j // c.page], j % c.page
        see = attn_ref.visible(n, ctx, c.mask, q0)
        for h in range(c.heads):
            k, vs, vc = c.k[page, off, h // g].astype(np.float64), scale[page, h // g, off // c.block], code[page, off, h // g]
            for i in range(n):
                s = c.scale * (k[see[i]] @ c.q[q0 + i, h].astype(np.float64))
                p = np.exp(s - s.max())
                p /= p.sum()
                out[q0 + i, h] = 2.0 ** -41 * (p * vs[see[i]]).max() * vc[see[i]].sum(0)
    return out


def check(c, pp, extra=0.0):
    want, tol = c.want()
    tol = tol + extra
    if c.dtype == "bf16":
        tol = tol + floor(c)
    got, status, _ = c.run(pp)
    assert status == pp.PP_OK
    off = np.abs(got - want) - tol
    assert off.max() <= 0, (float(off.max()), np.unravel_index(off.argmax(), off.shape), float((np.abs(got - want) / tol).max()))


def put(c, which, b, entries, x):
    """Entries of sequence b become x [n, kv, dim] (before the blocks are quantised again)."""
    x0 = (c.raw_k, c.raw_v)[which]
    e = np.asarray(entries)
    x0[c.pages[b, e // c.page], e % c.page] = x


class Raw(Case8):
    """Case8 whose entries can be changed before they are held in codes."""

    def __init__(self, *a, **kw):
        super().__init__(*a, **kw)
        self.raw_k, self.raw_v = self.k.copy(), self.v.copy()

    def hold(self):
        for i, x in enumerate((self.raw_k, self.raw_v)):
            self.held[i] = ref.quantised(np.where(np.isfinite(x), x, 0.0), self.block)
        self.refresh()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ahead", [8.0, 14.0, 20.0, 26.0])
@pytest.mark.parametrize("n,heads,kv,dim", [(1, 8, 2, 128), (1, 16, 2, 64), (1, 4, 1, 256), (2, 16, 2, 128), (20, 4, 2, 64)])
def test_one_key_of_small_value_takes_most(pp, dtype, ahead, n, heads, kv, dim):
    """The first key's score lies `ahead` of the others' and its values are 2^-12 of theirs, as the first token's are in
    many heads: the result is what the others' small weights make of their values."""
    ctx = 4096 if n < 20 else 700
    c = Raw([(n, ctx), (n, 300)], heads, kv, dim, 32, 16, dtype, seed=int(ahead) + n)
    rng = np.random.default_rng(1)
    u = rng.standard_normal((kv, dim))
    u /= np.linalg.norm(u, axis=1, keepdims=True)
    for b, (new, old) in enumerate([(n, ctx), (n, 300)]):
        e = np.arange(new + old)
        k = 0.1 * rng.standard_normal((new + old, kv, dim))
        k[0] = 8.0 * u
        v = rng.standard_normal((new + old, kv, dim)) + 1.0
        v[0] *= 2.0 ** -12
        put(c, 0, b, e, k)
        put(c, 1, b, e, v)
    grown = np.repeat(u, heads // kv, 0)[None] * (ahead / (8.0 * c.scale)) + 0.1 * rng.standard_normal((c.T, heads, dim))
    from test_gpu_attention import rounded
    c.q = rounded(grown, dtype)
    c.hold()
    check(c, pp)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ratio", [8, 14, 20, 26])
@pytest.mark.parametrize("n,heads,kv,dim,page,block", [(1, 8, 2, 128, 32, 16), (1, 8, 2, 128, 64, 64), (1, 4, 1, 256, 16, 16),
                                                       (2, 16, 2, 64, 128, 128), (30, 4, 2, 64, 32, 16)])
def test_blocks_of_large_scale_hold_one_channel(pp, dtype, ratio, n, heads, kv, dim, page, block):
    """Every third block has values of about 2^ratio in one channel and zeros elsewhere; the other blocks fill the others."""
    seqs = [(n, 1500), (n, 333)]
    c = Raw(seqs, heads, kv, dim, page, block, dtype, seed=ratio + n)
    rng = np.random.default_rng(2)
    for b, (new, old) in enumerate(seqs):
        e = np.arange(new + old)
        v = rng.standard_normal((new + old, kv, dim)) + 0.5
        v[:, :, 5] = 0
        big = e // block % 3 == 1
        v[big] = 0
        v[big, :, 5] = 2.0 ** ratio * rng.uniform(0.5, 1.0, (int(big.sum()), kv))
        put(c, 1, b, e, v)
    c.hold()
    check(c, pp)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("by", [-110, -60, 60, 100])
@pytest.mark.parametrize("n", [1, 30])
def test_value_scales_of_any_size(pp, dtype, by, n):
    """A cache filled elsewhere: all value scales 2^by of what they would be; some blocks another 2^10 smaller."""
    c = Case8([(n, 700), (n, 40)], 8, 2, 128, 32, 16, dtype, seed=n, stale=0.0)
    v = c.held[1]
    rng = np.random.default_rng(4)
    v.scale *= (2.0 ** (by - 10.0 * rng.integers(0, 2, v.scale.shape))).astype(np.float32)
    c.refresh()
    check(c, pp)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("top", [12, 20])
@pytest.mark.parametrize("n,heads,kv,dim", [(1, 8, 2, 128), (2, 16, 2, 64), (1, 4, 1, 256), (30, 4, 2, 64)])
def test_queries_with_one_large_element(pp, dtype, top, n, heads, kv, dim):
    """One element of a query head is 2^top, where the keys are zero; the scores come from the small ones."""
    seqs = [(n, 500), (n, 60)]
    c = Raw(seqs, heads, kv, dim, 16, 16, dtype, seed=top)
    for b, (new, old) in enumerate(seqs):
        e = np.arange(new + old)
        k = c.raw_k[c.pages[b, e // 16], e % 16]
        k[:, :, 3] = 0
        put(c, 0, b, e, k)
    c.q[:, :, 3] = 2.0 ** top
    c.hold()
    extra = np.zeros((c.T, heads, dim))
    if dtype == "bf16":
        # few rows: a query element below 2^-14 of its head's largest is held to 2^-21 of that, which moves a score by up to
        # ds = scale sum |k| dq and a weight by a factor within exp(2 ds)
        dq = np.where(np.abs(c.q) < 2.0 ** (top - 14), 2.0 ** (top - 21), 0.0)
        for b, (new, old) in enumerate(seqs):
            k, v = (np.abs(attn_ref.gather(x, c.pages[b], old + new)) for x in (c.k, c.v))
            for i in range(int(c.starts[b]), int(c.starts[b]) + new):
                for h in range(heads):
                    g = h * kv // heads
                    extra[i, h] = np.expm1(2 * c.scale * (k[:, g] @ dq[i, h]).max()) * v[:, g].max(0)
    check(c, pp, extra)
