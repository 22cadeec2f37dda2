"""Cases of the serving operators that hold the key/value cache in 8 bits, and of the norms of query and key heads.

Five operators, as one decode step over an 8-bit cache uses them:

* norm:    every head of the queries and keys divided by its root mean square, times a weight, then rotated by its
           token's position; and the gradients of that;
* append:  queries (normed and) rotated, keys (normed and) rotated and values written in 8 bits into the pages of their
           sequences, with a scale for each block of tokens and key head;
* read:    entries of the cache back as numbers;
* attend:  attention of each sequence's new tokens (one token, a tree of drafted tokens, or a prompt) over its entries;
* commit:  the accepted path of a drafted tree moved together behind the cached tokens, in every layer.

An entry's value is code * scale, the code an e4m3 number.  A scale is a power of two, the smallest one with
448 * scale >= the largest magnitude of its block and head.  A block that already holds cached entries keeps its scale
until a new entry needs a larger one; the cached codes are then rounded again at the new scale.

`run` computes them with elementary torch operations in fp32 (`own` false) or through the package's binding (`own`
true).  `exact` restates the definitions in fp64.  Head shapes are those of the package's model shapes (32 query
heads of 128 with 32 or 8 key heads, 40 of 128, 16 of 64); sequence lengths follow a fixed spread, so that a
case's work does not depend on the seed.
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ESZ = {"bf16": 2, "f32": 4}
EPS = 1e-6
CODE = torch.float8_e4m3fn
LEAST_EXPONENT = -60


# --------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one decode step's queries and keys of a batch of 8
        dict(name="norm_decode_8", op="norm", dtype="bf16", tokens=8, heads=32, kv_heads=8, dim=128, rot=128,
             layout="half", grad=False, max_pos=8192),
        # a prompt of odd length on a small fp32 model, a quarter of the head rotated
        dict(name="norm_prompt_f32", op="norm", dtype="f32", tokens=2047, heads=16, kv_heads=16, dim=64, rot=16,
             layout="interleaved", grad=False, max_pos=2047),
        # gradients over 4 prompts of 2048 tokens
        dict(name="norm_grad_8192", op="norm", dtype="bf16", tokens=8192, heads=32, kv_heads=8, dim=128, rot=128,
             layout="half", grad=True, max_pos=2048),
        # one token for each of 64 sequences, most of them into a block that holds cached ones
        dict(name="append_decode_64", op="append", dtype="bf16", seqs=64, new_lo=1, new_hi=1, ctx_lo=64, ctx_hi=1024,
             heads=32, kv_heads=8, dim=128, rot=128, layout="half", norm=False, page=64, block=16, tree=False),
        # 4 prompts, ragged, up to 2048 tokens, heads normed on the way, a scale a page
        dict(name="append_prompt_8k", op="append", dtype="bf16", seqs=4, new_lo=1900, new_hi=2048, ctx_lo=0, ctx_hi=0,
             heads=40, kv_heads=40, dim=128, rot=128, layout="half", norm=True, page=64, block=64, tree=False),
        # whole short sequences of a small fp32 model
        dict(name="read_f32_3", op="read", dtype="f32", seqs=3, new_lo=100, new_hi=713, ctx_lo=0, ctx_hi=0, heads=16,
             kv_heads=16, dim=64, page=16, block=16, tree=False),
        # the last few thousand tokens of 64 sequences
        dict(name="read_64", op="read", dtype="bf16", seqs=64, new_lo=500, new_hi=3500, ctx_lo=0, ctx_hi=1000, heads=32,
             kv_heads=8, dim=128, page=64, block=32, tree=False),
        # a drafted tree on a small fp32 model
        dict(name="attend_tree_f32", op="attend", dtype="f32", seqs=3, new_lo=9, new_hi=13, ctx_lo=100, ctx_hi=1000,
             heads=16, kv_heads=16, dim=64, page=16, block=16, tree=True),
        # batched decode over ragged contexts, shared key heads
        dict(name="attend_decode_64", op="attend", dtype="bf16", seqs=64, new_lo=1, new_hi=1, ctx_lo=64, ctx_hi=8191,
             heads=32, kv_heads=8, dim=128, page=64, block=16, tree=False),
        # drafted trees of up to 48 tokens over ragged contexts, small pages
        dict(name="attend_tree_8", op="attend", dtype="bf16", seqs=8, new_lo=17, new_hi=48, ctx_lo=500, ctx_hi=6001,
             heads=32, kv_heads=8, dim=128, page=16, block=16, tree=True),
        # one sequence's accepted path, one layer
        dict(name="commit_1", op="commit", dtype="bf16", seqs=1, layers=1, draft=40, accept=5, ctx_lo=300, ctx_hi=300,
             kv_heads=8, dim=128, page=16, block=16),
        # the accepted paths of 32 sequences in 32 layers
        dict(name="commit_32x32", op="commit", dtype="bf16", seqs=32, layers=32, draft=48, accept=8, ctx_lo=20,
             ctx_hi=300, kv_heads=8, dim=128, page=64, block=16),
    ]


def _log_int(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm (lo = 0 allowed)."""
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo + 1), math.log(hi + 2)))) - 1))


def _draw_once(rng):
    op = rng.choice(["norm", "append", "read", "attend", "attend", "attend", "commit"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    heads, kv_heads, dim = rng.choice([(32, 32, 128), (32, 8, 128), (40, 40, 128), (16, 16, 64), (32, 4, 128),
                                       (12, 3, 80)])
    block = rng.choice([16, 16, 32, 64, 128])
    page = block * rng.choice([1, 1, 2, 3, 4])
    rot = rng.choice([dim, dim, dim // 2, dim // 4])
    layout = rng.choice(["half", "interleaved"])
    if op == "norm":
        return dict(op=op, dtype=dtype, tokens=_log_int(rng, 1, 8192), heads=heads, kv_heads=kv_heads, dim=dim, rot=rot,
                    layout=layout, grad=rng.random() < 0.5, max_pos=_log_int(rng, 64, 8192))
    if op == "commit":
        accept = rng.randint(1, 8)
        lo = _log_int(rng, 0, 300)
        return dict(op=op, dtype=dtype, seqs=_log_int(rng, 1, 32), layers=_log_int(rng, 1, 32),
                    draft=rng.randint(2 * accept + block, 2 * accept + block + 48), accept=accept, ctx_lo=lo,
                    ctx_hi=lo + _log_int(rng, 0, 300), kv_heads=kv_heads, dim=dim, page=page, block=block)
    kind = "read" if op == "read" else rng.choice(["decode", "tree", "prompt"])
    seqs = _log_int(rng, 1, 64)
    if kind == "decode":
        lo = hi = 1
    elif kind == "tree":
        lo = rng.randint(2, 64)
        hi = min(64, lo + rng.randint(0, 24))
    else:
        seqs = seqs if kind == "read" else min(seqs, 8)
        lo = _log_int(rng, 2, 2048)
        hi = min(4096, lo + _log_int(rng, 0, 512))
    ctx_lo = _log_int(rng, 0, 8000)
    ctx_hi = min(8191, ctx_lo + _log_int(rng, 0, 4000))
    case = dict(op=op, dtype=dtype, seqs=seqs, new_lo=lo, new_hi=hi, ctx_lo=ctx_lo, ctx_hi=ctx_hi, heads=heads,
                kv_heads=kv_heads, dim=dim, page=page, block=block, tree=kind == "tree")
    if op == "append":
        case.update(rot=rot, layout=layout, norm=rng.random() < 0.5)
    return case


def _cost(case):
    w = work(case)
    rate = 2e12 if case["op"] != "attend" or case["dtype"] == "f32" else 200e12
    return w["bytes"] / 6.7e12 + w["flops"] / rate


def draw(rng):
    limit = {}
    for c in listed():
        limit[c["op"]] = max(limit.get(c["op"], 0.0), _cost(c))
    while True:
        case = _draw_once(rng)
        if _cost(case) <= limit[case["op"]] and _pool(case) <= 2 << 30:
            return case


# --------------------------------------------------------------------------- shapes that do not depend on the seed

def _spread(lo, hi, n, phase):
    """n whole numbers from lo to hi in a fixed irregular order."""
    return [lo + int((hi - lo + 1) * ((0.6180339887498949 * (i + phase)) % 1.0)) for i in range(n)]


def _lengths(case):
    new = [case["draft"]] * case["seqs"] if case["op"] == "commit" else \
        _spread(case["new_lo"], case["new_hi"], case["seqs"], 0.25)
    return new, _spread(case["ctx_lo"], case["ctx_hi"], case["seqs"], 0.5)


def _pool(case):
    """Bytes of a case's key and value codes."""
    if case["op"] == "norm":
        return 0
    new, ctx = _lengths(case)
    pages = sum(-(-(n + c) // case["page"]) for n, c in zip(new, ctx)) + 2
    return pages * case["page"] * case["kv_heads"] * case["dim"] * 2 * case.get("layers", 1)


def _tree(n, salt):
    """Parents of n drafted tokens (-1: the last cached token), each before its children."""
    rng = random.Random(1000 * n + salt)
    return [rng.randint(max(-1, i - 9), i - 1) for i in range(n)]


def _tree_of(parents):
    """(visible sets as whole numbers, depths) of drafted tokens."""
    vis, depth = [], []
    for i, p in enumerate(parents):
        vis.append((vis[p] if p >= 0 else 0) | 1 << i)
        depth.append(depth[p] + 1 if p >= 0 else 0)
    return vis, depth


def _frequencies(rot):
    """Radians per position of each rotated pair."""
    return [10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)]


def work(case):
    e = ESZ[case["dtype"]]
    if case["op"] == "norm":
        elems = case["tokens"] * (case["heads"] + case["kv_heads"]) * case["dim"]
        small = 4 * case["tokens"] + case["dim"] * 2 * (e + (4 if case["grad"] else 0))
        return {"bytes": (3 if case["grad"] else 2) * elems * e + small, "flops": (12 if case["grad"] else 6) * elems}
    new, ctx = _lengths(case)
    n, block, kv = sum(new), case["block"], case["kv_heads"] * case["dim"]
    scales = 8 * case["kv_heads"]  # of one block
    if case["op"] == "commit":
        blocks = [(c + case["accept"] - 1) // block - c // block + 1 for c in ctx]
        return {"bytes": case["layers"] * (case["seqs"] * case["accept"] * (4 * kv + scales) + sum(blocks) * scales) +
                case["seqs"] * (4 * case["accept"] + 12), "flops": 4 * case["layers"] * case["seqs"] * case["accept"] * kv}
    table = sum(-(-(a + c) // case["page"]) for a, c in zip(new, ctx))
    blocks = sum((a + c - 1) // block - c // block + 1 for a, c in zip(new, ctx))
    if case["op"] == "read":
        return {"bytes": n * kv * 2 * (1 + e) + blocks * scales + 4 * table + 8 * case["seqs"], "flops": 2 * n * kv}
    q_row = case["heads"] * case["dim"] * e
    if case["op"] == "append":
        old = sum(1 for c in ctx if c % block)  # blocks whose scale is read first
        return {"bytes": n * (2 * q_row + kv * 2 * (1 + e) + 4) + (blocks + old) * scales + 8 * case["seqs"],
                "flops": n * (case["heads"] + 2 * case["kv_heads"]) * case["dim"] * (8 if case["norm"] else 4)}
    pairs = 0
    for b, (a, c) in enumerate(zip(new, ctx)):
        seen = sum(d + 1 for d in _tree_of(_tree(a, b))[1]) if case["tree"] else a * (a + 1) // 2
        pairs += a * c + seen
    words = -(-max(new) // 32) if case["tree"] else 0
    held = sum(-(-(a + c) // block) for a, c in zip(new, ctx))
    return {"bytes": n * (2 * q_row + 4 * words) + sum(a + c for a, c in zip(new, ctx)) * 2 * kv + held * scales +
            4 * table + 8 * case["seqs"], "flops": 4 * pairs * case["heads"] * case["dim"]}


# -------------------------------------------------------------------------------------------------- inputs

def _power(amax):
    """The scale of a block whose largest magnitude is amax (fp32)."""
    m, x = torch.frexp(amax)
    e = torch.where(amax > 0, x - 9 + (m > 0.875).int(), LEAST_EXPONENT).clamp(min=LEAST_EXPONENT)
    return ((e + 127) << 23).int().view(torch.float32)


def _held(x, block):
    """Codes (as bytes) and scales [..., n_pages, heads, blocks] of pages x [..., n_pages, page, heads, dim]."""
    y = x.unflatten(-3, (-1, block))                                  # [..., n_pages, blocks, block, heads, dim]
    s = _power(y.abs().amax((-3, -1)))                                # [..., n_pages, blocks, heads]
    code = (y / s[..., None, :, None]).to(CODE).flatten(-4, -3)
    return code.view(torch.uint8), s.transpose(-1, -2).contiguous()


def _inputs(case, seed):
    """Tensors of one call, from the seed alone."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 29)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * std).to(dt)

    def weight(n):
        return (1.0 + 0.2 * torch.randn((n,), generator=g, device=DEV, dtype=torch.float32)).to(dt)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=DEV)

    s = {"case": case, "dt": dt}
    if "rot" in case:
        s["freq"] = torch.tensor(_frequencies(case["rot"]), dtype=torch.float32, device=DEV)
    if case.get("norm") or case["op"] == "norm":
        s["q_gamma"], s["k_gamma"] = weight(case["dim"]), weight(case["dim"])
    if case["op"] == "norm":
        T, D = case["tokens"], case["dim"]
        s["q"], s["k"] = normal(T, case["heads"], D, std=1.7), normal(T, case["kv_heads"], D, std=0.6)
        s["pos"] = torch.randint(0, case["max_pos"], (T,), generator=g, device=DEV, dtype=torch.int32)
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        if case["grad"]:
            s["q_grad"], s["k_grad"] = normal(T, case["heads"], D), normal(T, case["kv_heads"], D)
            s["dq_gamma"], s["dk_gamma"] = (torch.empty((D,), dtype=torch.float32, device=DEV) for _ in range(2))
        return s
    new, ctx = _lengths(case)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    T, page = starts[-1], case["page"]
    per = [-(-(a + c) // page) for a, c in zip(new, ctx)]
    n_pages = sum(per) + 2
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(new), max(per)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, k in enumerate(per):
        table[b, :k] = order[at:at + k]
        at += k
    s.update(q_start=ints(starts), ctx_len=ints(ctx), pages=table, new=new, ctx=ctx, starts=starts)
    shape = (n_pages, page, case["kv_heads"], case["dim"])
    if case["op"] == "commit":
        shape = (case["layers"],) + shape
    # keys have a few large channels, as trained models' do; tokens differ in size
    wide = 1.0 + 3.0 * (torch.arange(case["dim"], device=DEV) % 29 == 7).float()
    for name, chan in (("k", wide), ("v", torch.ones_like(wide))):
        x = torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * chan
        x *= torch.exp2(0.7 * torch.randn(shape[:-1], generator=g, device=DEV, dtype=torch.float32))[..., None]
        s[name + "_code"], s[name + "_scale"] = _held(x, case["block"])
        del x
    if case["op"] == "commit":
        # the first accepted token lies in a block past all that the path moves to, so that another pass on the same
        # state gives the same cache
        rng = random.Random(seed)
        acc = case["accept"]
        s["path"] = ints([sorted(rng.sample(range(acc + case["block"], case["draft"]), acc)) for _ in new])
        s["n_accept"] = ints([acc] * len(new))
        s["new_len"] = torch.empty_like(s["ctx_len"])
        return s
    if case["op"] == "read":
        s["k_out"], s["v_out"] = (torch.empty((T,) + shape[2:], dtype=dt, device=DEV) for _ in range(2))
        return s
    trees = [_tree_of(_tree(n, b)) for b, n in enumerate(new)] if case["tree"] else None
    depth = [trees[b][1][i] if trees else i for b, n in enumerate(new) for i in range(n)]
    first = [c for n, c in zip(new, ctx) for _ in range(n)]
    s["pos"] = ints([c + d for c, d in zip(first, depth)])
    s["q"] = normal(T, case["heads"], case["dim"])
    s["out"] = torch.empty_like(s["q"])
    if case["op"] == "append":
        s["k"] = (normal(T, case["kv_heads"], case["dim"]).float() * wide).to(dt)
        s["v"] = normal(T, case["kv_heads"], case["dim"])
        return s
    s["scale"] = case["dim"] ** -0.5
    s["mask"] = None
    if trees:
        words = -(-max(new) // 32)
        rows = [[(v >> (32 * w)) & 0xffffffff for w in range(words)] for vis, _ in trees for v in vis]
        s["mask"] = torch.tensor(rows, dtype=torch.int64, device=DEV).to(torch.int32)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2605_28283_gb300 import binding as pp
        s["pp"] = pp
        s["rot"] = pp.Rotation(s["freq"], case["layout"]) if "freq" in s else None
        s["norm"] = pp.HeadNorm(s["q_gamma"], s["k_gamma"], EPS) if "q_gamma" in s else None
        if case["op"] == "norm":
            s["ws"] = pp.alloc_head_norm_workspace(case["dim"]) if case["grad"] else None
            return s
        pick = (lambda x: x[0]) if case["op"] == "commit" else (lambda x: x)
        s["cache"] = pp.KVCache8(pick(s["k_code"]), pick(s["v_code"]), pick(s["k_scale"]), pick(s["v_scale"]),
                                 case.get("heads", case["kv_heads"]), s["dt"])
        s["batch"] = pp.Batch(s["q_start"], s["ctx_len"], s["pages"], s["starts"][-1])
        s["ws"] = pp.alloc_attn8_workspace(s["cache"])
    return s


# ---------------------------------------------------------------------------------------------- plain form, fp32

def _rotate(x, s, sign=1.0):
    """x [T, H, D] (fp32) with the first 2 * len(freq) elements of a head rotated; the angles in 64 bits."""
    f, layout = s["freq"], s["case"]["layout"]
    n = f.numel()
    angle = s["pos"].double()[:, None, None] * f.double()
    c, d = torch.cos(angle).float(), sign * torch.sin(angle).float()
    a, b = (x[..., :n], x[..., n:2 * n]) if layout == "half" else (x[..., 0:2 * n:2], x[..., 1:2 * n:2])
    ya, yb = a * c - b * d, b * c + a * d
    y = torch.cat([ya, yb], -1) if layout == "half" else torch.stack([ya, yb], -1).flatten(-2)
    return torch.cat([y, x[..., 2 * n:]], -1)


def _normed(x, gamma):
    return x * (1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)) * gamma


def _norm_grad(x, grad, gamma, s):
    x, g = x.float(), _rotate(grad.float(), s, -1.0)
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    u = g * gamma.float()
    dx = r * (u - x * (r * r * (u * x).mean(-1, keepdim=True)))
    return dx.to(grad.dtype), (g * x * r).sum((0, 1), dtype=torch.float64).float()


def _plain_norm(s):
    if not s["case"]["grad"]:
        return [_rotate(_normed(s[n].float(), s[n + "_gamma"].float()), s).to(s["dt"]) for n in ("q", "k")]
    dq, dq_gamma = _norm_grad(s["q"], s["q_grad"], s["q_gamma"], s)
    dk, dk_gamma = _norm_grad(s["k"], s["k_grad"], s["k_gamma"], s)
    return [dq, dk, dq_gamma, dk_gamma]


def _tokens(s):
    """(sequence, entry) of each new token."""
    t = torch.arange(s["starts"][-1], device=DEV)
    b = torch.searchsorted(s["q_start"][1:].long(), t, right=True)
    return b, s["ctx_len"].long()[b] + t - s["q_start"].long()[b]


def _place(s, b, entry):
    """(page, offset) of entries."""
    page = s["case"]["page"]
    return s["pages"].long()[b, entry // page], entry % page


def _stored(code, scale, page, off, block):
    """fp32 values of entries [..., heads, dim]; layers, where there are some, come first."""
    by = scale[..., page, :, off // block]
    return code.view(CODE)[..., page, off, :, :].float() * (by.movedim(-2, 0) if scale.dim() > 3 else by)[..., None]


def _write(s, name, x):
    """New tokens' values x [T, heads, dim] (fp32) into the codes and scales of `name`."""
    case, code, scale = s["case"], s[name + "_code"], s[name + "_scale"]
    block, H = case["block"], case["kv_heads"]
    b, entry = _tokens(s)
    page, off = _place(s, b, entry)
    # blocks numbered over all pages; what a block holds already counts where cached tokens lie in it
    blocks = case["page"] // block
    which = page * blocks + off // block
    need = torch.zeros((code.shape[0] * blocks, H), device=DEV)
    need.scatter_reduce_(0, which[:, None].expand(-1, H), x.abs().amax(-1), "amax")
    need = need[which]
    old = scale[page, :, off // block] * (entry - entry % block < s["ctx_len"].long()[b])[:, None]
    now = torch.where(need > 448.0 * old, _power(need), old)
    # cached entries of each sequence's first block, rounded again
    first = s["q_start"].long()[:-1]
    ctx = s["ctx_len"].long()
    at = (ctx - ctx % block)[:, None] + torch.arange(block, device=DEV)
    live = at < ctx[:, None]
    p, o = _place(s, torch.arange(ctx.numel(), device=DEV)[:, None], torch.minimum(at, ctx[:, None]))
    again = _stored(code, scale, p, o, block) / now[first][:, None, :, None]
    code[p[live], o[live]] = again[live].to(CODE).view(torch.uint8)
    scale[page, :, off // block] = now
    code[page, off] = (x / now[..., None]).to(CODE).view(torch.uint8)


def _cache_of(s):
    return [s["k_code"].view(CODE), s["v_code"].view(CODE), s["k_scale"], s["v_scale"]]


def _plain_append(s):
    q, k = s["q"].float(), s["k"].float()
    if s["case"]["norm"]:
        q, k = _normed(q, s["q_gamma"].float()), _normed(k, s["k_gamma"].float())
    _write(s, "k", _rotate(k, s))
    _write(s, "v", s["v"].float())
    return [_rotate(q, s).to(s["dt"])] + _cache_of(s)


def _plain_read(s):
    page, off = _place(s, *_tokens(s))
    return [_stored(s[n + "_code"], s[n + "_scale"], page, off, s["case"]["block"]).to(s["dt"]) for n in ("k", "v")]


def _plain_attend(s):
    case = s["case"]
    B, H, Hkv, D, page = len(s["new"]), case["heads"], case["kv_heads"], case["dim"], case["page"]
    most, longest = max(s["new"]), max(a + c for a, c in zip(s["new"], s["ctx"]))
    seq = torch.arange(B, device=DEV)[:, None]
    j = torch.arange(longest, device=DEV)[None, :]
    start, n, ctx = s["q_start"].long()[:-1, None], s["q_start"].long().diff()[:, None], s["ctx_len"].long()[:, None]
    p, o = _place(s, seq, torch.minimum(j, n + ctx - 1))
    k, v = (_stored(s[x + "_code"], s[x + "_scale"], p, o, case["block"]).transpose(1, 2) for x in ("k", "v"))
    i = torch.arange(most, device=DEV)[None, :]
    token = start + torch.minimum(i, n - 1)                                      # [B, most]
    q = s["q"].float()[token].view(B, most, Hkv, H // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, D)
    score = torch.matmul(q, k.transpose(-1, -2)).view(B, Hkv, -1, most, longest) * s["scale"]
    new = (j - ctx)[:, None, :]                                                  # a new token's number
    if s["mask"] is None:
        see = new <= i[..., None]
    else:
        word = (new.clamp(0, 32 * s["mask"].shape[1] - 1) // 32).expand(-1, most, -1)
        see = (new < 0) | (torch.gather(s["mask"][token], 2, word) >> (new % 32).int()) & 1 > 0
    see = see & (new < n[..., None])
    score = torch.where(see[:, None, None], score, float("-inf"))
    top = score.amax(-1, keepdim=True)
    w = torch.exp(score - torch.where(torch.isfinite(top), top, 0.0))
    w = w / w.sum(-1, keepdim=True)
    out = torch.matmul(w.view(B, Hkv, -1, longest), v).view(B, Hkv, -1, most, D).permute(0, 3, 1, 2, 4)
    s["out"][token[i < n]] = out.reshape(B, most, H, D)[i < n].to(s["dt"])
    return s["out"]


def _move(s, name):
    case, code, scale = s["case"], s[name + "_code"], s[name + "_scale"]
    L, B, A, block, H = case["layers"], case["seqs"], case["accept"], case["block"], case["kv_heads"]
    ctx, seq = s["ctx_len"].long()[:, None], torch.arange(case["seqs"], device=DEV)[:, None]
    dst = ctx + torch.arange(A, device=DEV)
    sp, so = _place(s, seq, ctx + s["path"].long())
    dp, do = _place(s, seq, dst)
    x = _stored(code, scale, sp, so, block)                                      # [L, B, A, H, D]
    which = dst // block - ctx // block                                          # a sequence's first block is 0
    need = torch.zeros((L, B, A // block + 2, H), device=DEV)
    need.scatter_reduce_(2, which[None, :, :, None].expand(L, -1, -1, H), x.abs().amax(-1), "amax")
    need = need.gather(2, which[None, :, :, None].expand(L, -1, -1, H))
    stays = (dst - dst % block < ctx)[None, :, :, None]
    old = scale[:, dp, :, do // block].permute(2, 0, 1, 3) * stays
    now = torch.where(need > 448.0 * old, _power(need), old)
    at = ctx - ctx % block + torch.arange(block, device=DEV)
    live = at < ctx
    p, o = _place(s, seq, torch.minimum(at, ctx))
    again = _stored(code, scale, p, o, block) / now[:, :, :1, :, None]
    code[:, p[live], o[live]] = again[:, live].to(CODE).view(torch.uint8)
    scale[:, dp, :, do // block] = now.permute(1, 2, 0, 3)
    code[:, dp, do] = (x / now[..., None]).to(CODE).view(torch.uint8)


def _plain_commit(s):
    _move(s, "k")
    _move(s, "v")
    return _cache_of(s) + [s["ctx_len"] + s["n_accept"]]


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return {"norm": _plain_norm, "append": _plain_append, "read": _plain_read, "attend": _plain_attend,
                "commit": _plain_commit}[op](s)
    pp = s["pp"]
    if op == "norm" and not case["grad"]:
        pp.pp_head_norm_rope(s["norm"], s["rot"], s["pos"], s["q"], s["k"], s["q_out"], s["k_out"])
        return [s["q_out"], s["k_out"]]
    if op == "norm":
        pp.pp_head_norm_rope_grad(s["norm"], s["rot"], s["pos"], s["q"], s["k"], s["q_grad"], s["k_grad"], s["q_out"],
                                  s["k_out"], s["dq_gamma"], s["dk_gamma"], s["ws"])
        return [s["q_out"], s["k_out"], s["dq_gamma"], s["dk_gamma"]]
    if op == "append":
        pp.pp_kv8_append(s["cache"], s["batch"], s["norm"], s["rot"], s["pos"], s["q"], s["k"], s["v"], s["out"],
                         s["ws"])
        return [s["out"]] + _cache_of(s)
    if op == "read":
        pp.pp_kv8_read(s["cache"], s["batch"], s["k_out"], s["v_out"], s["ws"])
        return [s["k_out"], s["v_out"]]
    if op == "attend":
        pp.pp_tree_attention8(s["cache"], s["batch"], s["q"], s["mask"], s["scale"], s["out"], s["ws"])
        return s["out"]
    pp.pp_kv8_commit(s["cache"], s["batch"], s["path"], s["n_accept"], s["ws"], new_len=s["new_len"],
                     n_layers=case["layers"], layer_stride=s["k_code"].stride(0),
                     scale_layer_stride=s["k_scale"].stride(0))
    return _cache_of(s) + [s["new_len"]]


# ------------------------------------------------------------------------------------------------ exact, fp64

def _turned(x, s, sign):
    """fp64 rotation as a product of complex numbers, one for each pair."""
    freq, layout = s["freq"], s["case"]["layout"]
    n = freq.numel()
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV),
                       sign * torch.outer(s["pos"].double(), freq.double()))
    head, rest = x[..., :2 * n], x[..., 2 * n:]
    pairs = head.unflatten(-1, (2, n)).transpose(-1, -2) if layout == "half" else head.unflatten(-1, (n, 2))
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None, :])
    if layout == "half":
        z = z.transpose(-1, -2)
    return torch.cat([z.flatten(-2), rest], -1)


def _exact_norm(x, gamma):
    rows = x.double().flatten(0, 1)
    size = torch.linalg.vector_norm(rows, dim=1) ** 2 / rows.shape[1] + EPS
    return (rows * size[:, None] ** -0.5 * gamma.double()).view(x.shape)


def _exact_norm_grad(s, name):
    """The gradient of a row as that of x (x.x / D + eps)^(-1/2), written out as a product with its Jacobian."""
    x, gamma = s[name].double(), s[name + "_gamma"].double()
    back = _turned(s[name + "_grad"].double(), s, -1.0)
    size = torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / x.shape[-1] + EPS
    along = torch.einsum("thd,thd->th", back * gamma, x)[..., None]
    return (back * gamma) * size ** -0.5 - x * along / x.shape[-1] * size ** -1.5, \
        torch.einsum("thd,thd->d", back, x * size ** -0.5)


def _numbers(code):
    """fp64 values of e4m3 codes: sign, 4 bits of exponent (bias 7), 3 of fraction."""
    c = code.int()
    e, f = c >> 3 & 15, (c & 7).double()
    mag = torch.where(e > 0, (1.0 + f / 8.0) * torch.exp2(e.double() - 7.0), f * 2.0 ** -9)
    return torch.where(c >> 7 > 0, -mag, mag)


def _rounded(x):
    """fp64 numbers of magnitude up to 448 to the nearest e4m3 number, ties to the even one."""
    e = torch.frexp(x)[1].clamp(min=-5) - 4
    step = torch.exp2(e.double())
    return torch.round(x / step) * step


def _exact_scale(amax):
    """Per value: the smallest power of two s >= 2^-60 with amax <= 448 s."""
    s = torch.exp2(torch.ceil(torch.log2(amax.clamp(min=1e-30) / 448.0)).clamp(min=float(LEAST_EXPONENT)))
    s = torch.where(amax > 448.0 * s, 2.0 * s, s)
    return torch.where((amax <= 224.0 * s) & (s > 2.0 ** LEAST_EXPONENT), s / 2.0, s)


def _exact_fill(case, val, code, scale, table, ctx, src):
    """The entries of one sequence from ctx on become src [..., n, heads, dim], in codes (fp64 numbers) and scales;
    layers, where there are some, come first."""
    page, block = case["page"], case["block"]
    at, n = 0, src.shape[-3]
    while at < n:
        lo = ctx + at - (ctx + at) % block
        end = min(n, lo + block - ctx)
        p, o, blk = table[lo // page], lo % page, lo % page // block
        keep = max(0, min(block, ctx - lo))
        x = src[..., at:end, :, :]
        amax = x.abs().amax((-3, -1))
        now = _exact_scale(amax)
        if keep:
            now = torch.where(amax > 448.0 * scale[..., p, :, blk], now, scale[..., p, :, blk])
            code[..., p, o:o + keep, :, :] = _rounded(val[..., p, o:o + keep, :, :] / now[..., None, :, None])
        scale[..., p, :, blk] = now
        e = (ctx + at) % page
        code[..., p, e:e + end - at, :, :] = _rounded(x / now[..., None, :, None])
        at = end


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "norm":
        if not case["grad"]:
            return [_turned(_exact_norm(s[n], s[n + "_gamma"]), s, 1.0) for n in ("q", "k")]
        (dq, dq_gamma), (dk, dk_gamma) = _exact_norm_grad(s, "q"), _exact_norm_grad(s, "k")
        return [dq, dk, dq_gamma, dk_gamma]
    page, heads, kv, dim, block = case["page"], case.get("heads", 0), case["kv_heads"], case["dim"], case["block"]
    tables = [row.tolist() for row in s["pages"]]
    if case["op"] == "commit":
        out = []
        for name in ("k", "v"):
            code, scale = _numbers(s[name + "_code"]), s[name + "_scale"].double()
            val = code * scale.repeat_interleave(block, -1).transpose(-1, -2)[..., None]
            for b, c in enumerate(s["ctx"]):
                src = [c + i for i in s["path"][b].tolist()]
                x = torch.stack([val[:, tables[b][e // page], e % page] for e in src], 1)
                _exact_fill(case, val, code, scale, tables[b], c, x)
            out.append((code, scale))
        return [out[0][0], out[1][0], out[0][1], out[1][1], None]
    if case["op"] == "append":
        q, k = s["q"].double(), s["k"].double()
        if case["norm"]:
            q, k = _exact_norm(q, s["q_gamma"]), _exact_norm(k, s["k_gamma"])
        q, k = _turned(q, s, 1.0), _turned(k, s, 1.0)
        out = []
        for name, x in (("k", k), ("v", s["v"].double())):
            code, scale = _numbers(s[name + "_code"]), s[name + "_scale"].double()
            val = code * scale.repeat_interleave(block, -1).transpose(-1, -2)[..., None]
            for b, (n, c) in enumerate(zip(s["new"], s["ctx"])):
                lo = s["starts"][b]
                _exact_fill(case, val, code, scale, tables[b], c, x[lo:lo + n])
            out.append((code, scale))
        return [q, out[0][0], out[1][0], out[0][1], out[1][1]]

    def values(name, b, lo, hi, h):
        at = torch.arange(lo, hi, device=DEV)
        rows, offs = s["pages"][b].long()[at // page], at % page
        return _numbers(s[name + "_code"][rows, offs, h]) * s[name + "_scale"].double()[rows, h, offs // block][:, None]

    if case["op"] == "read":
        return [torch.cat([torch.stack([values(name, b, c, c + n, h) for h in range(kv)], 1)
                           for b, (n, c) in enumerate(zip(s["new"], s["ctx"]))]) for name in ("k", "v")]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    for b, (n, c) in enumerate(zip(s["new"], s["ctx"])):
        lo = s["starts"][b]
        see = torch.ones((n, n + c), dtype=torch.bool, device=DEV)
        if case["tree"]:
            vis = _tree_of(_tree(n, b))[0]
            see[:, c:] = torch.tensor([[bool(v >> j & 1) for j in range(n)] for v in vis], device=DEV)
        else:
            see[:, c:] = torch.ones((n, n), dtype=torch.bool, device=DEV).tril()
        for h in range(kv):
            k, v = values("k", b, 0, n + c, h), values("v", b, 0, n + c, h)
            for i in range(h * heads // kv, (h + 1) * heads // kv):
                score = (s["q"][lo:lo + n, i].double() @ k.T) / math.sqrt(dim)
                out[lo:lo + n, i] = torch.softmax(score.masked_fill(~see, float("-inf")), -1) @ v
    return out
