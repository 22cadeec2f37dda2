"""Cases of the serving operators around the sparse FFN: rotary positions, the paged key/value cache and the
attention of new tokens over it.

Four operators, as one decode step uses them:

* rope:    y = x rotated by its token's position (or rotated back: the gradient of the rotation);
* append:  queries rotated, keys rotated and values copied into the pages of their sequences;
* attend:  attention of each sequence's new tokens (one token, a tree of drafted tokens, or a prompt) over its
           cached tokens and over those new tokens that its mask lets it see;
* commit:  the accepted path of a drafted tree moved together behind the cached tokens, in every layer.

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


# --------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one decode step's queries of a batch of 8
        dict(name="rope_decode_8", op="rope", dtype="bf16", tokens=8, heads=32, dim=128, rot=128, layout="half",
             inverse=False, max_pos=8192),
        # gradient of the rotation over 4 prompts of 2048 tokens, 40 heads
        dict(name="rope_grad_8192", op="rope", dtype="bf16", tokens=8192, heads=40, dim=128, rot=128, layout="half",
             inverse=True, max_pos=2048),
        # a drafted tree for each of 3 sequences of a small fp32 model, a quarter of the head rotated
        dict(name="append_tree_f32", op="append", dtype="f32", seqs=3, new_lo=13, new_hi=13, ctx_lo=20, ctx_hi=700,
             heads=16, kv_heads=16, dim=64, rot=16, layout="interleaved", page=16, tree=True),
        # one token for each of 64 sequences
        dict(name="append_decode_64", op="append", dtype="bf16", seqs=64, new_lo=1, new_hi=1, ctx_lo=64, ctx_hi=1024,
             heads=32, kv_heads=8, dim=128, rot=128, layout="half", page=64, tree=False),
        # 4 prompts, ragged, up to 2048 tokens
        dict(name="append_prompt_8k", op="append", dtype="bf16", seqs=4, new_lo=1900, new_hi=2048, ctx_lo=0, ctx_hi=0,
             heads=40, kv_heads=40, dim=128, rot=128, layout="half", page=64, tree=False),
        # batch-1 decode, a key head for each query head
        dict(name="attend_decode_1", op="attend", dtype="bf16", seqs=1, new_lo=1, new_hi=1, ctx_lo=1023, ctx_hi=1023,
             heads=32, kv_heads=32, dim=128, page=64, tree=False),
        # a drafted tree on a small fp32 model
        dict(name="attend_tree_f32", op="attend", dtype="f32", seqs=3, new_lo=9, new_hi=13, ctx_lo=100, ctx_hi=1000,
             heads=16, kv_heads=16, dim=64, page=16, tree=True),
        # batched decode over ragged contexts, shared key heads
        dict(name="attend_decode_64", op="attend", dtype="bf16", seqs=64, new_lo=1, new_hi=1, ctx_lo=64, ctx_hi=8191,
             heads=32, kv_heads=8, dim=128, page=64, tree=False),
        # drafted trees of up to 48 tokens over ragged contexts, small pages
        dict(name="attend_tree_8", op="attend", dtype="bf16", seqs=8, new_lo=17, new_hi=48, ctx_lo=500, ctx_hi=6001,
             heads=32, kv_heads=8, dim=128, page=16, tree=True),
        # 4 prompts of 2048 tokens
        dict(name="attend_prompt_8k", op="attend", dtype="bf16", seqs=4, new_lo=2048, new_hi=2048, ctx_lo=0, ctx_hi=0,
             heads=40, kv_heads=40, dim=128, page=64, tree=False),
        # one sequence's accepted path, one layer
        dict(name="commit_1", op="commit", dtype="bf16", seqs=1, layers=1, draft=24, accept=5, ctx_lo=300, ctx_hi=300,
             kv_heads=8, dim=128, page=16),
        # the accepted paths of 32 sequences in 32 layers
        dict(name="commit_32x32", op="commit", dtype="bf16", seqs=32, layers=32, draft=48, accept=8, ctx_lo=20,
             ctx_hi=300, kv_heads=8, dim=128, page=64),
    ]


def _log_int(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm (lo = 0 allowed)."""
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo + 1), math.log(hi + 2)))) - 1))


def _draw_once(rng):
    op = rng.choice(["rope", "append", "attend", "attend", "attend", "commit"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    heads, kv_heads, dim = rng.choice([(32, 32, 128), (32, 8, 128), (40, 40, 128), (16, 16, 64), (32, 4, 128),
                                       (12, 3, 80)])
    page = rng.choice([8, 16, 24, 32, 64, 128])
    rot = rng.choice([dim, dim, dim // 2, dim // 4])
    layout = rng.choice(["half", "interleaved"])
    if op == "rope":
        return dict(op=op, dtype=dtype, tokens=_log_int(rng, 1, 8192), heads=heads, dim=dim, rot=rot, layout=layout,
                    inverse=rng.random() < 0.5, max_pos=_log_int(rng, 64, 8192))
    if op == "commit":
        draft = rng.randint(2, 64)
        lo = _log_int(rng, 0, 300)
        return dict(op=op, dtype=dtype, seqs=_log_int(rng, 1, 32), layers=_log_int(rng, 1, 32), draft=draft,
                    accept=rng.randint(1, max(1, min(8, draft // 2))), ctx_lo=lo, ctx_hi=lo + _log_int(rng, 0, 300),
                    kv_heads=kv_heads, dim=dim, page=page)
    kind = rng.choice(["decode", "tree", "prompt"])
    seqs = _log_int(rng, 1, 64)
    if kind == "decode":
        lo = hi = 1
    elif kind == "tree":
        lo = rng.randint(2, 64)
        hi = min(64, lo + rng.randint(0, 24))
    else:
        seqs = min(seqs, 8)
        lo = _log_int(rng, 2, 2048)
        hi = min(2048, lo + _log_int(rng, 0, 512))
    ctx_lo = _log_int(rng, 0, 8000)
    ctx_hi = min(8191, ctx_lo + _log_int(rng, 0, 4000))
    case = dict(op=op, dtype=dtype, seqs=seqs, new_lo=lo, new_hi=hi, ctx_lo=ctx_lo, ctx_hi=ctx_hi, heads=heads,
                kv_heads=kv_heads, dim=dim, page=page, tree=kind == "tree")
    if op == "append":
        case.update(rot=rot, layout=layout)
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
        if _cost(case) <= limit[case["op"]] and _pool(case) <= 3 << 30:
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
    """Bytes of a case's key and value pages."""
    if case["op"] == "rope":
        return 0
    new, ctx = _lengths(case)
    pages = sum(-(-(n + c) // case["page"]) for n, c in zip(new, ctx)) + 2
    return pages * case["page"] * case["kv_heads"] * case["dim"] * ESZ[case["dtype"]] * 2 * case.get("layers", 1)


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


def _frequencies(rot, scaled):
    """Radians per position of each rotated pair; `scaled` divides the slow half by 4, as long contexts do."""
    f = [10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)]
    return [v / 4.0 if scaled and i >= rot // 4 else v for i, v in enumerate(f)]


def work(case):
    e = ESZ[case["dtype"]]
    if case["op"] == "rope":
        elems = case["tokens"] * case["heads"]
        return {"bytes": 2 * elems * case["dim"] * e + 4 * case["tokens"], "flops": 3 * elems * case["rot"]}
    new, ctx = _lengths(case)
    kv_row = case["kv_heads"] * case["dim"] * e
    if case["op"] == "commit":
        return {"bytes": case["seqs"] * (4 * case["accept"] * kv_row * case["layers"] + 4 * case["accept"] + 12),
                "flops": 0}
    q_row = case["heads"] * case["dim"] * e
    n = sum(new)
    if case["op"] == "append":
        return {"bytes": n * (2 * q_row + 4 * kv_row + 4) + 8 * case["seqs"],
                "flops": 3 * n * (case["heads"] + case["kv_heads"]) * case["rot"]}
    pairs = 0
    for b, (a, c) in enumerate(zip(new, ctx)):
        seen = sum(d + 1 for d in _tree_of(_tree(a, b))[1]) if case["tree"] else a * (a + 1) // 2
        pairs += a * c + seen
    words = -(-max(new) // 32) if case["tree"] else 0
    table = sum(-(-(a + c) // case["page"]) for a, c in zip(new, ctx))
    return {"bytes": n * (2 * q_row + 4 * words) + sum(a + c for a, c in zip(new, ctx)) * 2 * kv_row + 4 * table +
            8 * case["seqs"], "flops": 4 * pairs * case["heads"] * case["dim"]}


# -------------------------------------------------------------------------------------------------- inputs

def _inputs(case, seed):
    """Tensors of one call, from the seed alone."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 17)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * std).to(dt)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=DEV)

    s = {"case": case}
    if "rot" in case:
        s["freq"] = torch.tensor(_frequencies(case["rot"], case["op"] == "append"), dtype=torch.float32, device=DEV)
    if case["op"] == "rope":
        s["x"] = normal(case["tokens"], case["heads"], case["dim"])
        s["pos"] = torch.randint(0, case["max_pos"], (case["tokens"],), generator=g, device=DEV, dtype=torch.int32)
        s["y"] = torch.empty_like(s["x"])
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
    s["k_cache"], s["v_cache"] = normal(*shape), normal(*shape)
    if case["op"] == "commit":
        # the first accepted token lies past the places that the path moves to, so that another pass on the same
        # state gives the same cache
        rng = random.Random(seed)
        acc = case["accept"]
        s["path"] = ints([sorted(rng.sample(range(acc, case["draft"]), acc)) for _ in new])
        s["n_accept"] = ints([acc] * len(new))
        s["new_len"] = torch.empty_like(s["ctx_len"])
        return s
    trees = [_tree_of(_tree(n, b)) for b, n in enumerate(new)] if case["tree"] else None
    depth = [trees[b][1][i] if trees else i for b, n in enumerate(new) for i in range(n)]
    first = [c for n, c in zip(new, ctx) for _ in range(n)]
    s["pos"] = ints([c + d for c, d in zip(first, depth)])
    s["q"] = normal(T, case["heads"], case["dim"], std=1.3)
    s["out"] = torch.empty_like(s["q"])
    if case["op"] == "append":
        s["k"], s["v"] = normal(T, case["kv_heads"], case["dim"]), normal(T, case["kv_heads"], case["dim"])
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
        if "freq" in s:
            s["rot"] = pp.Rotation(s["freq"], case["layout"])
        if case["op"] != "rope":
            kc, vc = s["k_cache"], s["v_cache"]
            heads = case.get("heads", case["kv_heads"])
            s["cache"] = pp.KVCache(kc[0], vc[0], heads) if case["op"] == "commit" else pp.KVCache(kc, vc, heads)
            s["batch"] = pp.Batch(s["q_start"], s["ctx_len"], s["pages"], s["starts"][-1])
            s["ws"] = pp.alloc_attn_workspace(s["cache"])
    return s


# ---------------------------------------------------------------------------------------------- plain form, fp32

def _phasor(angle):
    return torch.cos(angle), torch.sin(angle)


def _times(a, b):
    return a[0] * b[0] - a[1] * b[1], a[0] * b[1] + a[1] * b[0]


def _cos_sin(pos, freq):
    """cos and sin of pos * freq.  The angle goes to thousands of radians, so the product is taken apart into
    pieces that fp32 holds exactly (12 bits of the position times 12 of the frequency) and a small rest."""
    hi = (freq.view(torch.int32) & -4096).view(torch.float32)
    lo = freq - hi
    p0, p1 = (pos & 4095).float()[:, None], (pos & -4096).float()[:, None]
    small = (p0 + p1) * lo
    return _times(_times(_phasor(p1 * hi), _phasor(p0 * hi)), _phasor(small))


def _rotate(x, pos, freq, layout, inverse):
    """fp32 rotation of x [T, H, D]; the first 2 * len(freq) elements of a head are rotated."""
    c, s = _cos_sin(pos, freq)
    c, s = c[:, None, :], (-s if inverse else s)[:, None, :]
    n = freq.numel()
    y = x.float().clone()
    if layout == "half":
        a, b = x[..., :n].float(), x[..., n:2 * n].float()
        y[..., :n], y[..., n:2 * n] = a * c - b * s, b * c + a * s
    else:
        a, b = x[..., 0:2 * n:2].float(), x[..., 1:2 * n:2].float()
        y[..., 0:2 * n:2], y[..., 1:2 * n:2] = a * c - b * s, b * c + a * s
    return y


def _slots(s):
    """(page, offset) of each new token."""
    page = s["case"]["page"]
    t = torch.arange(s["starts"][-1], device=DEV)
    b = torch.searchsorted(s["q_start"][1:].long(), t, right=True)
    at = s["ctx_len"].long()[b] + t - s["q_start"].long()[b]
    return s["pages"].long()[b, at // page], at % page


def _plain_append(s):
    case = s["case"]
    q = _rotate(s["q"], s["pos"], s["freq"], case["layout"], False).to(s["q"].dtype)
    k = _rotate(s["k"], s["pos"], s["freq"], case["layout"], False).to(s["k"].dtype)
    where = _slots(s)
    s["k_cache"][where] = k
    s["v_cache"][where] = s["v"]
    return [q, s["k_cache"], s["v_cache"]]


def _plain_attend(s):
    case = s["case"]
    group, page = case["heads"] // case["kv_heads"], case["page"]
    out = s["out"]
    for b, (n, c) in enumerate(zip(s["new"], s["ctx"])):
        lo, total = s["starts"][b], n + c
        rows = s["pages"][b, :-(-total // page)].long()
        k = s["k_cache"][rows].flatten(0, 1)[:total].float().permute(1, 2, 0)       # [Hkv, D, total]
        v = s["v_cache"][rows].flatten(0, 1)[:total].float().transpose(0, 1)        # [Hkv, total, D]
        q = s["q"][lo:lo + n].float().view(n, -1, group, case["dim"]).permute(1, 2, 0, 3)
        score = torch.matmul(q.reshape(q.shape[0], group * n, -1), k) * s["scale"]
        score = score.view(-1, group, n, total)
        j = torch.arange(n, device=DEV)
        if s["mask"] is None:
            see = j[None, :] <= j[:, None]
        else:
            see = (s["mask"][lo:lo + n][:, j // 32] >> (j % 32).int()) & 1 > 0
        score[..., c:] = torch.where(see, score[..., c:], float("-inf"))
        top = score.amax(-1, keepdim=True)
        p = torch.exp(score - torch.where(torch.isfinite(top), top, 0.0))
        p = p / p.sum(-1, keepdim=True)
        o = torch.matmul(p.view(-1, group * n, total), v).view(-1, group, n, case["dim"])
        out[lo:lo + n] = o.permute(2, 0, 1, 3).reshape(n, -1, case["dim"]).to(out.dtype)
    return out


def _plain_commit(s):
    page = s["case"]["page"]
    ctx = s["ctx_len"].long()[:, None]
    src = ctx + s["path"].long()
    dst = ctx + torch.arange(src.shape[1], device=DEV)[None, :]
    b = torch.arange(src.shape[0], device=DEV)[:, None]
    table = s["pages"].long()
    for cache in (s["k_cache"], s["v_cache"]):
        cache[:, table[b, dst // page], dst % page] = cache[:, table[b, src // page], src % page]
    return [s["k_cache"], s["v_cache"], s["ctx_len"] + s["n_accept"]]


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        if op == "rope":
            return _rotate(s["x"], s["pos"], s["freq"], case["layout"], case["inverse"]).to(s["x"].dtype)
        return {"append": _plain_append, "attend": _plain_attend, "commit": _plain_commit}[op](s)
    pp = s["pp"]
    if op == "rope":
        pp.pp_rope(s["rot"], s["pos"], s["x"], s["y"], inverse=case["inverse"])
        return s["y"]
    if op == "append":
        pp.pp_kv_append(s["cache"], s["batch"], s["rot"], s["pos"], s["q"], s["k"], s["v"], s["out"], s["ws"])
        return [s["out"], s["k_cache"], s["v_cache"]]
    if op == "attend":
        pp.pp_tree_attention(s["cache"], s["batch"], s["q"], s["mask"], s["scale"], s["out"], s["ws"])
        return s["out"]
    pp.pp_kv_commit(s["cache"], s["batch"], s["path"], s["n_accept"], s["ws"], new_len=s["new_len"],
                    n_layers=case["layers"], layer_stride=s["k_cache"].stride(0))
    return [s["k_cache"], s["v_cache"], s["new_len"]]


# ------------------------------------------------------------------------------------------------ exact, fp64

def _turned(x, pos, freq, layout, sign):
    """fp64 rotation as a product of complex numbers, one for each pair."""
    n = freq.numel()
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), sign * torch.outer(pos.double(), freq.double()))
    x = x.double()
    head, rest = x[..., :2 * n], x[..., 2 * n:]
    pairs = head.unflatten(-1, (2, n)).transpose(-1, -2) if layout == "half" else head.unflatten(-1, (n, 2))
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None, :])
    if layout == "half":
        z = z.transpose(-1, -2)
    return torch.cat([z.flatten(-2), rest], -1)


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "commit":  # moves whole rows: nothing is computed
        return None
    if case["op"] == "rope":
        return _turned(s["x"], s["pos"], s["freq"], case["layout"], -1.0 if case["inverse"] else 1.0)
    page, heads, kv, dim = case["page"], case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "append":
        q, k = (_turned(s[n], s["pos"], s["freq"], case["layout"], 1.0) for n in ("q", "k"))
        kc, vc = s["k_cache"].double(), s["v_cache"].double()
        for b, (n, c) in enumerate(zip(s["new"], s["ctx"])):
            table = s["pages"][b].tolist()
            for i in range(n):
                p, o = table[(c + i) // page], (c + i) % page
                kc[p, o], vc[p, o] = k[s["starts"][b] + i], s["v"][s["starts"][b] + i].double()
        return [q, kc, vc]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    for b, (n, c) in enumerate(zip(s["new"], s["ctx"])):
        lo = s["starts"][b]
        at = torch.arange(n + c, device=DEV)
        rows, offs = s["pages"][b].long()[at // page], at % page
        see = torch.ones((n, n + c), dtype=torch.bool, device=DEV)
        if case["tree"]:
            vis = _tree_of(_tree(n, b))[0]
            see[:, c:] = torch.tensor([[bool(v >> j & 1) for j in range(n)] for v in vis], device=DEV)
        else:
            see[:, c:] = torch.ones((n, n), dtype=torch.bool, device=DEV).tril()
        for h in range(heads):
            k = s["k_cache"][rows, offs, h * kv // heads].double()
            v = s["v_cache"][rows, offs, h * kv // heads].double()
            score = (s["q"][lo:lo + n, h].double() @ k.T) / math.sqrt(dim)
            out[lo:lo + n, h] = torch.softmax(score.masked_fill(~see, float("-inf")), -1) @ v
    return out
