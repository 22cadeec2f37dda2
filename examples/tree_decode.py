"""Greedy decoding with trees of drafted tokens, on a small model with random weights.

One step of a layer stack, as a serving loop runs it:

  q, k, v projections                     (torch products)
  pp_kv_append       rotate q and k, write k and v to their pages
  pp_tree_attention  every new token over its context and its ancestors
  output projection                       (torch product)
  pp_layer_chained   x = RMSNorm(x + attention), router, sparse FFN
  ...
  pp_kv_commit       after the last layer: the accepted path, in every layer's cache

A step takes the last token and a tree of guesses behind it (here: what followed earlier occurrences of the last
tokens), computes the next token of every node at once, and accepts the path of guesses that greedy decoding would
have taken.  The text is the same as without guesses (in bf16 up to near-ties, which the rounding of steps of other
sizes may decide otherwise); `main` prints how many steps each way takes.

  python examples/tree_decode.py [--tokens N] [--dtype bf16|f32]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2605_28283_gb300 import binding as pp  # noqa: E402

PAGE = 16


class TreeDecoder:
    """A stack of attention + sparse-FFN layers over one sequence's paged cache."""

    def __init__(self, vocab=96, d_model=256, n_layers=2, heads=4, kv_heads=2, n_experts=16, dtype="f32", p=0.7,
                 max_tokens=1024, max_step=64, seed=0):
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.heads, self.kv_heads, self.dim, self.p = heads, kv_heads, d_model // heads, p
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def weight(*shape, std):
            return (torch.randn(shape, generator=g, device="cuda") * std).to(self.dtype)

        d, kv = d_model, kv_heads * self.dim
        self.embed, self.head = weight(vocab, d, std=1.0), weight(vocab, d, std=1.0)
        self.layers = [dict(qkv=weight(d + 2 * kv, d, std=d ** -0.5), out=weight(d, d, std=d ** -0.5),
                            router=weight(n_experts, d, std=3 * d ** -0.5),
                            up=weight(n_experts * 64, d, std=d ** -0.5),
                            down=weight(d, n_experts * 64, std=(n_experts * 64) ** -0.5)) for _ in range(n_layers)]
        pages = -(-max_tokens // PAGE)
        shape = (n_layers, pages, PAGE, kv_heads, self.dim)
        self.k, self.v = (torch.zeros(shape, dtype=self.dtype, device="cuda") for _ in range(2))
        self.caches = [pp.KVCache(self.k[i], self.v[i], heads) for i in range(n_layers)]
        self.table = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)[None]
        self.rot = pp.Rotation.make(self.dim)
        self.desc = pp.make_desc(d, n_experts, dtype, "relu")
        self.ws = pp.alloc_attn_workspace(self.caches[0])
        self.ffn_ws = pp.alloc_workspace(self.desc, max_step)
        self.length = torch.zeros(1, dtype=torch.int32, device="cuda")  # committed cache entries
        self.new_length = torch.empty_like(self.length)

    def forward(self, tokens, depth=None, mask=None):
        """Logits [T, vocab] of new tokens behind the committed ones: a chain, or a tree given by its nodes' depths
        and visibility bits.  Their keys and values are appended, not committed."""
        T = len(tokens)
        x = self.embed[torch.tensor(tokens, device="cuda")]
        q_start = torch.tensor([0, T], dtype=torch.int32, device="cuda")
        batch = pp.Batch(q_start, self.length, self.table, T)
        positions = None if depth is None else self.length + torch.tensor(depth, dtype=torch.int32, device="cuda")
        nq, nkv = self.heads * self.dim, self.kv_heads * self.dim
        for cache, w in zip(self.caches, self.layers):
            qkv = x @ w["qkv"].T
            q, k, v = qkv[:, :nq], qkv[:, nq:nq + nkv], qkv[:, nq + nkv:]
            pp.pp_kv_append(cache, batch, self.rot, positions, q, k, v, q, self.ws)  # queries rotated in place
            attn = torch.empty((T, nq), dtype=self.dtype, device="cuda")
            pp.pp_tree_attention(cache, batch, q, mask, self.dim ** -0.5, attn, self.ws)
            y_attn = attn @ w["out"].T
            mid, y = torch.empty_like(x), torch.empty_like(x)
            pp.pp_layer_chained(self.desc, x, y_attn, None, 1e-6, T, w["router"], None, w["up"], w["down"], self.p, None,
                                mid, y, self.ffn_ws)
            s = (mid + y).float()
            x = (s * torch.rsqrt(s.square().mean(-1, keepdim=True) + 1e-6)).to(self.dtype)
        self.batch = batch
        return (x @ self.head.T).float()

    def commit(self, path):
        """Keep the entries of `path` (ascending numbers of the last forward's tokens) in every layer."""
        p = torch.tensor([path], dtype=torch.int32, device="cuda")
        n = torch.tensor([len(path)], dtype=torch.int32, device="cuda")
        pp.pp_kv_commit(self.caches[0], self.batch, p, n, self.ws, new_len=self.new_length, n_layers=len(self.caches),
                        layer_stride=self.k.stride(0))
        self.length, self.new_length = self.new_length, self.length

    def check(self):
        for ws in (self.ws, self.ffn_ws):
            status = pp.pp_get_device_status(ws)
            if status != pp.PP_OK:
                raise pp.PPError(status, "tree_decode")


def guess_tree(text, width, depth, limit):
    """Nodes (token, parent) below the last token: what followed the latest earlier occurrences of the text's last
    token, `width` of them, `depth` tokens each, common beginnings shared."""
    nodes = [(text[-1], -1)]
    children = {}
    starts = [i for i in range(len(text) - 2, -1, -1) if text[i] == text[-1]][:width]
    for i in starts:
        at = 0
        for tok in text[i + 1:i + 1 + depth]:
            key = (at, tok)
            if key not in children:
                if len(nodes) == limit:
                    break
                children[key] = len(nodes)
                nodes.append((tok, at))
            at = children[key]
    return nodes


def tree_tensors(nodes):
    """(depths, mask bits [T, words] int32 on the GPU) of nodes listed parents first."""
    words = -(-len(nodes) // 32)
    depth, rows = [], []
    for i, (_, parent) in enumerate(nodes):
        depth.append(0 if parent < 0 else depth[parent] + 1)
        bits = (0 if parent < 0 else rows[parent]) | 1 << i
        rows.append(bits)
    mask = torch.tensor([[(b >> (32 * w)) & 0xffffffff for w in range(words)] for b in rows], dtype=torch.int64)
    return depth, mask.to(torch.int32).cuda()


def generate(model, prompt, n, width=0, depth=6, limit=32):
    """n greedy tokens behind the prompt; width > 0: with trees of guesses.  Returns (tokens, steps)."""
    text = list(prompt)
    if len(prompt) > 1:
        model.forward(prompt[:-1])
        model.commit(list(range(len(prompt) - 1)))
    steps = 0
    while len(text) < len(prompt) + n:
        nodes = guess_tree(text, width, depth, limit) if width else [(text[-1], -1)]
        depths, mask = tree_tensors(nodes)
        best = model.forward([t for t, _ in nodes], depths, mask).argmax(-1).tolist()
        path, at = [0], 0
        while True:
            text.append(best[at])
            step = [i for i, (tok, parent) in enumerate(nodes) if parent == at and tok == best[at]]
            if not step:
                break
            at = step[0]
            path.append(at)
        model.commit(path)
        steps += 1
    model.check()
    return text[len(prompt):len(prompt) + n], steps


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=128)
    ap.add_argument("--dtype", choices=["bf16", "f32"], default="bf16")
    args = ap.parse_args()
    prompt = [(7 * i) % 23 for i in range(40)]
    for width in (0, 4):
        tokens, steps = generate(TreeDecoder(dtype=args.dtype), prompt, args.tokens, width=width)
        print("%s: %d tokens in %d steps: %s ..." % ("trees of guesses" if width else "one token a step", len(tokens), steps,
                                                      tokens[:12]))


if __name__ == "__main__":
    main()
