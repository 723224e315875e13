"""Tree decoding of a small random model with the library's tree operators.

Each step verifies a tree of drafted tokens in one pass: the last emitted token
and, below it, what followed the same tokens earlier in the sequence (a lookup
in the sequence itself stands in for a draft model), several continuations a
position.  The target draws a token at every node, the walk down the tree keeps
the branch that it agrees with, and that branch's keys and values become the
sequence's next cache entries.  A tree of one node is ordinary autoregressive
decoding, which the same code does for comparison.

    python examples/tree_decode.py [--sample] [--tokens N]
"""
from __future__ import annotations

import argparse
import os
import sys
from typing import List, Sequence, Tuple

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2504_18583_gb300 import tree  # noqa: E402

PAGE = 16


class Model:
    """A decoder with per-head norms of queries and keys: random weights, fp32 products, a bf16 cache."""

    def __init__(self, vocab=512, layers=2, d=256, heads=(8, 2), hd=64, seed=1):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.vocab, self.layers, self.hd = vocab, layers, hd
        self.Hq, self.Hkv = heads

        def w(*shape, scale=None):
            return torch.randn(shape, generator=g, device="cuda") * (scale or shape[-1] ** -0.5)

        self.embed = w(vocab, d, scale=1.0)
        self.head = w(vocab, d)
        self.wqkv = [w((self.Hq + 2 * self.Hkv) * hd, d) for _ in range(layers)]
        self.wo = [w(d, self.Hq * hd) for _ in range(layers)]
        self.w1 = [w(2 * d, d) for _ in range(layers)]
        self.w2 = [w(d, 2 * d) for _ in range(layers)]
        self.q_gain, self.k_gain = [(1.0 + 0.1 * w(hd, scale=1.0)).bfloat16() for _ in range(2)]
        self.freq, self.amplitude = tree.rope_frequencies(hd, 10000.0, "yarn", 4.0, 64, 1.0, 32.0)

    @staticmethod
    def norm(x):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)

    def forward(self, tokens, plan, pool, table, ctx_len, n_nodes):
        """Logits [B, N, vocab] of a tree's nodes; their keys and values go to the pool."""
        mask, pos, slots = plan
        B, N = tokens.shape
        h = self.embed[tokens.long().view(-1).clamp(min=0)]
        for l in range(self.layers):
            qkv = (self.norm(h) @ self.wqkv[l].T).bfloat16()
            q = tree.qk_norm_rope(qkv, self.Hq, self.Hkv, pos.view(-1), slots.view(-1), pool[l, 0], pool[l, 1], self.freq,
                                  q_gain=self.q_gain, k_gain=self.k_gain, amplitude=self.amplitude)
            o = tree.tree_attention(q.view(B, N, self.Hq, self.hd), pool[l, 0], pool[l, 1], table, ctx_len, n_nodes, mask)
            h = h + o.float().view(B * N, -1) @ self.wo[l].T
            h = h + torch.nn.functional.silu(self.norm(h) @ self.w1[l].T) @ self.w2[l].T
        return (self.norm(h) @ self.head.T).view(B, N, self.vocab) * 3.0


def lookup_tree(history: Sequence[int], width: int, branches: int, depth: int) -> Tuple[List[int], List[int]]:
    """Tokens and parents of a tree whose root is the last token: below each
    branch's end, what followed the same two tokens (or one) before."""
    tokens, parents = [history[-1]], [-1]
    open_nodes = [(0, list(history[-2:]), 0)]
    while open_nodes and len(tokens) < width:
        node, tail, level = open_nodes.pop(0)
        if level == depth:
            continue
        found: List[int] = []
        for n in (2, 1):
            for i in range(len(history) - 1, n - 1, -1):
                if list(history[i - n:i]) == tail[-n:] and history[i] not in found:
                    found.append(history[i])
        for t in found[:branches]:
            if len(tokens) < width:
                open_nodes.append((len(tokens), (tail + [t])[-2:], level + 1))
                tokens.append(t)
                parents.append(node)
    return tokens, parents


def generate(model: Model, prompts: Sequence[Sequence[int]], n_new: int, width: int = 16, branches: int = 3, depth: int = 5,
             sample: bool = False, seed: int = 0):
    """Token lists and the number of target passes.  width 1: autoregressive."""
    B = len(prompts)
    most = max(len(p) for p in prompts) + n_new + 2 * width
    pages = -(-most // PAGE)
    g = torch.Generator().manual_seed(seed)
    table = torch.randperm(B * pages, generator=g).to(torch.int32).view(B, pages).cuda()
    pool = torch.empty((model.layers, 2, B * pages, model.Hkv, PAGE, model.hd), dtype=torch.bfloat16, device="cuda")
    draws = torch.Generator(device="cuda").manual_seed(seed)
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    ctx_len = dev([0] * B)
    # the prompt is a chain: every token but the last one goes through the cache first
    for at in range(0, max(len(p) for p in prompts) - 1, 64):
        part = [list(p[:-1][at:at + 64]) for p in prompts]
        N = max(max(len(x) for x in part), 1)
        chain = dev([[i - 1 for i in range(N)]] * B)
        n_nodes = dev([len(x) for x in part])
        plan = tree.tree_plan(chain, n_nodes, ctx_len, table, B * pages)
        model.forward(dev([x + [0] * (N - len(x)) for x in part]), plan, pool, table, ctx_len, n_nodes)
        ctx_len = ctx_len + n_nodes
    out = [list(p) for p in prompts]
    passes = 0
    while min(len(o) - len(p) for o, p in zip(out, prompts)) < n_new:
        trees = [lookup_tree(o, width, branches, depth) for o in out]
        live = [len(o) - len(p) < n_new for o, p in zip(out, prompts)]
        n_nodes = dev([len(t[0]) if on else 0 for t, on in zip(trees, live)])
        tokens = dev([t[0] + [-1] * (width - len(t[0])) for t in trees])
        parents = dev([t[1] + [-1] * (width - len(t[1])) for t in trees])
        plan = tree.tree_plan(parents, n_nodes, ctx_len, table, B * pages)
        logits = model.forward(tokens, plan, pool, table, ctx_len, n_nodes).view(B * width, -1)
        rows = (B * width,)
        u = torch.rand(rows, generator=draws, device="cuda")
        full = lambda v, t=torch.float32: torch.full(rows, v, dtype=t, device="cuda")  # noqa: E731
        drawn, _ = tree.sample(logits, u, full(0.8 if sample else 0.0), full(50, torch.int32), full(0.95), full(0.02))
        _, emitted, ctx_len = tree.tree_commit(drawn.view(B, width), tokens, parents, n_nodes, ctx_len, table, pool)
        for o, row, p in zip(out, emitted.tolist(), prompts):
            o += [t for t in row if t >= 0][:n_new - (len(o) - len(p))]
        # a sequence that is done keeps its cache; its last tokens may not be in it, and it is not asked again
        passes += 1
    return out, passes


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--sample", action="store_true")
    ap.add_argument("--tokens", type=int, default=96)
    args = ap.parse_args()
    model = Model()
    g = torch.Generator().manual_seed(5)
    prompts = [torch.randint(0, model.vocab, (n,), generator=g).tolist() for n in (40, 7, 100)]
    tree_out, tree_passes = generate(model, prompts, args.tokens, sample=args.sample)
    ar_out, ar_passes = generate(model, prompts, args.tokens, width=1, sample=args.sample)
    for p, o in zip(prompts, tree_out):
        print("...", o[len(p):len(p) + 24])
    print(f"{args.tokens} tokens a sequence: {tree_passes} passes with trees, {ar_passes} without")


if __name__ == "__main__":
    main()
