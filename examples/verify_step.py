"""A decode loop around the restricted head: draft trees are grown by the head, verified by one layer of attention over an 8-bit
cache, and their tokens sampled.

    python examples/verify_step.py [--steps 8] [--temperature 0.8]

The "model" is one attention layer with random weights between the embedding of a token and the LM head; it stands for
the places at which a program has these calls, not for a language model.  Every step, for each sequence:

  1. the restricted head proposes a tree: its best tokens, and under the best of them the next ones (active_lmhead_topk);
  2. K and V of the tree's nodes go into the cache behind the sequence's tokens (kv_write);
  3. all nodes attend over the cache at once, each to the sequence and to its own ancestors (kv_attention with tree words);
  4. the target's logits of every node give a token (sample); a child that carries its parent's token is accepted;
  5. K and V of the accepted nodes are written again, side by side (kv_write), and the sequence is longer by them.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2605_27390_amd as ev  # noqa: E402

WIDTH = 4                                                     # children of a node that has any
DEPTH = 3                                                     # nodes on the best path below the root


class Loop:
    def __init__(self, S=4, V=8192, active=2048, d=512, heads=4, group=2, dim=64, page=64, capacity=1024, kind="e4m3", seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weights(*shape):
            return torch.randn(shape, generator=g, device="cuda").mul_(1 / math.sqrt(shape[-1])).to(torch.bfloat16)

        self.S, self.V, self.d, self.heads, self.group, self.dim = S, V, d, heads, group, dim
        self.embed, self.W_lm = torch.randn((V, d), generator=g, device="cuda").to(torch.bfloat16), weights(V, d).mul_(4)
        self.W_qkv, self.W_o = weights((heads * group + 2 * heads) * dim, d), weights(d, heads * group * dim)
        # the draft's active vocabulary
        ids = torch.randperm(V, generator=g, device="cuda")[:active].to(torch.int32)
        self.W_act, self.act_ids = ev.PackedMatrix(active, d), torch.empty(active, dtype=torch.int32, device="cuda")
        ev.active_gather(self.W_lm, ids, None, self.W_act, self.act_ids)
        # the cache: every sequence has its pages
        width = capacity // page
        self.capacity = width * page                          # tokens of a sequence, the nodes of a tree among them
        self.cache = ev.KVCache(S * width, page, heads, dim, kind)
        self.table = torch.randperm(S * width, generator=g, device="cuda").to(torch.int32).view(S, width)
        self.lens = [0] * S                                   # tokens in the cache
        self.last = torch.randint(0, V, (S,), generator=g, device="cuda").tolist()     # the newest token, not in the cache yet
        self.tokens = [[t] for t in self.last]
        self.g = g

    def _i32(self, x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    def project(self, tokens):
        """Queries, keys and values of a flat list of tokens, as the fused projection leaves them."""
        H, G, D = self.heads, self.group, self.dim
        x = self.embed[torch.tensor(tokens, device="cuda")]
        qkv = (x @ self.W_qkv.t()).view(len(tokens), H * G + 2 * H, D)
        return x, qkv[:, :H * G], qkv[:, H * G:H * G + H], qkv[:, H * G + H:]

    def trees(self):
        """Per sequence: tokens and parents (-1: the root) of its nodes, a parent before its children."""
        nodes = [[(t, -1)] for t in self.last]
        tip = [0] * self.S
        for _ in range(DEPTH):
            h = self.embed[torch.tensor([nodes[s][tip[s]][0] for s in range(self.S)], device="cuda")]
            _, ids, _ = ev.active_lmhead_topk(h, self.W_act, self.act_ids, WIDTH)
            for s, best in enumerate(ids.tolist()):
                parent, tip[s] = tip[s], len(nodes[s])
                nodes[s] += [(t, parent) for t in best]
        return nodes

    def step(self, temperature=0.8, top_k=50, top_p=0.95, min_p=0.02):
        """One round of drafting and verification; returns what the target saw (for a look from outside)."""
        nodes = self.trees()
        rows = [len(n) for n in nodes]
        for s, (n, r) in enumerate(zip(self.lens, rows)):
            if n + r > self.capacity:                         # (tokens past the page table are dropped, and rows would lose their places)
                raise ValueError(f"sequence {s} has {n} tokens, and {r} nodes more do not fit its {self.capacity}")
        off = [0]
        for n in rows:
            off.append(off[-1] + n)
        flat = [t for n in nodes for t, _ in n]
        bits = []
        for n in nodes:
            own = []
            for j, (_, parent) in enumerate(n):
                own.append((own[parent] if parent >= 0 else 0) | 1 << j)
            bits += own
        x, q, k, v = self.project(flat)
        starts, row_off = self._i32(self.lens), self._i32(off)
        most = max(rows)
        ev.kv_write(self.cache, k, v, self.table, starts, row_off, most)
        lens = self._i32([n + r for n, r in zip(self.lens, rows)])
        tree = torch.tensor(bits, dtype=torch.int64, device="cuda")
        out, lse = ev.kv_attention(q, self.cache, self.table, lens, row_off, most, tree=tree)
        h = x + out.reshape(len(flat), -1) @ self.W_o.t()
        logits = (h @ self.W_lm.t())
        T = logits.shape[0]
        u = torch.rand(T, generator=self.g, device="cuda")
        fill = lambda value, dtype=torch.float32: torch.full((T,), value, dtype=dtype, device="cuda")   # noqa: E731
        drawn, logprob = ev.sample(logits, u, temperature=fill(temperature), top_k=fill(top_k, torch.int32), top_p=fill(top_p),
                                   min_p=fill(min_p))
        choice = drawn.tolist()
        kept, kept_off, grown = [], [0], []
        for s, n in enumerate(nodes):
            at, path = 0, [0]
            while True:
                token = choice[off[s] + at]
                child = next((j for j, (t, parent) in enumerate(n) if parent == at and t == token), None)
                if child is None:
                    break
                path.append(child)
                at = child
            kept += [off[s] + j for j in path]
            kept_off.append(len(kept))
            grown.append([n[j][0] for j in path[1:]] + [choice[off[s] + at]])
        at = torch.tensor(kept, device="cuda")
        ev.kv_write(self.cache, k[at], v[at], self.table, starts, self._i32(kept_off), max(b - a for a, b in zip(kept_off, kept_off[1:])))
        for s, new in enumerate(grown):
            self.lens[s] += len(new)                          # the root and the accepted nodes; the last token comes next
            self.tokens[s] += new
            self.last[s] = new[-1]
        return {"q": q, "lens": lens, "row_off": off, "tree": bits, "out": out, "lse": lse, "logits": logits, "drawn": drawn,
                "logprob": logprob, "grown": grown, "max_rows": most}


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--steps", type=int, default=8)
    p.add_argument("--temperature", type=float, default=0.8)
    a = p.parse_args()
    loop = Loop()
    for i in range(a.steps):
        if max(loop.lens) + 1 + WIDTH * DEPTH > loop.capacity:
            print(f"after {i} steps: no room for another tree")
            break
        r = loop.step(temperature=a.temperature)
        print(f"step {i}: tokens per sequence {[len(x) for x in r['grown']]}, lengths {loop.lens}")
    for s, t in enumerate(loop.tokens):
        print(f"sequence {s}: {t}")


if __name__ == "__main__":
    main()
