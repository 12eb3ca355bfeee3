"""Decoding with drafted trees over a paged cache: prompts in chunks, drafts
verified together, accepted paths kept.

A few sequences run through a small model's attention layers (random projections
stand in for the rest of the model).  The prompt goes in by chunks: every chunk's
queries and keys are normed per head and rotated, its keys and values appended, its
queries attend.  Then every step drafts a tree of tokens for each sequence, appends
them all, each at its depth's position, and attends with all of them at once, each
seeing the cache and its own ancestors.  What is accepted of a tree (here a path
drawn at random; a model compares its own choices with the drafts) is moved to the
front of the drafts' slots, in every layer; the others are written over by the
next step.

    python examples/verify_drafts.py
"""
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2606_31093_amd import kvx                          # noqa: E402
from paper_2606_31093_amd.workloads import PoolSpec           # noqa: E402


def draft_tree(rng, n):
    """Parents of n drafted tokens (-1: the last token of the cache), each later than its own."""
    return [-1] + [int(rng.integers(max(0, j - 4), j)) for j in range(1, n)]


def ancestors(parents):
    """Of each draft the bits of its ancestors and itself."""
    bits = []
    for j, p in enumerate(parents):
        bits.append((1 << j) | (bits[p] if p >= 0 else 0))
    return bits


def path_to(parents, j):
    out = []
    while j >= 0:
        out.append(j)
        j = parents[j]
    return out[::-1]


class Model:
    """The attention layers of a small model over one pool."""

    def __init__(self, n, limit, q_heads=8, width=256, device="cuda", layers=3):
        self.spec = PoolSpec(L=layers, C=2, H=2, D=128, T=16, N=n * -(-limit // 16) + 3, e=2, layout="LPCTHD")
        self.n, self.q_heads, self.device, self.width = n, q_heads, device, width
        spec, g = self.spec, torch.Generator(device=device)
        g.manual_seed(1)
        self.pool = torch.zeros(spec.nbytes, dtype=torch.uint8, device=device)
        self.slots_per = -(-limit // spec.T)
        pages = np.random.default_rng(2).permutation(spec.N)[:n * self.slots_per].astype(np.int32)
        self.pt = torch.from_numpy(pages).to(device)
        self.err = torch.zeros(1, dtype=torch.int32, device=device)
        heads = q_heads + 2 * spec.H
        self.weights = torch.randn(spec.L, width, heads * spec.D, generator=g, device=device) / width ** 0.5
        freq, amplitude = kvx.rope_frequencies(spec.D)
        self.rope = kvx.Rope(torch.from_numpy(freq).to(device), amplitude=amplitude)
        self.q_norm, self.k_norm = (kvx.Norm(torch.rand(spec.D, generator=g, device=device) + 0.5) for _ in range(2))
        self.scores = kvx.Scores(cap=30.0)
        self.workspace = kvx.queries_workspace(spec, n, q_heads, max(64, limit), limit, device=device)

    def project(self, x):
        """Queries, keys and values side by side, [layer, rows, heads, head_dim], of embeddings x [rows, width]."""
        rows = torch.stack([x @ w for w in self.weights]).to(torch.bfloat16)
        return rows.view(len(self.weights), len(x), -1, self.spec.D)

    def forward(self, rows, length, counts, positions, bits=None):
        """Every layer's outputs for new tokens' rows (project): counts[r] of them for sequence r, behind its
        length[r] positions; bits: they are drafts that form trees."""
        spec, dev = self.spec, self.device
        first = np.concatenate([[0], np.cumsum(counts)[:-1]]).astype(int)
        append = kvx.device_append_reqs([[r * self.slots_per, first[r], length[r], 0, counts[r]] for r in range(self.n)], dev)
        seen = kvx.device_queries_reqs([[r * self.slots_per, first[r], 0, length[r] + counts[r], counts[r], 0]
                                        for r in range(self.n)], dev)
        at = torch.tensor(positions, dtype=torch.int32, device=dev)
        tree = None if bits is None else torch.from_numpy(np.array(bits, np.uint64).view(np.int64)).to(dev)
        most, longest, outs = max(counts), max(a + b for a, b in zip(length, counts)), []
        for layer in range(spec.L):
            q, k, v = rows[layer].split([self.q_heads, spec.H, spec.H], dim=1)
            q_rot, out = torch.empty_like(q), torch.empty_like(q)
            kvx.kvx_append_normed(self.pool, spec, layer, k, v, self.pt, append, most, q=q, q_out=q_rot, rope=self.rope,
                                  q_norm=self.q_norm, k_norm=self.k_norm, positions=at, dev_err=self.err)
            args = (most, longest, self.workspace)
            if tree is None:
                kvx.kvx_attend_prompt(q_rot, out, self.pool, spec, layer, self.pt, seen, *args, scores=self.scores,
                                      dev_err=self.err)
            else:
                kvx.kvx_attend_tree(q_rot, out, self.pool, spec, layer, self.pt, seen, tree, *args, scores=self.scores,
                                    dev_err=self.err)
            outs.append(out)
        return outs

    def keep(self, length, paths):
        """Accepted drafts to the front of the drafts' slots, in every layer."""
        first = np.concatenate([[0], np.cumsum([len(p) for p in paths])]).astype(int)
        reqs = kvx.device_path_reqs([[r * self.slots_per, first[r], length[r], len(p)] for r, p in enumerate(paths)],
                                    self.device)
        path = torch.tensor([j for p in paths for j in p], dtype=torch.int32, device=self.device)
        kvx.kvx_keep_path(self.pool, self.spec, self.pt, reqs, max(len(p) for p in paths), path, dev_err=self.err)


def run(n=3, prompt=200, chunk=64, steps=12, drafts=24, verbose=True, device="cuda"):
    """Returns the model, each sequence's kept rows [layer, length, heads, head_dim], the lengths, and of the last step
    the outputs [layer][rows, q heads, head_dim], each sequence's path, first row and length before it."""
    limit = prompt + steps * drafts
    m, rng = Model(n, limit, device=device), np.random.default_rng(3)
    g = torch.Generator(device=device)
    g.manual_seed(4)

    def tokens(count):                 # embeddings, in the place of a model's, projected
        return m.project(torch.randn(count, m.width, generator=g, device=device))
    length, kept, last = [0] * n, [[] for _ in range(n)], None
    for at in range(0, prompt, chunk):
        count = min(chunk, prompt - at)
        rows = tokens(n * count)
        m.forward(rows, length, [count] * n, [at + i for _ in range(n) for i in range(count)])
        for r in range(n):
            kept[r].append(rows[:, r * count:(r + 1) * count])
            length[r] += count
    for step in range(steps):
        trees = [draft_tree(rng, drafts) for _ in range(n)]
        rows = tokens(n * drafts)
        depth = [[len(path_to(t, j)) - 1 for j in range(drafts)] for t in trees]
        outs = m.forward(rows, length, [drafts] * n, [length[r] + d for r in range(n) for d in depth[r]],
                         [b for t in trees for b in ancestors(t)])
        paths = [path_to(t, int(rng.integers(0, drafts))) for t in trees]
        m.keep(length, paths)
        last = outs, paths, [r * drafts for r in range(n)], list(length)
        for r, p in enumerate(paths):
            kept[r].append(rows[:, torch.tensor(p, device=device) + r * drafts])
            length[r] += len(p)
        if verbose:
            print(f"step {step + 1}: {[len(p) for p in paths]} of {drafts} drafts accepted, lengths {length}", flush=True)
    torch.cuda.synchronize()
    if int(m.err.item()):
        raise RuntimeError(f"device error bits {int(m.err.item())}")
    return m, [torch.cat(x, dim=1) for x in kept], length, last


if __name__ == "__main__":
    run()
