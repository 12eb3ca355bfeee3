"""Decoding with a bounded paged cache: append, attend, select, move.

A few sequences are decoded token by token through a small model's attention
layers (random projections stand in for the rest of the model).  Every step
rotates and appends the new tokens' keys and values, attends over the pages and
adds up what each cached position contributes.  A sequence that reaches its
limit is cut back to its budget: each layer and head keeps the first positions,
the newest ones and those of the largest accumulated weight, moved into fresh
pages; the old pages return to the free list.

    python examples/decode_step.py
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


class Sequences:
    """The pages, lengths and accumulated weights of a batch of sequences."""

    def __init__(self, spec, n, q_heads, budget, limit, device):
        self.spec, self.n, self.q_heads, self.budget, self.limit = spec, n, q_heads, budget, limit
        self.device = device
        self.pool = torch.zeros(spec.nbytes, dtype=torch.uint8, device=device)
        self.free = list(range(spec.N))
        self.slots_per = -(-limit // spec.T)                  # table entries of a sequence
        self.pages = [[] for _ in range(n)]
        self.length = [0] * n                                 # positions in the cache
        self.position = [0] * n                               # tokens seen: rotation goes on after an eviction
        self.acc = torch.zeros(n, spec.L, spec.H, limit, device=device)
        self.err = torch.zeros(1, dtype=torch.int32, device=device)
        freq, amplitude = kvx.rope_frequencies(spec.D, factor=4.0, scaling="ramp", trained=4096)
        self.rope = kvx.Rope(torch.from_numpy(freq).to(device), amplitude=amplitude)
        self.workspace = kvx.attend_workspace(spec, n, q_heads, limit, accumulate=True, device=device)

    def table(self, lists):
        t = np.zeros((self.n, self.slots_per), np.int32)
        for r, pages in enumerate(lists):
            t[r, :len(pages)] = pages
        return torch.from_numpy(t.reshape(-1)).to(self.device)

    def begin_step(self):
        """A slot for every sequence's new token; the step's table and records."""
        spec = self.spec
        for r in range(self.n):
            if self.length[r] == len(self.pages[r]) * spec.T:
                self.pages[r].append(self.free.pop())
        new = [[r * self.slots_per, r, self.length[r], self.position[r], 1] for r in range(self.n)]
        per_seq = spec.L * spec.H * self.limit
        seen = [[r * self.slots_per, r * per_seq, 0, self.length[r] + 1] for r in range(self.n)]
        self.pt = self.table(self.pages)
        self.append_reqs = kvx.device_append_reqs(new, self.device)
        self.attend_reqs = kvx.device_attend_reqs(seen, self.device)
        for r in range(self.n):
            self.length[r] += 1
            self.position[r] += 1

    def layer(self, layer, q, k, v):
        """Attention of one layer: the new tokens' outputs."""
        spec = self.spec
        q_rot, out = torch.empty_like(q), torch.empty_like(q)
        kvx.kvx_append(self.pool, spec, layer, k, v, self.pt, self.append_reqs, 1, q=q, q_out=q_rot, rope=self.rope,
                       dev_err=self.err)
        # the layer's accumulators of sequence 0; the records' offsets lead to the others'
        acc = self.acc.view(-1)[layer * spec.H * self.limit:]
        kvx.kvx_attend(q_rot, out, self.pool, spec, layer, self.pt, self.attend_reqs, max(self.length), self.workspace,
                       acc=acc, acc_stride=self.limit, dev_err=self.err)
        return out

    def evict(self, sink=4, recent=32):
        """Cuts the sequences that have reached the limit back to the budget;
        returns the pages freed."""
        full = [r for r in range(self.n) if self.length[r] == self.limit]
        if not full:
            return 0
        spec, lists, keep = self.spec, self.spec.L * self.spec.H, self.budget
        fresh = [[self.free.pop() for _ in range(-(-keep // spec.T))] if r in full else [] for r in range(self.n)]
        kept = torch.empty(len(full), lists, keep, dtype=torch.int32, device=self.device)
        left = torch.empty(len(full), lists, keep, device=self.device)
        choose = [[r * lists * self.limit, i * lists * keep, i * lists * keep, self.limit, keep, sink, recent]
                  for i, r in enumerate(full)]
        move = [[r * self.slots_per, r * self.slots_per, i * lists * keep, 0, 0, keep] for i, r in enumerate(full)]
        kvx.kvx_select_kept(self.acc, self.limit, lists, kvx.device_select_reqs(choose, self.device), self.limit, kept,
                            keep, left, keep, self.err)
        kvx.kvx_transfer_kept(self.pool, spec, self.pool, spec, self.pt, self.table(fresh),
                              kvx.device_reqs(move, self.device), keep, kept, keep, dev_err=self.err)
        freed = 0
        for i, r in enumerate(full):
            self.acc[r].zero_()
            self.acc[r, :, :, :keep] = left[i].view(spec.L, spec.H, keep)
            freed += len(self.pages[r]) - len(fresh[r])
            self.free += self.pages[r]
            self.pages[r], self.length[r] = fresh[r], keep
        return freed


def run(steps=400, n=3, budget=128, limit=192, verbose=True, device="cuda"):
    """Decodes ``steps`` tokens of ``n`` sequences; returns the sequences and the
    last step's outputs [layer][sequence, head, head_dim]."""
    spec = PoolSpec(L=3, C=2, H=2, D=128, T=64, N=n * (-(-limit // 64) + -(-budget // 64)) + 2, e=2, layout="LPCTHD")
    q_heads, width = 8, 256
    s = Sequences(spec, n, q_heads, budget, limit, device)
    g = torch.Generator(device=device)
    g.manual_seed(1)
    heads = q_heads + 2 * spec.H
    weights = torch.randn(spec.L, width, heads * spec.D, generator=g, device=device) / width ** 0.5
    outs = []
    for step in range(steps):
        s.begin_step()
        x = torch.randn(n, width, generator=g, device=device)
        outs = []
        for layer in range(spec.L):
            rows = (x @ weights[layer]).to(torch.bfloat16).view(n, heads, spec.D)
            q, k, v = rows.split([q_heads, spec.H, spec.H], dim=1)
            outs.append(s.layer(layer, q, k, v))
        freed = s.evict()
        if freed and verbose:
            print(f"token {step + 1}: every layer and head keeps {budget} of {limit} positions, {freed} pages freed",
                  flush=True)
    torch.cuda.synchronize()
    if int(s.err.item()):
        raise RuntimeError(f"device error bits {int(s.err.item())}")
    return s, outs


if __name__ == "__main__":
    seqs, _ = run()
    print(f"{seqs.position[0]} tokens decoded, {seqs.length[0]} positions held, {len(seqs.free)} of {seqs.spec.N} "
          "pages free")
