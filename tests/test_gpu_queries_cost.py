"""Attention of several queries under limits (max_queries, max_tokens) far above what its
records hold, as a captured call has them: it must not cost much more than under limits
that fit.  Each pair is timed in turn on the same pools, and the least times are
compared: the bounds lie between what the call takes and what it took when it was at
fault."""
import numpy as np
import pytest
import torch

from paper_2606_31093_amd import kvx
from paper_2606_31093_amd.workloads import PoolSpec
from test_gpu_cost import check, least

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("recs,fits,wide,bound", [
    # one request: a chunk (at fault 3.0) and a single token (19.8) behind a long context
    ([(0, 100000, 512)], (512, 100000), (16384, 131072), 1.5), ([(0, 131072, 1)], (1, 131072), (16384, 131072), 5.0),
    # short requests: whole prompts (24 and 380), single tokens (124)
    ([(0, 256, 256)] * 32, (256, 256), (1 << 16, 512), 2.5), ([(0, 256, 256)] * 32, (256, 256), (1 << 20, 512), 2.5),
    ([(0, 256, 1)] * 32, (256, 256), (1 << 16, 512), 5.0), ([(0, 1000, 1000)] * 4, (1000, 1000), (1 << 20, 1024), 2.0),
])
def test_limits_far_above_the_records(recs, fits, wide, bound):
    pages = sum(-(-r[1] // 64) for r in recs)
    spec = PoolSpec(1, 2, 8, 128, T=64, N=pages + 1, e=2)
    pool = torch.randn(spec.elems, device="cuda").bfloat16().view(torch.uint8)
    pt = torch.randperm(pages, device="cuda").int()
    off = np.concatenate([[0], np.cumsum([-(-r[1] // 64) for r in recs])[:-1]])
    row = np.concatenate([[0], np.cumsum([r[2] for r in recs])])
    q = torch.randn(int(row[-1]), 32, 128, device="cuda").bfloat16()
    out = torch.zeros_like(q)
    reqs = kvx.device_queries_reqs([(off[i], row[i], *r, 0) for i, r in enumerate(recs)])

    def call(most_q, most):
        ws = kvx.queries_workspace(spec, len(recs), 32, most_q, most)
        return lambda: kvx.kvx_attend_prompt(q, out, pool, spec, 0, pt, reqs, most_q, most, ws)
    a, b = least(call(*wide), call(*fits), rounds=5, reps=5)
    check(a / b, bound, f"{len(recs)} x {recs[0]} under {wide}, {a:.1f} us, under {fits} {b:.1f}")
