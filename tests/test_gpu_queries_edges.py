"""Several tokens of a request on the GPU: arguments at the ends of their ranges."""
import numpy as np
import pytest
import torch

from paper_2606_31093_amd import kvx
from paper_2606_31093_amd.workloads import PoolSpec
from test_gpu_decode import error_word, tensor

pytestmark = pytest.mark.gpu

MOST = (1 << 31) - 1


# ---------------------------------------------------------------------------
# kvx_append_normed
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("off", [0, 4])
def test_record_positions_that_are_not_used(off):
    """With positions of their own, records may hold any position that is not negative; without, the last
    token's has to be below 2^31."""
    spec = PoolSpec(1, 2, 2, 64, T=16, N=8, e=2)
    x = torch.randn(20, 6, 64, device="cuda").bfloat16()
    q, k, v = x.split([2, 2, 2], dim=1)
    rope, w = kvx.Rope(torch.rand(8, device="cuda"), off), kvx.Norm(torch.rand(64, device="cuda"))
    pos = torch.arange(100, 120, dtype=torch.int32, device="cuda")

    def call(at, positions):
        pool, q_out, err = torch.zeros(spec.nbytes, dtype=torch.uint8, device="cuda"), torch.zeros_like(q), error_word()
        reqs = kvx.device_append_reqs([[0, 0, 5, at, 20]])
        kvx.kvx_append_normed(pool, spec, 0, k, v, tensor(np.arange(8, dtype=np.int32)), reqs, 20, q=q, q_out=q_out, rope=rope,
                              q_norm=w, k_norm=w, positions=positions, dev_err=err)
        return pool, q_out.view(torch.int16), int(err.item())
    want = call(0, pos)
    assert want[0].any() and want[1].any() and want[2] == 0
    for at in (7, MOST - 20, MOST - 19, MOST):
        got = call(at, pos)
        assert got[2] == 0 and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for at, positions in ((-1, pos), (-1 - MOST, pos), (MOST - 19, None), (MOST, None)):
        got = call(at, positions)
        assert got[2] == kvx.DERR_BAD_REQ and not got[0].any() and not got[1].any()
    assert call(MOST - 20, None)[2] == 0
