"""Several tokens of a request on the GPU: arguments and values at the ends of their ranges, against
definitions in 64 bits (np_queries).  Bounds as in test_gpu_queries.py."""
import numpy as np
import pytest
import torch

import np_decode
import np_queries as ref
import test_gpu_queries as base
from paper_2606_31093_amd import kvx
from paper_2606_31093_amd.workloads import PoolSpec
from test_gpu_decode import U, error_word, rows_tensor, rows_values, tensor

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


# rows of about 2^e, with one element of 2^one among them (None: none), and the norm's eps
SIZES = [(66, None, 0.0), (126, None, 1e-6), (126, None, 0.0), (0, 70, 0.0), (0, 100, 1e-5), (-64, None, 0.0), (-70, None, 0.0),
         (-126, None, 0.0), (-132, None, 0.0), (-70, None, 1e-44), (-120, None, 1e-33), (-30, None, 1e-20), (-63, None, 1e-12),
         (-39, None, 0.0), (-41, None, 0.0), (100, None, 3e38), (63, None, 0.0), (64, None, 1e-6)]


@pytest.mark.parametrize("rot,off,inter", [(64, 0, False), (64, 0, True), (20, 4, False), (0, 0, False)])
@pytest.mark.parametrize("D,q_norm", [(64, (0, 64)), (256, (0, 256)), (128, (64, 64))])
def test_norms_of_large_and_small_rows(D, q_norm, rot, off, inter):
    """bfloat16 rows whose elements' squares overflow 32 bits, vanish in them, or vanish beside eps.  Rounding to
    bfloat16 is off by 2^-134 at least; an element more than 2^-126 of the largest below it may lose digits."""
    rng = np.random.default_rng(D + rot)
    spec = PoolSpec(1, 2, 1, D, T=16, N=4, e=2)
    n, u = len(SIZES), U["bf16"]
    x = np.ldexp(rng.uniform(0.75, 1.5, (n, 3, D)) * rng.choice([-1, 1], (n, 3, D)), np.array([s[0] for s in SIZES])[:, None, None])
    for r, (_, one, _) in enumerate(SIZES):
        if one is not None:
            x[r, :, q_norm[0] + 5] = 2.0 ** one
    xb = np_decode.bits(x.astype(np.float32), "bf16")
    x = np_decode.values(xb, "bf16")
    weight = (rng.random(q_norm[1]) + 0.5).astype(np.float32)
    freq = (10000.0 ** (-np.arange(rot // 2) * 2 / max(rot, 1))).astype(np.float32)
    xt = rows_tensor(xb, "bf16")
    q, k, v = xt[:, :1], xt[:, 1:2], xt[:, 2:]
    pool, q_out, err = torch.zeros(spec.nbytes, dtype=torch.uint8, device="cuda"), torch.zeros_like(q), error_word()
    for r, (_, _, eps) in enumerate(SIZES):
        w = kvx.Norm(tensor(weight), q_norm[0], eps)
        kvx.kvx_append_normed(pool, spec, 0, k, v, tensor(np.arange(4, dtype=np.int32)), kvx.device_append_reqs([[0, r, r, r, 1]]), 1,
                              q=q, q_out=q_out, rope=kvx.Rope(tensor(freq), off, inter) if rot else None, q_norm=w, k_norm=w,
                              dev_err=err)
    assert int(err.item()) == 0
    got_q = rows_values(q_out, "bf16")
    got_k = np_decode.values(np_decode.canonical(pool.cpu().numpy(), spec)[0, np.arange(n) // 16, 0, np.arange(n) % 16], "bf16")
    for r, (_, _, eps) in enumerate(SIZES):
        eps = float(np.float32(eps))
        y = ref.norm(x[r, :2], weight.astype(np.float64), q_norm[0], eps)
        # elements that are normed and not rotated, and pairs of normed ones
        tol = (D / 2 + 6) * 2.0 ** -24 * np.abs(y)
        for j in range(rot // 2):
            a, b = (off + 2 * j, off + 2 * j + 1) if inter else (off + j, off + j + rot // 2)
            size = (np.abs(y[:, a]) + np.abs(y[:, b]))[:, None]
            tol[:, [a, b]] = np.maximum(tol[:, [a, b]], (D / 2 + 6) * 2.0 ** -24 * size) + 2.0 ** -20 * size
        z = ref.rotate(y, np.full(rot // 2, r), freq, off, inter, 1.0)
        fits = np.abs(z) < 3.3e38                    # the rest overflows, in the formula too
        got = np.stack([got_q[r, 0], got_k[r, 0]])
        bound = np.maximum(u * np.abs(z), 2.0 ** -134) + (1 + u) * tol + 2.0 ** -126 * np.abs(y).max()
        assert np.isfinite(got[fits]).all() and (np.abs(got - z)[fits] <= bound[fits]).all(), (r, SIZES[r])


@pytest.mark.parametrize("inter,off", [(False, 0), (True, 0), (False, 4)])
def test_norms_of_zeros_and_what_is_not_finite(inter, off):
    """Rows of zeros without eps (0 / 0), with eps, and with an infinity (0 beside it) or a NaN."""
    spec = PoolSpec(1, 2, 1, 64, T=16, N=4, e=2)
    x = torch.ones(5, 3, 64, device="cuda").bfloat16()
    x[0], x[1], x[2, :, 50], x[3, :, 50], x[4, :, 50] = 0, 0, float("inf"), float("nan"), -float("inf")
    q, k, v = x.split([1, 1, 1], dim=1)
    pool, q_out = torch.zeros(spec.nbytes, dtype=torch.uint8, device="cuda"), torch.full_like(q, 7)
    for r, eps in enumerate((0.0, 1e-30, 0.0, 1e-6, 1e-6)):
        w = kvx.Norm(None, 0, eps, 64)
        kvx.kvx_append_normed(pool, spec, 0, k, v, tensor(np.arange(4, dtype=np.int32)), kvx.device_append_reqs([[0, r, r, 0, 1]]), 1,
                              q=q, q_out=q_out, rope=kvx.Rope(torch.zeros(8, device="cuda"), off, inter), q_norm=w, k_norm=w)
    got_k = pool.view(torch.bfloat16).view(4, 2, 16, 64)[0, 0, :5]
    for got in (q_out[:, 0].float(), got_k.float()):
        assert torch.isnan(got[0]).all() and (got[1] == 0).all() and torch.isnan(got[3]).all()
        for r in (2, 4):
            assert torch.isnan(got[r, 50]) and (got[r, :50] == 0).all() and (got[r, 51:] == 0).all()


# ---------------------------------------------------------------------------
# kvx_attend_prompt, kvx_attend_tree
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("kind,cache", base.TYPES)
@pytest.mark.parametrize("D,G", [(64, 4), (128, 7), (256, 2)])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("scale,size", [(2.0 ** 13, 2.0 ** -14), (2.0 ** 17, 2.0 ** -17), (2.0 ** -12, 16.0), (3.0, 0.25)])
def test_bias_under_large_and_small_scales(scale, size, tree, D, G, kind, cache):
    """A bias keeps its digits whatever the scale makes of the products: slopes are small beside a large one,
    large beside a small one."""
    spec = PoolSpec(1, 2, 1, D, T=16, N=60, e=1 if cache == "e4m3" else 2)
    recs = [(0, 300, 64, 0), (0, 130, 40, 0), (3, 90, 60, 0)]
    base.queries_case(3, spec, kind, cache, recs, G, scale=scale, slopes=True, size=size, tree=tree)
    base.queries_case(4, spec, kind, cache, [(0, 260, 2, 0), (7, 90, 1, 0)], G, scale=scale, slopes=True, size=size, tree=tree)
