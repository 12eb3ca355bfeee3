"""Several tokens of a request on the GPU: arguments and values at the ends of their ranges, against
definitions in 64 bits (np_queries); limits far above what the records hold.  Bounds
as in test_gpu_queries.py."""
import numpy as np
import pytest
import torch

import np_decode
import np_queries as ref
import test_gpu_queries as base
import test_gpu_queries_forms as forms
from paper_2606_31093_amd import kvx
from paper_2606_31093_amd.workloads import PoolSpec
from test_gpu_decode import U, error_word, rows_tensor, rows_values, tensor
from test_gpu_queries_forms import several_launches  # noqa: F401

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


@pytest.mark.parametrize("off", [0, 3])
def test_most_heads(off):
    """A token of 2^26 elements, the most, in heads of 8."""
    H = 1 << 22
    spec = PoolSpec(1, 2, H, 8, T=1, N=2, e=2)
    x = torch.ones(1, 2 * H, 8, device="cuda").bfloat16()
    pool, err = torch.zeros(spec.nbytes, dtype=torch.uint8, device="cuda"), error_word()
    kvx.kvx_append_normed(pool, spec, 0, x[:, :H] * 4, x[:, H:] * 3, tensor(np.array([1], np.int32)),
                          kvx.device_append_reqs([[0, 0, 0, 0, 1]]), 1, rope=kvx.Rope(torch.zeros(1, device="cuda"), off),
                          k_norm=kvx.Norm(torch.full((8,), 2.0, device="cuda"), 0, 0.0), dev_err=err)
    got = pool.view(torch.bfloat16).view(2, 2, H, 8)
    assert int(err.item()) == 0 and not got[0].any() and (got[1, 0] == 2).all() and (got[1, 1] == 3).all()


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


ONE = [
    # (H, G, D, C, v, record, max_queries, max_tokens, more).  Few blocks under limits of many; as many as have a
    # workgroup each, exactly and under wider limits; more than there are workgroups; one less than that many
    (8, 4, 128, 2, 0, (0, 3000, 40, 0), 16384, 20000, {}), (8, 4, 128, 2, 0, (5, 3000, 1, 0), 1 << 22, 1 << 22, {}),
    (256, 1, 64, 2, 0, (0, 1100, 1024, 0), 1024, 1100, {}), (256, 1, 64, 2, 0, (0, 1100, 1024, 7), 9000, 70000, {}),
    (256, 1, 64, 2, 0, (0, 2304, 2304, 0), 2304, 2304, {}), (256, 1, 64, 2, 0, (0, 1500, 768, 0), 4096, 4096, {}),
    (128, 2, 128, 2, 0, (0, 1200, 1100, 0), 1100, 1200, dict(slopes=True)), (64, 2, 256, 2, 0, (0, 1100, 1024, 0), 1024, 1100, dict(cap=30.0)),
    (64, 2, 256, 2, 0, (0, 1100, 90, 0), 1024, 1100, dict(window=77)), (1, 16, 576, 1, 512, (0, 900, 60, 0), 1 << 20, 5000, {}),
    (8, 4, 128, 2, 0, (0, 3000, 60, 0), 1 << 20, 5000, dict(tree=True)), (8, 1, 128, 2, 0, (0, 64, 0, 0), 1 << 20, 5000, {}),
]


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("H,G,D,C,v,rec,most_q,most,more", ONE)
def test_one_record_under_wide_limits(H, G, D, C, v, rec, most_q, most, more, cache):
    """What the record holds, not the limits, says whether every block has a workgroup of its own."""
    spec = PoolSpec(1, C, H, D, T=64, N=-(-rec[1] // 64) + 2, e=1 if cache == "e4m3" else 2)
    forms.large_case(1, spec, "bf16", cache, [rec], G, v or None, max_queries=most_q, max_tokens=most, **more)


@pytest.mark.parametrize("H,G,D,rec,most_q,most", [(256, 1, 64, (0, 1500, 1100, 0), 1100, 1500), (8, 4, 128, (0, 900, 30, 0), 1 << 20, 5000)])
def test_one_record_in_launches_of_few(several_launches, H, G, D, rec, most_q, most):
    """At most 1024 workgroups a launch."""
    spec = PoolSpec(1, 2, H, D, T=64, N=40, e=2)
    forms.large_case(2, spec, "bf16", "bf16", [rec], G, max_queries=most_q, max_tokens=most)


@pytest.mark.parametrize("limits", [(256, 300), (100000, 400), (1 << 20, 512), (4096, 1000)])
def test_many_records_under_wide_limits(limits):
    """Short records, up to as many workgroups as they may need and with far more than that."""
    spec = PoolSpec(1, 2, 4, 128, T=16, N=500, e=2)
    recs = [(r % 3, 3 + 7 * r, 1 + 5 * r, 0) for r in range(40)]
    forms.large_case(3, spec, "bf16", "bf16", recs, 4, max_queries=limits[0], max_tokens=limits[1])


def test_malformed_record_under_wide_limits():
    spec = PoolSpec(1, 2, 64, 64, T=16, N=40, e=2)
    pool, pt = torch.zeros(spec.nbytes, dtype=torch.uint8, device="cuda"), tensor(np.arange(40, dtype=np.int32))
    q = torch.randn(600, 64, 64, device="cuda").bfloat16()
    ws = kvx.queries_workspace(spec, 1, 64, 1 << 20, 600)
    for rec in ((0, 0, 0, 601, 600, 0), (0, 1, 0, 600, 600, 0), (0, 0, 5, 4, 1, 0), (-1, 0, 0, 600, 600, 0)):
        out, err = torch.full_like(q, 7), error_word()
        kvx.kvx_attend_prompt(q, out, pool, spec, 0, pt, kvx.device_queries_reqs([rec]), 1 << 20, 600, ws, dev_err=err)
        assert int(err.item()) == kvx.DERR_BAD_REQ and (out == 7).all()


def test_graph_of_other_lengths():
    """One captured call, replayed for records that take either division and for a malformed one, with eager
    calls in between: outputs by the definition, and equal bits of equal calls."""
    spec = PoolSpec(1, 2, 128, 64, T=64, N=60, e=2)
    H, D, most_q, most = spec.H, spec.D, 2500, 3500
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    pool = torch.randn(spec.elems, generator=g, device="cuda").bfloat16().view(torch.uint8)
    pt = torch.randperm(60, generator=g, device="cuda").int()
    q = torch.randn(most_q, H, D, generator=g, device="cuda").bfloat16()
    out, lse, err = torch.zeros_like(q), torch.zeros(most_q, H, device="cuda"), error_word()
    reqs = kvx.device_queries_reqs([(0, 0, 0, 1, 1, 0)])
    ws = kvx.queries_workspace(spec, 1, H, most_q, most)

    def call():
        kvx.kvx_attend_prompt(q, out, pool, spec, 0, pt, reqs, most_q, most, ws, lse=lse, dev_err=err)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    values = forms.cache_of(pool, spec, "bf16")[0]
    u = U["bf16"]
    for rec in [(0, 0, 0, 3400, 1, 0), (0, 0, 0, 2500, 2500, 0), (0, 5, 0, 3000, 2, 0), (0, 0, 0, 3501, 5, 0), (0, 100, 0, 2300, 2048, 0),
                (0, 0, 100, 3300, 1800, 0)]:
        reqs.copy_(kvx.device_queries_reqs([rec]))
        bad = rec[3] > most
        w_out, w_lse, mag, dots, size = (None,) * 5 if bad else forms.exact(q, values, spec, pt, rec, D ** -0.5, D, None, 0.0, None, 0, None)
        seen = []
        for turn in range(4):
            out.fill_(7), lse.fill_(7), ws.fill_(0xff), err.zero_()
            torch.cuda.synchronize()
            graph.replay() if turn % 2 == 0 else call()
            torch.cuda.synchronize()
            assert int(err.item()) == (kvx.DERR_BAD_REQ if bad else 0)
            mine = torch.zeros(most_q, dtype=torch.bool, device="cuda")
            if not bad:
                mine[rec[1]:rec[1] + rec[4]] = True
            assert (out[~mine] == 7).all() and (lse[~mine] == 7).all()
            seen.append((out.clone(), lse.clone()))
            assert torch.equal(out, seen[0][0]) and torch.equal(lse, seen[0][1])
        if not bad:
            ds = (D + 8) * 2.0 ** -24 * dots + 2.0 ** -21 * size
            tol = u * w_out.abs() + (1 + u) * (u + 2 * ds + 2.0 ** -20)[..., None] * mag
            assert ((out[mine].double() - w_out).abs() <= tol).all(), rec
            assert ((lse[mine].double() - w_lse).abs() <= ds + 2.0 ** -20 * (1 + w_lse.abs())).all(), rec


# ---------------------------------------------------------------------------
# divisions of the work, held to the definition
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("n", [1, 40, 300])
def test_split_records_among_malformed_ones(n):
    """Records whose units lie in several shares, alone and among malformed ones, which move the shares: each
    within the definition's bound.  In these sizes 32 positions that are lost or counted twice exceed it in 99 of
    100 rows, an eighth of the positions in all, at three of four values."""
    spec = PoolSpec(1, 2, 2, 128, T=64, N=100, e=2)
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    pool = torch.randn(spec.elems, generator=g, device="cuda").bfloat16().view(torch.uint8)
    pt = torch.randperm(100, generator=g, device="cuda").int()
    q = torch.randn(1000, 8, 128, generator=g, device="cuda").bfloat16()
    values, u = forms.cache_of(pool, spec, "bf16")[0], U["bf16"]
    good = [(0, 0, 0, 3000, n, 0), (50, 500, 10, 2000, n, 0)]
    want = [forms.exact(q, values, spec, pt, rec, 128 ** -0.5, 128, None, 0.0, None, 0, None) for rec in good]
    for recs in (good, [(0, 998, 0, 3000, 5, 0), good[0], (0, 0, 0, 3001, 1, 0), (0, 0, 5, 4, 1, 0), good[1], (0, 0, 0, 9, 10, 0)]):
        out, lse = torch.full_like(q, 7), torch.full((1000, 8), 7.0, device="cuda")
        ws = kvx.queries_workspace(spec, len(recs), 8, n, 3000)
        kvx.kvx_attend_prompt(q, out, pool, spec, 0, pt, kvx.device_queries_reqs(recs), n, 3000, ws, lse=lse)
        for rec, (w_out, w_lse, mag, dots, size) in zip(good, want):
            mine = slice(rec[1], rec[1] + n)
            ds = (128 + 8) * 2.0 ** -24 * dots + 2.0 ** -21 * size
            tol = u * w_out.abs() + (1 + u) * (u + 2 * ds + 2.0 ** -20)[..., None] * mag
            assert ((out[mine].double() - w_out).abs() <= tol).all(), (rec, len(recs))
            assert ((lse[mine].double() - w_lse).abs() <= ds + 2.0 ** -20 * (1 + w_lse.abs())).all(), (rec, len(recs))


def test_verified_drafts_and_decoding_within_their_bounds():
    """The example's accepted drafts against their tokens decoded in order: two results of one definition, each off by
    its bound.  That takes sum w |v|, which the same calls give for values without their signs."""
    import verify_drafts as ex
    m, kept, length, (outs, paths, first, before) = ex.run(verbose=False)
    rows = torch.cat(kept, dim=1)
    plain = rows.clone()
    plain[:, :, m.q_heads + m.spec.H:] = plain[:, :, m.q_heads + m.spec.H:].abs()
    sides = []
    for r in (rows, plain):
        fresh = ex.Model(m.n, 200 + 12 * 24)
        fresh.pt = m.pt
        sides.append(fresh.forward(r, [0] * m.n, length, [i for n in length for i in range(n)]))
    D, u, cap = m.spec.D, U["bf16"], m.scores.cap
    # a normed row's length is at most its largest factor (1.5) times the root of D, so that sum |q k| scale is at
    # most 2.25 D / sqrt D; scores lie below the cap
    ds = (D + 8) * 2.0 ** -24 * 2.25 * D ** 0.5 * 1.02 + 2.0 ** -20 * cap + 2.0 ** -21 * cap
    start = 0
    for r, n in enumerate(length):
        for layer in range(m.spec.L):
            got = outs[layer][torch.tensor(paths[r], device="cuda") + first[r]].double()
            want, mag = (x[layer][start + before[r]:start + before[r] + len(paths[r])].double() for x in sides)
            mag = mag / (1 - u) * (1 + 2 * (u + 2 * ds + 2.0 ** -20))          # itself off by its bound
            tol = u * (got.abs() + want.abs()) / (1 - u) + 2 * (1 + u) * (u + 2 * ds + 2.0 ** -20) * mag
            assert ((got - want).abs() <= tol).all()
        start += n


# ---------------------------------------------------------------------------
# shapes
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("C,H,D,G,v", [(2, 3, 8, 1, 0), (2, 2, 24, 5, 0), (2, 6, 72, 2, 0), (2, 1, 136, 3, 0), (2, 4, 200, 1, 0), (2, 1, 248, 9, 0),
                                       (2, 2, 264, 2, 0), (2, 1, 512, 1, 0), (1, 1, 520, 40, 8), (1, 3, 264, 2, 256), (1, 1, 136, 1, 136),
                                       (2, 1, 16, 200, 0)])
def test_head_sizes(C, H, D, G, v, kind):
    """Multiples of 8 that no kernel is made for, few and many query heads of a cache head."""
    spec = PoolSpec(1, C, H, D, T=16, N=60, e=2, layout="LPCTHD" if G % 2 else "PLCHTD")
    recs = [(0, 70, 40, 0), (0, 1, 1, 0), (3, 129, 5, 0), (0, 33, 33, 20), (5, 5, 1, 0), (40, 64, 30, 0)]
    base.queries_case(D, spec, kind, kind, recs, G, v or None, spoil=True, gap=1, cap=9.0 if D % 3 else 0.0, slopes=D % 16 == 8)
    base.queries_case(D, spec, kind, kind, [(0, 150, 1, 0), (7, 64, 1, 0)], G, v or None, spoil=True, strided=True)
    base.queries_case(D, spec, kind, kind, [(0, 150, 12, 0), (9, 64, 30, 0)], G, v or None, spoil=True, tree=True)
