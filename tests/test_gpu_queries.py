"""Several tokens of a request over a paged cache on the GPU (kvx_append_normed,
kvx_attend_prompt, kvx_attend_tree, kvx_keep_path) against the definitions in 64
bits (np_queries), at the sizes, masks and strides where kernels go wrong.

Bounds.  u is the unit roundoff of the rows' type, half its epsilon.
- A norm's sum of D squares in 32 bits is off by at most D 2^-24 of itself, its root
  by half of that, and quotient, root and two products add 2^-24 each: (D / 2 + 6)
  2^-24 of a normed value.  A rotation adds 2^-20 A (|a| + |b|) as kvx_append's, the
  stored type its rounding: u of the value, in half below 2^-14, where values are 2^-24
  apart, 2^-25.
- A score's sum of D products is off by at most (D + 8) 2^-24 sum |q k| scale.  Its cap
  is 1 - 2 / (1 + e^2x), whose exponential and reciprocal are good to 2^-22: 2 cap
  2^-22 more, 2^-20 cap with the products' roundings.  Factors, bias and the difference
  to the maximum are each rounded to 2^-24 of at most |s| + bias: 2^-21 of it.  Call the
  sum ds; with the weights' own 2^-20 and their rounding to the rows' type, out is off
  by u |out| + (u + 2 ds + 2^-20) sum w |v|, lse by ds + 2^-20 (1 + |lse|).
- What is moved is exact."""
import numpy as np
import pytest
import torch

import np_decode
import np_queries as ref
from paper_2606_31093_amd import kvx
from paper_2606_31093_amd.workloads import LAYOUTS, PoolSpec
from test_gpu_decode import U, error_word, make_pool, make_table, rows_tensor, rows_values, tensor

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")]


# ---------------------------------------------------------------------------
# kvx_append_normed
# ---------------------------------------------------------------------------

def normed_case(seed, spec, kind, cache, lens, starts, positions, Hq, rot, off, inter, q_norm=None, k_norm=None, axes=0,
                turns=False, amplitude=1.0, in_place=False, weightless=False, stride=0):
    """q_norm, k_norm: (off, dim) or None; positions: of each record's first token."""
    rng = np.random.default_rng(seed)
    total, H, C, D = sum(lens), spec.H, spec.C, spec.D
    xb = np_decode.bits((rng.standard_normal((total, Hq + C * H, D)) * 3).astype(np.float32), kind)
    x = np_decode.values(xb, kind)
    pool = make_pool(rng, spec, cache)
    pt, offs = make_table(rng, spec, [s + n for s, n in zip(starts, lens)])
    first = np.concatenate([[0], np.cumsum(lens)[:-1]]).astype(int)
    rows = [[offs[r], first[r], starts[r], positions[r], lens[r]] for r in range(len(lens))]
    half = rot // 2
    freq = (10000.0 ** (-np.arange(half) * 2 / max(rot, 1))).astype(np.float32)
    scales = (rng.random((C, H)) * 0.05 + 0.02).astype(np.float32) if cache == "e4m3" else None
    eps = 1e-5
    weights = [None if n is None else (np.ones(n[1]) if weightless else rng.random(n[1]) + 0.5).astype(np.float32)
               for n in (q_norm, k_norm)]
    norms = [None if n is None else kvx.Norm(None, n[0], eps, n[1]) if weightless else kvx.Norm(tensor(w), n[0], eps)
             for n, w in zip((q_norm, k_norm), weights)]
    pos = axis = None
    if axes:
        pos = rng.integers(-5, 1 << 18, (axes, total)).astype(np.int32)
        if axes > 1:
            axis = (np.arange(half) % axes if turns else np.arange(half) * axes // max(half, 1)).astype(np.int32)
    xt = rows_tensor(xb, kind)
    q, k, v = xt[:, :Hq], xt[:, Hq:Hq + H], xt[:, Hq + H:]
    q_out = q if in_place else torch.zeros(total, Hq, D, dtype=q.dtype, device="cuda")
    tp, err = tensor(pool), error_word()
    pos_t = None
    if axes:
        wide = np.full((axes, total + stride), 1 << 29, np.int32)
        wide[:, :total] = pos
        pos_t = tensor(wide)[:, :total] if axes > 1 else tensor(pos[0])
    kvx.kvx_append_normed(tp, spec, spec.L - 1, k, v if C == 2 else None, tensor(pt), kvx.device_append_reqs(rows),
                          max(lens + [0]), q=q if Hq else None, q_out=q_out if Hq else None,
                          rope=kvx.Rope(tensor(freq), off, inter, amplitude) if rot else None, q_norm=norms[0],
                          k_norm=norms[1], positions=pos_t, axis=None if axis is None else tensor(axis),
                          scales=None if scales is None else tensor(scales), dev_err=err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0
    got_q = rows_values(q_out, kind)
    got, before = np_decode.canonical(tp.cpu().numpy(), spec), np_decode.canonical(pool, spec)
    written = np.zeros(before.shape, bool)
    u = U[kind]

    def rounding(y):
        return np.maximum(u * np.abs(y), 2.0 ** -25 if kind == "f16" else 0.0)

    for r, n in enumerate(lens):
        for i in range(n):
            row = first[r] + i
            at = np.full(half, positions[r] + i) if not axes else pos[axis if axis is not None else np.zeros(half, int), row]
            y = x[row].copy()
            for s, w, nm in ((slice(0, Hq), weights[0], q_norm), (slice(Hq, Hq + H), weights[1], k_norm)):
                if nm is not None:
                    y[s] = ref.norm(y[s], w.astype(np.float64), nm[0], eps)
            tol = (D / 2 + 6) * 2.0 ** -24 * np.abs(y)
            pairs = np.zeros_like(y)
            for j in range(half):
                a, b = (off + 2 * j, off + 2 * j + 1) if inter else (off + j, off + j + half)
                pairs[:Hq + H, [a, b]] = (np.abs(y[:Hq + H, a]) + np.abs(y[:Hq + H, b]))[:, None]
            tol = np.maximum(tol, (D / 2 + 6) * 2.0 ** -24 * amplitude * pairs) + 2.0 ** -20 * amplitude * pairs
            y[:Hq + H] = ref.rotate(y[:Hq + H], at, freq, off, inter, amplitude)
            assert (np.abs(got_q[row] - y[:Hq]) <= rounding(y[:Hq]) + (1 + u) * tol[:Hq]).all()
            page, slot = np_decode.resolve(pt, offs[r], starts[r] + i, spec.T, spec.N)
            for c in range(C):
                written[spec.L - 1, page, c, slot] = True
                z, t = y[Hq + c * H:Hq + (c + 1) * H], tol[Hq + c * H:Hq + (c + 1) * H]
                have = np_decode.values(got[spec.L - 1, page, c, slot], cache)
                if cache == "e4m3":
                    z, t = z / scales[c][:, None].astype(np.float64), t / scales[c][:, None]
                    z = np.clip(z, -448, 448)
                    # the quotient by the scale is rounded to 2^-24 first
                    assert (np.abs(have - z) <= np.maximum(2.0 ** -4 * np.abs(z), 2.0 ** -10) + 2 * t + 2.0 ** -23 * np.abs(z)).all()
                elif c == 1:
                    assert (have == z).all()            # values are copied
                else:
                    assert (np.abs(have - z) <= rounding(z) + (1 + u) * t).all()
    assert (got[~written] == before[~written]).all()


NORMED_SHAPES = [
    # (C, H, D, Hq, rot, off, q_norm, k_norm): whole heads; half and the end rotated; odd sizes; one pair; a part
    # normed; MLA; no rotation; no queries; wide heads
    (2, 2, 128, 8, 128, 0, (0, 128), (0, 128)), (2, 3, 64, 3, 32, 0, (0, 64), (0, 64)), (2, 1, 80, 4, 20, 4, (0, 80), (0, 80)),
    (2, 2, 96, 2, 32, 64, None, (0, 96)), (2, 1, 16, 1, 2, 3, (0, 16), (8, 8)), (2, 2, 32, 6, 0, 0, (0, 32), None),
    (1, 1, 576, 5, 64, 512, None, (0, 512)), (2, 4, 48, 0, 48, 0, None, (0, 48)), (2, 1, 256, 7, 256, 0, (0, 256), (0, 256)),
    (2, 1, 1024, 2, 1024, 0, (0, 1024), (0, 1024)), (2, 2, 80, 3, 80, 0, (0, 80), (16, 64)), (2, 1, 8, 1, 8, 0, (0, 8), (0, 8)),
    (2, 1, 128, 2, 8, 60, (0, 64), (64, 64)),
]


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("kind,cache", TYPES)
@pytest.mark.parametrize("C,H,D,Hq,rot,off,q_norm,k_norm", NORMED_SHAPES)
def test_append_normed(C, H, D, Hq, rot, off, q_norm, k_norm, kind, cache, inter):
    if cache == "e4m3" and D % 16:
        pytest.skip("rows of an 8-bit cache are whole 16 bytes")
    spec = PoolSpec(2, C, H, D, T=16, N=20, e=1 if cache == "e4m3" else 2, layout=LAYOUTS[(D + Hq) % 4])
    axes = 0 if rot == 0 else (D + Hq + inter) % 4
    normed_case(7, spec, kind, cache, [1, 0, 17, 33, 2], [15, 0, 3, 0, 40], [0, 5, 131000, 7, 1 << 30], Hq, rot, off, inter,
                q_norm, k_norm, axes=axes, turns=inter, amplitude=1.0 if inter else 1.25, stride=3)


@pytest.mark.parametrize("axes,turns", [(1, False), (2, True), (3, False), (3, True), (16, True)])
def test_append_normed_axes(axes, turns):
    spec = PoolSpec(1, 2, 2, 128, T=64, N=40, e=2)
    normed_case(3, spec, "bf16", "bf16", [70, 1, 300], [0, 5, 63], [0, 0, 0], 4, 128, 0, False, (0, 128), (0, 128), axes, turns)


def test_append_normed_in_place_and_without_weights():
    spec = PoolSpec(1, 2, 2, 128, T=64, N=40, e=2)
    normed_case(4, spec, "bf16", "bf16", [70, 1, 3], [0, 5, 63], [0, 9, 0], 4, 128, 0, True, (0, 128), (0, 128), in_place=True,
                weightless=True)
    normed_case(5, spec, "f16", "f16", [70, 1, 3], [0, 5, 63], [0, 9, 0], 4, 20, 4, False, (0, 128), (0, 128), in_place=True)


def test_append_normed_without_norms_is_append():
    """The same bits as kvx_append, also of what is neither rotated nor normed (a NaN with a payload)."""
    rng = np.random.default_rng(5)
    spec = PoolSpec(1, 2, 2, 64, T=16, N=8, e=2)
    xb = np_decode.bits(rng.standard_normal((20, 8, 64)).astype(np.float32), "bf16")
    xb[3, :, 40] = 0x7fa5
    xt = rows_tensor(xb, "bf16")
    q, k, v = xt[:, :4], xt[:, 4:6], xt[:, 6:]
    freq = tensor((10000.0 ** (-np.arange(16) / 16)).astype(np.float32))
    pt, reqs = tensor(np.arange(8, dtype=np.int32)), kvx.device_append_reqs([[0, 0, 5, 77, 20]])
    outs = []
    for call in (kvx.kvx_append, kvx.kvx_append_normed):
        for inter in (False, True):
            pool, q_out = torch.zeros(spec.nbytes, dtype=torch.uint8, device="cuda"), torch.zeros_like(q)
            call(pool, spec, 0, k, v, pt, reqs, 20, q=q, q_out=q_out, rope=kvx.Rope(freq, 4 if inter else 8, inter))
            outs.append((pool, q_out.view(torch.int16)))
    for a, b in zip(outs[:2], outs[2:]):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_append_normed_bad_axis_and_pages():
    spec = PoolSpec(1, 2, 1, 64, T=16, N=4, e=2)
    q = torch.randn(20, 2, 64, device="cuda").bfloat16()
    k = torch.randn(20, 1, 64, device="cuda").bfloat16()
    freq = tensor(np.ones(8, np.float32))
    w = kvx.Norm(torch.ones(64, device="cuda"))
    for bad in (-1, 2, 1 << 30):
        pool, q_out, err = torch.zeros(spec.nbytes, dtype=torch.uint8, device="cuda"), torch.zeros_like(q), error_word()
        axis = tensor(np.array([0, 1, 0, 1, bad, 0, 0, 0], np.int32))
        kvx.kvx_append_normed(pool, spec, 0, k, k, tensor(np.arange(4, dtype=np.int32)), kvx.device_append_reqs([[0, 0, 0, 0, 20]]),
                              20, q=q, q_out=q_out, rope=kvx.Rope(freq), q_norm=w, k_norm=w,
                              positions=torch.zeros(2, 20, dtype=torch.int32, device="cuda"), axis=axis, dev_err=err)
        assert int(err.item()) == kvx.DERR_BAD_REQ and not pool.any() and not q_out.any()
    # a page that is not there, and a malformed record among good ones
    pool, q_out, err = torch.zeros(spec.nbytes, dtype=torch.uint8, device="cuda"), torch.zeros_like(q), error_word()
    kvx.kvx_append_normed(pool, spec, 0, k, k, tensor(np.array([9, 1], np.int32)),
                          kvx.device_append_reqs([[0, 0, 0, 0, 18], [0, 19, 0, 0, 5], [0, 18, 40, 0, 1]]), 20, q=q, q_out=q_out,
                          rope=kvx.Rope(freq), q_norm=w, k_norm=w, dev_err=err)
    assert int(err.item()) == kvx.DERR_DST_PAGE | kvx.DERR_BAD_REQ | kvx.DERR_PT_RANGE
    assert q_out[:19].abs().sum(dim=(1, 2)).bool().all() and not q_out[19].any()
    at = np_decode.canonical(pool.cpu().numpy(), spec)
    assert at[0, 1, 0, :2].any() and not at[0, 1, :, 2:].any() and not at[0, [0, 2, 3]].any()


# ---------------------------------------------------------------------------
# kvx_attend_prompt, kvx_attend_tree
# ---------------------------------------------------------------------------

def random_tree(rng, n, empty=False):
    bits = []
    for j in range(n):
        b = 1 << j
        if j:
            b |= bits[int(rng.integers(max(0, j - 5), j))]
        bits.append(b)
    if empty:
        bits[n // 2] = 0
    return bits


def queries_case(seed, spec, kind, cache, recs, G, v_dim=None, scale=None, cap=0.0, slopes=False, window=0, tree=False,
                 spoil=False, size=1.0, gap=0, workspace=None, call_args=None, expect=0, pt_edit=None, strided=False, wide_cap=False):
    """recs: (start, end, n_queries, prefix); gap: rows between records that belong to none."""
    rng = np.random.default_rng(seed)
    H, C, D = spec.H, spec.C, spec.D
    v = v_dim or D
    Hq = H * G
    pool = make_pool(rng, spec, cache)
    pt, offs = make_table(rng, spec, [r[1] for r in recs])
    rows, total = [], gap
    for off, (start, end, n, prefix) in zip(offs, recs):
        rows.append((off, total, start, end, n, prefix))
        total += n + gap
    bits = None
    if tree:
        bits = rng.integers(0, 1 << 63, total).astype(np.uint64) << np.uint64(1)
        for _, row, _, _, n, _ in rows:
            bits[row:row + n] = np.array(random_tree(rng, n, n > 4), np.uint64)
            if n < 64:
                bits[row:row + n] |= rng.integers(0, 2, n).astype(np.uint64) << np.uint64(63)   # ignored
    if spoil:
        # NaN and infinities in slots that belong to nobody, and in positions before a record's start
        c = np_decode.canonical(pool, spec)
        used = np.zeros(c.shape[1:2] + c.shape[3:4], bool)
        for off, _, start, end, n, _ in rows:
            for t in range(start, end):
                page, slot = np_decode.resolve(pt, off, t, spec.T, spec.N)
                used[page, slot] = True
        bad = {"bf16": 0x7fc0, "f16": 0x7c00, "e4m3": 0x7f}[cache]
        for page, slot in zip(*np.nonzero(~used)):
            c[:, page, :, slot] = bad
    if pt_edit:
        pt_edit(pt)
    qb = np_decode.bits((rng.standard_normal((total, Hq, D)) * size).astype(np.float32), kind)
    scales = (rng.random((C, H)) * 0.02 + 0.005).astype(np.float32) if cache == "e4m3" else None
    sl = (rng.random(Hq) * 0.5).astype(np.float32) if slopes else None
    scale = D ** -0.5 if scale is None else scale
    want = ref.attend(np_decode.values(qb, kind), np_decode.values(np_decode.canonical(pool, spec), cache), spec, spec.L - 1, pt,
                      rows, scale, v, scales, cap, sl, window, bits)
    q = rows_tensor(qb, kind)
    out = torch.full((total, Hq + 1, v + 8) if strided else (total, Hq, v), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full((total, Hq), 7.0, device="cuda")
    err = error_word()
    most_q, most = max([r[2] for r in recs] + [0]), max([r[1] - r[0] for r in recs] + [0])
    ws = kvx.queries_workspace(spec, len(recs), Hq, most_q, most, v)
    ws.fill_(0xff)                       # a workspace may hold anything
    args = dict(scores=kvx.Scores(scale, cap, None if sl is None else tensor(sl), window),
                scales=None if scales is None else tensor(scales), lse=lse, dev_err=err, **(call_args or {}))
    view = out[:, :Hq, :v]
    head = (q, view, tensor(pool), spec, spec.L - 1, tensor(pt), kvx.device_queries_reqs(rows))
    if tree:
        kvx.kvx_attend_tree(*head, tensor(bits.view(np.int64)), most_q, most, ws, **args)
    else:
        kvx.kvx_attend_prompt(*head, most_q, most, ws, **args)
    torch.cuda.synchronize()
    assert int(err.item()) == expect
    check(want, rows_values(view, kind), lse.cpu().numpy().astype(np.float64), kind, D, 0.0 if wide_cap else cap,
          2.0 ** -19 if wide_cap else 0.0)
    if strided:
        assert (out[:, Hq:] == 7).all() and (out[:, :, v:] == 7).all()


def check(want, got, got_lse, kind, D, cap=0.0, relative=0.0):
    w_out, w_lse, mine, mag, dots, size, sums = want
    assert (got[~mine] == 7).all() and (got_lse[~mine] == 7).all()
    u = U[kind]
    ds = ((D + 8) * 2.0 ** -24 * dots + 2.0 ** -20 * cap + (2.0 ** -21 + relative) * size)[:, None]
    off = np.abs(got - w_out) - (u * np.abs(w_out) + (1 + u) * (u + 2 * ds + 2.0 ** -20)[..., None] * mag)
    if kind == "f16":
        off -= 2.0 ** -25 + 2.0 ** -32 * sums
    assert np.isfinite(got[mine]).all()
    assert (off[mine] <= 0).all(), float(off[mine].max())
    empty = np.isneginf(w_lse) & mine[:, None]
    assert np.isneginf(got_lse[empty]).all() and (got[empty] == 0).all()
    some = mine[:, None] & ~empty
    lse_off = np.abs(got_lse - np.where(some, w_lse, 0)) - (ds + 2.0 ** -20 * (1 + np.abs(np.where(some, w_lse, 0))))
    assert (lse_off[some] <= 0).all(), float(lse_off[some].max())


RECS = [(0, 70, 70, 0), (0, 1, 1, 0), (3, 40, 5, 0), (0, 33, 33, 20), (64, 130, 2, 0), (0, 0, 0, 0), (5, 5, 1, 0), (0, 95, 31, 95),
        (40, 64, 30, 0), (0, 129, 65, 7)]
SHAPES = [
    # (C, H, D, G, v): every kernel, sizes inside and at their ends, K without V
    (2, 2, 64, 4, 0), (2, 1, 128, 1, 0), (2, 2, 128, 4, 0), (2, 1, 128, 7, 0), (2, 2, 80, 3, 0), (2, 1, 192, 2, 0), (2, 1, 256, 5, 0),
    (1, 1, 576, 16, 512), (1, 2, 128, 3, 96), (2, 1, 320, 2, 0), (1, 1, 64, 2, 8), (2, 1, 16, 2, 0),
]


@pytest.mark.parametrize("kind,cache", TYPES)
@pytest.mark.parametrize("C,H,D,G,v", SHAPES)
def test_prompt(C, H, D, G, v, kind, cache):
    spec = PoolSpec(2, C, H, D, T=16, N=60, e=1 if cache == "e4m3" else 2, layout=LAYOUTS[(D // 16 + G) % 4])
    queries_case(D + G, spec, kind, cache, RECS, G, v or None, spoil=True, gap=2)


@pytest.mark.parametrize("kind,cache", TYPES)
@pytest.mark.parametrize("C,H,D,G,v", SHAPES)
def test_prompt_few_queries(C, H, D, G, v, kind, cache):
    """Up to 32 rows: single tokens and a few, at lengths around tiles and wavefronts."""
    spec = PoolSpec(1, C, H, D, T=24, N=80, e=1 if cache == "e4m3" else 2, layout=LAYOUTS[(D // 16 + G + 1) % 4])
    n = max(1, 32 // G)
    recs = [(0, n, n, 0), (0, 1, 1, 0), (0, 31 + n, n, 0), (0, 129, 1, 0), (31, 200, min(n, 3), 0), (0, 257, n, 0), (7, 7, 0, 0),
            (0, 300, 1, 300), (100, 400, n, 0)]
    queries_case(D + G, spec, kind, cache, recs, G, v or None, spoil=True, gap=1)


@pytest.mark.parametrize("kind,cache", TYPES)
@pytest.mark.parametrize("cap,slopes,window", [(5.0, False, 0), (0.0, True, 0), (0.0, False, 1), (0.0, False, 20), (2.0, True, 33)])
@pytest.mark.parametrize("C,H,D,G,v", [(2, 2, 64, 4, 0), (2, 1, 128, 7, 0), (2, 1, 256, 2, 0), (1, 1, 576, 16, 512)])
def test_prompt_scores(C, H, D, G, v, cap, slopes, window, kind, cache):
    spec = PoolSpec(1, C, H, D, T=16, N=60, e=1 if cache == "e4m3" else 2, layout=LAYOUTS[(D // 16 + G) % 4])
    queries_case(3, spec, kind, cache, RECS, G, v or None, cap=cap, slopes=slopes, window=window, spoil=True, size=4.0)
    few = [(0, 100, 2, 0), (17, 90, 1, 0), (0, 260, 2, 0), (0, 64, 1, 64)]
    queries_case(4, spec, kind, cache, few, G, v or None, cap=cap, slopes=slopes, window=window, spoil=True, size=4.0)


@pytest.mark.parametrize("kind,cache", [("bf16", "bf16"), ("f16", "e4m3")])
@pytest.mark.parametrize("C,H,D,G,v", [(2, 2, 64, 4, 0), (2, 1, 128, 7, 0), (2, 1, 256, 2, 0), (1, 1, 576, 16, 512)])
@pytest.mark.parametrize("cap,scale", [(200.0, 2.0), (1e6, None), (2.0 ** 100, None)])
def test_wide_caps(cap, scale, C, H, D, G, v, kind, cache):
    """Scores far below the cap, and some near it, keep their digits: tanh is off by 22 roundings of 2^-24
    at 1/4, where the series ends (the sum 1 + e^2x, its reciprocal and 1 less twice that: 11; those of the
    exponent: 9; the cap's: 2), and by fewer elsewhere, below 2^-19 of it."""
    spec = PoolSpec(1, C, H, D, T=16, N=60, e=1 if cache == "e4m3" else 2, layout=LAYOUTS[D // 16 % 4])
    queries_case(5, spec, kind, cache, RECS, G, v or None, scale=scale, cap=cap, slopes=D == 128, size=4.0, wide_cap=True)
    few = [(0, 100, 2, 0), (17, 90, 1, 0), (0, 260, 2, 0)]
    queries_case(6, spec, kind, cache, few, G, v or None, scale=scale, cap=cap, size=4.0, wide_cap=True)


@pytest.mark.parametrize("D", [64, 256])
def test_tiny_caps(D):
    """Scores of 0 under a cap so small that a score over it is infinite: the mean of what is seen."""
    spec = PoolSpec(1, 2, 1, D, T=16, N=60, e=2, layout="LPCTHD")
    queries_case(7, spec, "bf16", "bf16", RECS, 2, scale=8.0, cap=1e-39, size=0.0)


@pytest.mark.parametrize("kind,cache", TYPES)
@pytest.mark.parametrize("cap,slopes,window", [(0.0, False, 0), (3.0, True, 0), (0.0, True, 9), (0.0, False, 2)])
@pytest.mark.parametrize("C,H,D,G,v", [(2, 2, 64, 4, 0), (2, 1, 128, 7, 0), (2, 1, 256, 2, 0), (1, 1, 576, 16, 512), (2, 1, 128, 1, 0)])
def test_tree(C, H, D, G, v, cap, slopes, window, kind, cache):
    spec = PoolSpec(1, C, H, D, T=16, N=80, e=1 if cache == "e4m3" else 2, layout=LAYOUTS[(D // 16 + G) % 4])
    recs = [(0, 100, 20, 0), (0, 64, 64, 0), (90, 130, 60, 0), (0, 7, 1, 0), (3, 80, 33, 0), (0, 0, 0, 0), (20, 20, 5, 0),
            (0, 200, 7, 0)]
    queries_case(D + G, spec, kind, cache, recs, G, v or None, cap=cap, slopes=slopes, window=window, tree=True, spoil=True, gap=1)
    few = [(0, 260, max(1, 32 // G), 0), (33, 95, 1, 0), (0, 2, 2 if G <= 16 else 1, 0)]
    queries_case(D, spec, kind, cache, few, G, v or None, cap=cap, slopes=slopes, window=window, tree=True, spoil=True)


@pytest.mark.parametrize("kind,cache", [("bf16", "bf16"), ("f16", "e4m3")])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("C,H,D,G,v,n", [(2, 2, 64, 4, 0, 1), (2, 2, 64, 4, 0, 20), (2, 1, 128, 4, 0, 1), (2, 1, 128, 2, 0, 40),
                                         (2, 1, 128, 5, 0, 60), (2, 1, 256, 8, 0, 1), (2, 1, 256, 2, 0, 60), (1, 1, 576, 16, 512, 2),
                                         (1, 1, 576, 16, 512, 9), (2, 1, 320, 4, 0, 3), (1, 2, 80, 3, 40, 8)])
def test_split_and_joined(C, H, D, G, v, n, tree, kind, cache):
    """Long requests of few queries, whose units are split among workgroups and joined."""
    spec = PoolSpec(1, C, H, D, T=16, N=460, e=1 if cache == "e4m3" else 2, layout=LAYOUTS[G % 4])
    recs = [(0, 3001, n, 0), (77, 2000, 1, 0), (0, n, n, 0), (9, 9, 0, 0), (900, 1500, n, 0)]
    queries_case(D + G, spec, kind, cache, recs, G, v or None, tree=tree, spoil=True)
    if not tree:
        queries_case(D + G, spec, kind, cache, recs, G, v or None, window=700, spoil=True)


@pytest.mark.parametrize("C,H,D,G", [(2, 1, 128, 2), (2, 3, 64, 1)])
def test_long_prompt(C, H, D, G):
    """More than a block of rows, and blocks whose tiles are all seen, partly and not at all."""
    spec = PoolSpec(1, C, H, D, T=64, N=16, e=2)
    queries_case(1, spec, "bf16", "bf16", [(0, 700, 700, 0)], G)
    queries_case(2, spec, "bf16", "bf16", [(0, 700, 600, 300)], G, window=128)
    queries_case(3, spec, "bf16", "bf16", [(0, 260, 260, 260), (50, 300, 200, 0)], G)


@pytest.mark.parametrize("scale", [-0.3, 0.0, 1e-30])
@pytest.mark.parametrize("n", [2, 40])
def test_scale(scale, n):
    """A negative scale, none, and one so small that all scores are alike."""
    spec = PoolSpec(1, 2, 1, 64, T=16, N=20, e=2)
    for cap in (0.0, 4.0):
        queries_case(1, spec, "bf16", "bf16", [(0, 100, n, 0), (0, n, n, 0)], 4, scale=scale, cap=cap)


@pytest.mark.parametrize("T", [1, 7, 64])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_pages(layout, T):
    spec = PoolSpec(2, 2, 3, 64, T=T, N=-(-400 // T) + 6, e=2, layout=layout)
    queries_case(1, spec, "f16", "f16", [(0, 90, 90, 0), (5, 131, 3, 0), (0, 150, 64, 0)], 2, spoil=True, strided=True)
    queries_case(1, spec, "f16", "f16", [(0, 131, 3, 0), (50, 150, 1, 0)], 2, spoil=True, strided=True)


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("D,G,n", [(64, 4, 30), (128, 8, 30), (128, 2, 30), (128, 2, 3), (256, 2, 30), (64, 1, 5)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_a_row_does_not_see(D, G, n, tree, bad):
    """NaN and infinities in the keys and values of the last position (or draft) reach only the rows
    that see it."""
    rng = np.random.default_rng(D + G)
    spec = PoolSpec(1, 2, 1, D, T=16, N=12, e=2)
    for where in (n - 1, n // 2, 1):
        end = 100
        base = end - n
        pool = make_pool(rng, spec, "bf16")
        pt, _ = make_table(rng, spec, [end])
        page, slot = np_decode.resolve(pt, 0, base + where, spec.T, spec.N)
        clean = pool.copy()
        code = int(np_decode.bf16_bits(np.float32(bad)))
        c = np_decode.canonical(pool, spec)
        c[0, page, 1, slot, 0, 3:5] = code
        if bad != bad:
            c[0, page, 0, slot, 0, 7] = code
        q = (torch.randn(n, G, D, device="cuda") * 2).bfloat16()
        bits = torch.tensor([int(np.array(b, np.uint64).view(np.int64)) for b in random_tree(rng, n)], device="cuda")
        outs = []
        for p in (clean, pool):
            out, lse = torch.zeros_like(q), torch.zeros(n, G, device="cuda")
            ws = kvx.queries_workspace(spec, 1, G, n, end)
            head = (q, out, tensor(p), spec, 0, tensor(pt), kvx.device_queries_reqs([[0, 0, 0, end, n, 0]]))
            if tree:
                kvx.kvx_attend_tree(*head, bits, n, end, ws, lse=lse)
            else:
                kvx.kvx_attend_prompt(*head, n, end, ws, lse=lse)
            outs.append((out.float(), lse))
        see = (bits >> where & 1).bool() if tree else torch.arange(n, device="cuda") >= where
        assert torch.isfinite(outs[0][0]).all()
        assert torch.equal(outs[1][0][~see], outs[0][0][~see]) and torch.equal(outs[1][1][~see], outs[0][1][~see])
        hit = outs[1][0][see]
        if bad != bad:
            assert torch.isnan(hit).all()
        else:
            assert (hit[:, :, 3:5] == bad).all()
            rest = [d for d in range(D) if d not in (3, 4)]
            # the row's other values: its weight in 32 bits instead of rounded, and two roundings of outputs
            most = np.abs(np_decode.values(np_decode.canonical(clean, spec)[0, :, 1], "bf16")).max()
            assert (hit[:, :, rest] - outs[0][0][see][:, :, rest]).abs().max() <= 3 * U["bf16"] * most


def test_unresolved_pages():
    spec = PoolSpec(1, 2, 2, 128, T=16, N=30, e=2)

    def edit(pt):
        pt[2], pt[9] = 1 << 20, -1
    for recs in ([(0, 90, 60, 0), (20, 150, 30, 0)], [(0, 90, 1, 0), (20, 150, 2, 0)]):
        queries_case(1, spec, "bf16", "bf16", recs, 4, pt_edit=edit, expect=kvx.DERR_SRC_PAGE)


def test_malformed_records():
    spec = PoolSpec(1, 2, 2, 64, T=16, N=30, e=2)
    rng = np.random.default_rng(1)
    pool = tensor(make_pool(rng, spec, "bf16"))
    pt = tensor(np.arange(30, dtype=np.int32))
    bad = [(-1, 0, 0, 10, 2, 0), (0, -1, 0, 10, 2, 0), (0, 0, -1, 10, 2, 0), (0, 0, 10, 9, 2, 0), (0, 0, 0, 10, -1, 0), (0, 0, 0, 10, 11, 0),
           (0, 0, 0, 101, 2, 0), (0, 0, 0, 90, 65, 0), (0, 69, 0, 90, 2, 0), (0, 0, 0, 10, 2, -1), (0, 1 << 62, 0, 10, 2, 0)]
    for tree in (False, True):
        for most_q in (65, 64, 8):
            for rec in bad + [(0, 0, 0, 10, 2, 1)] * tree:
                if rec[4] == 65 and most_q == 65 and not tree:
                    continue
                q = torch.randn(70, 4, 64, device="cuda").bfloat16()
                out, lse, err = torch.full_like(q, 7), torch.full((70, 4), 7.0, device="cuda"), error_word()
                reqs = kvx.device_queries_reqs([rec, (0, 40, 0, 20, 3, 0)])
                ws = kvx.queries_workspace(spec, 2, 4, most_q, 100)
                args = (most_q, 100, ws)
                if tree:
                    kvx.kvx_attend_tree(q, out, pool, spec, 0, pt, reqs, torch.full((70,), 7, dtype=torch.int64, device="cuda"), *args,
                                        lse=lse, dev_err=err)
                else:
                    kvx.kvx_attend_prompt(q, out, pool, spec, 0, pt, reqs, *args, lse=lse, dev_err=err)
                assert int(err.item()) == kvx.DERR_BAD_REQ
                assert (out[:40] == 7).all() and (out[43:] == 7).all() and (out[40:43] != 7).any(dim=2).all()
                assert (lse[:40] == 7).all() and (lse[43:] == 7).all()
    # a table too short
    err = error_word()
    out = torch.zeros_like(q)
    kvx.kvx_attend_prompt(q, out, pool, spec, 0, pt[:1], kvx.device_queries_reqs([(0, 0, 0, 20, 3, 0)]), 3, 20, ws, dev_err=err)
    assert int(err.item()) == kvx.DERR_PT_RANGE


def test_queries_equal_attend():
    """A single query is kvx_attend's, within twice its bound."""
    rng = np.random.default_rng(2)
    spec = PoolSpec(1, 2, 2, 128, T=16, N=60, e=2)
    pool, pt = tensor(make_pool(rng, spec, "bf16")), tensor(rng.permutation(60).astype(np.int32))
    q = torch.randn(2, 8, 128, device="cuda").bfloat16()
    a, b = torch.zeros_like(q), torch.zeros_like(q)
    kvx.kvx_attend(q, a, pool, spec, 0, pt, kvx.device_attend_reqs([[0, 0, 0, 500], [32, 0, 3, 200]]), 500,
                   kvx.attend_workspace(spec, 2, 8, 500))
    kvx.kvx_attend_prompt(q, b, pool, spec, 0, pt, kvx.device_queries_reqs([[0, 0, 0, 500, 1, 0], [32, 1, 3, 200, 1, 0]]), 1, 500,
                          kvx.queries_workspace(spec, 2, 8, 1, 500))
    assert (a.float() - b.float()).abs().max() <= 4 * U["bf16"] * a.float().abs().max()


# ---------------------------------------------------------------------------
# kvx_keep_path
# ---------------------------------------------------------------------------

def path_case(seed, spec, paths, starts, most=None):
    rng = np.random.default_rng(seed)
    pool = rng.integers(0, 256, spec.nbytes).astype(np.uint8)
    pt, offs = make_table(rng, spec, [s + (p[-1] + 1 if p else 1) for s, p in zip(starts, paths)])
    flat = np.array([k for p in paths for k in p] + [0], np.int32)
    first = np.concatenate([[0], np.cumsum([len(p) for p in paths])]).astype(int)
    want = pool.copy()
    width = {1: np.uint8, 2: np.uint16, 4: np.uint32, 8: np.uint64}[spec.e]
    order = np_decode.ORDER[spec.layout]
    size = dict(l=spec.L, p=spec.N, c=spec.C, t=spec.T, h=spec.H, d=spec.D)
    w = want.view(width).reshape([size[x] for x in order]).transpose([order.index(x) for x in "lpcthd"])
    old = w.copy()
    for r, p in enumerate(paths):
        for i, k in enumerate(p):
            a = np_decode.resolve(pt, offs[r], starts[r] + k, spec.T, spec.N)
            b = np_decode.resolve(pt, offs[r], starts[r] + i, spec.T, spec.N)
            w[:, b[0], :, b[1]] = old[:, a[0], :, a[1]]
    t, err = tensor(pool), error_word()
    kvx.kvx_keep_path(t, spec, tensor(pt), kvx.device_path_reqs([[offs[r], first[r], starts[r], len(p)] for r, p in enumerate(paths)]),
                      max([len(p) for p in paths]) if most is None else most, tensor(flat), dev_err=err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0
    assert (t.cpu().numpy() == want).all()


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("C,H,D,e,T", [(2, 2, 64, 2, 16), (1, 1, 576, 2, 64), (2, 3, 16, 1, 7), (2, 1, 8, 4, 1), (2, 5, 80, 8, 24)])
def test_keep_path(C, H, D, e, T, layout):
    spec = PoolSpec(3, C, H, D, T=T, N=-(-500 // T) + 20, e=e, layout=layout)
    paths = [[0, 1, 5, 9], [], [7], list(range(0, 128, 2)), [0], [0, 1, 2, 3], [1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 63], list(range(1, 65))]
    path_case(D, spec, paths, [13, 0, 1, 5, 100, 7, 15, 3], most=64)


def test_keep_path_many_records():
    rng = np.random.default_rng(1)
    spec = PoolSpec(2, 2, 2, 32, T=16, N=1600, e=2)
    paths = [sorted(rng.choice(20, int(rng.integers(0, 9)), replace=False).tolist()) for _ in range(700)]
    path_case(1, spec, paths, rng.integers(0, 10, 700).tolist())


def test_keep_path_malformed():
    spec = PoolSpec(1, 2, 1, 64, T=16, N=8, e=2)
    good = [0, 2, 3]
    path = tensor(np.array(good + [1, 1, 2] + [2, 1, 3] + [-1, 5, 6] + [0, 1 << 30, 5], np.int32))
    pt = tensor(np.array([3, 1, 99, 2], np.int32))
    pool0 = torch.randint(0, 256, (spec.nbytes,), dtype=torch.uint8, device="cuda")
    for rec in [(-1, 0, 0, 3), (0, -1, 0, 3), (0, 0, -1, 3), (0, 0, 0, -1), (0, 0, 0, 9), (0, 13, 0, 3), (0, 3, 0, 3), (0, 6, 0, 3),
                (0, 9, 0, 3), (0, 12, (1 << 31) - 5, 2), (0, 1 << 62, 0, 3)]:
        pool, err = pool0.clone(), error_word()
        kvx.kvx_keep_path(pool, spec, pt, kvx.device_path_reqs([rec]), 8, path, dev_err=err)
        assert int(err.item()) == kvx.DERR_BAD_REQ and torch.equal(pool, pool0)
    for rec, bits in (((0, 1, 30, 1), kvx.DERR_SRC_PAGE), ((0, 1, 63, 1), kvx.DERR_PT_RANGE), ((2, 1, 0, 1), kvx.DERR_SRC_PAGE | kvx.DERR_DST_PAGE)):
        pool, err = pool0.clone(), error_word()
        kvx.kvx_keep_path(pool, spec, pt, kvx.device_path_reqs([rec]), 8, path, dev_err=err)
        assert int(err.item()) & bits and torch.equal(pool, pool0)


def test_keep_path_host_pool():
    spec = PoolSpec(2, 2, 2, 64, T=16, N=4, e=2)
    pool = torch.empty(spec.nbytes, dtype=torch.uint8, pin_memory=True)
    pool.copy_(torch.randint(0, 256, (spec.nbytes,), dtype=torch.uint8))
    dev = pool.cuda()
    args = (tensor(np.arange(4, dtype=np.int32)), kvx.device_path_reqs([[0, 0, 14, 3]]), 3, tensor(np.array([0, 4, 20], np.int32)))
    kvx.kvx_keep_path(pool, spec, *args)
    kvx.kvx_keep_path(dev, spec, *args)
    torch.cuda.synchronize()
    assert torch.equal(pool, dev.cpu())
