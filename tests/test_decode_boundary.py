"""Host-side checks of the decode step's calls without a GPU: records match
the C layout, every kind of bad argument returns its documented status before
anything touches the device, workspaces grow with their arguments, and the
frequencies follow their definitions."""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest

from paper_2606_31093_amd import build_lib, kvx
from paper_2606_31093_amd.workloads import PoolSpec

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20      # a 16-byte aligned address that is never dereferenced


@pytest.fixture(scope="module")
def lib():
    if build_lib.is_stale():
        build_lib.build()
    return kvx.lib()


def test_records_match_c(tmp_path):
    fields = {"kvx_append_req": kvx.APPEND_REQ_DTYPE, "kvx_attend_req": kvx.ATTEND_REQ_DTYPE,
              "kvx_select_req": kvx.SELECT_REQ_DTYPE}
    lines = [f'printf("{t} %zu\\n", sizeof({t}));' for t in (*fields, "kvx_rows", "kvx_rope")]
    lines += [f'printf("{t}.{f} %zu\\n", offsetof({t}, {f}));' for t, d in fields.items() for f in d.names]
    src = tmp_path / "l.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "kvx.h"\nint main(void) {' + "\n".join(lines) +
                   "return 0; }")
    exe = tmp_path / "l"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = dict(x.rsplit(" ", 1) for x in subprocess.run([str(exe)], capture_output=True, text=True,
                                                        check=True).stdout.split("\n") if x)
    for t, d in fields.items():
        assert int(got[t]) == d.itemsize
        for f in d.names:
            assert int(got[f"{t}.{f}"]) == d.fields[f][1]
    assert int(got["kvx_rows"]) == len(kvx._ROWS_PACK(0, 0, 0, 0, 0, 0, 0, 0))
    assert int(got["kvx_rope"]) == len(kvx._ROPE_PACK(0, 0, 0, 0, 0.0))


def rows(heads, dim, n=10, base=FAKE, s_row=None, s_head=None, dtype=0, reserved=0):
    return kvx._ROWS_PACK(base, n, heads * dim if s_row is None else s_row, dim if s_head is None else s_head, heads, dim,
                          dtype, reserved)


KV = PoolSpec(2, 2, 4, 64, T=16, N=8, e=2)
ONE = PoolSpec(2, 1, 1, 576, T=16, N=8, e=2)
F8 = PoolSpec(2, 2, 4, 64, T=16, N=8, e=1)


def append(spec=KV, layer=0, scales=None, q=rows(8, 64), q_out=rows(8, 64), k=rows(4, 64), v=rows(4, 64), rope=None,
           pt=FAKE, pt_len=1, reqs=FAKE, n=0, most=1, err=None, base=FAKE):
    return kvx.lib().kvx_append(bytes(kvx.pool_desc(spec, base)), layer, scales, q, q_out, k, v, rope, pt, pt_len, reqs, n,
                                most, err, None)


def rope(freq=FAKE, dim=64, off=0, inter=0):
    return kvx._ROPE_PACK(freq, dim, off, inter, 1.0)


@pytest.mark.parametrize("kw,status", [
    ({}, 0), (dict(q=None, q_out=None), 0), (dict(rope=rope()), 0), (dict(spec=F8, scales=FAKE), 0),
    (dict(spec=ONE, q=None, q_out=None, k=rows(1, 576), v=None), 0), (dict(base=None), -1), (dict(base=FAKE + 8), -3),
    (dict(spec=PoolSpec(2, 2, 4, 64, T=16, N=8, e=4)), -2), (dict(spec=PoolSpec(2, 2, 4, 64, T=16, N=8, e=8)), -2),
    (dict(layer=2), -5), (dict(layer=-1), -5), (dict(scales=FAKE), -2), (dict(spec=F8, scales=FAKE + 2), -3),
    (dict(q=None), -1), (dict(q_out=None), -1), (dict(k=None), -1), (dict(v=None), -1),
    (dict(spec=ONE, q=None, q_out=None, k=rows(1, 576), v=rows(1, 576)), -2), (dict(k=rows(3, 64)), -2),
    (dict(k=rows(4, 32)), -2), (dict(v=rows(4, 64, n=9)), -2), (dict(v=rows(4, 64, dtype=1)), -2),
    (dict(q=rows(8, 64, dtype=1)), -2), (dict(q_out=rows(7, 64)), -2), (dict(q_out=rows(8, 64, n=11)), -2),
    (dict(k=rows(4, 64, dtype=2)), -2), (dict(k=rows(4, 64, reserved=1)), -5), (dict(k=rows(4, 64, base=FAKE + 8)), -3),
    (dict(k=rows(4, 64, s_row=260)), -3), (dict(k=rows(4, 64, s_head=65)), -3), (dict(k=rows(4, 64, s_row=-256)), -5),
    (dict(k=rows(4, 64, base=0)), -1), (dict(k=rows(4, 64, n=-1)), -2), (dict(k=rows(4, 64, n=1 << 40, s_row=1 << 40)), -5),
    (dict(rope=rope(dim=63)), -2), (dict(rope=rope(dim=-2)), -2), (dict(rope=rope(off=2)), -2), (dict(rope=rope(off=-2)), -2),
    (dict(rope=rope(inter=2)), -5), (dict(rope=rope(freq=0)), -1), (dict(rope=rope(freq=FAKE + 2)), -3),
    (dict(rope=rope(freq=0, dim=0)), 0), (dict(n=-1), -5), (dict(n=65537), -5), (dict(n=1, reqs=None), -1),
    (dict(n=1, reqs=FAKE + 4), -3), (dict(most=-1), -5), (dict(most=(1 << 22) + 1), -5), (dict(pt_len=-1), -5),
    (dict(pt=None), -1), (dict(pt=FAKE + 2), -3), (dict(err=FAKE + 2), -3),
])
def test_append_refusals(lib, kw, status):
    assert append(**kw) == status
    assert bool(kvx.kvx_last_error()) == bool(status)


def attend(spec=KV, layer=0, scales=None, q=rows(8, 64), out=rows(8, 64), lse=None, pt=FAKE, pt_len=1, reqs=FAKE, n=0,
           most=1, acc=None, acc_len=0, stride=0, ws=FAKE, ws_bytes=1 << 30, err=None):
    return kvx.lib().kvx_attend(bytes(kvx.pool_desc(spec, FAKE)), layer, scales, q, out, lse, 1.0, pt, pt_len, reqs, n, most,
                                acc, acc_len, stride, ws, ws_bytes, err, None)


BIG = PoolSpec(1, 2, 1, 640, T=16, N=8, e=2)


@pytest.mark.parametrize("kw,status", [
    ({}, 0), (dict(spec=ONE, q=rows(128, 576), out=rows(128, 512)), 0), (dict(spec=F8, scales=FAKE), 0),
    (dict(q=rows(6, 64), out=rows(6, 64)), -2), (dict(q=rows(2048, 64), out=rows(2048, 64)), -2),
    (dict(out=rows(8, 56)), -2), (dict(spec=ONE, q=rows(4, 576), out=rows(4, 576)), -2), (dict(q=rows(8, 32)), -2),
    (dict(out=rows(4, 64)), -2), (dict(out=rows(8, 64, dtype=1)), -2), (dict(spec=BIG, q=rows(1, 640), out=rows(1, 640)), -2),
    (dict(q=None), -1), (dict(out=None), -1), (dict(n=11), -5), (dict(n=5, out=rows(8, 64, n=4)), -5),
    (dict(lse=FAKE + 2), -3), (dict(acc=FAKE, acc_len=-1), -5), (dict(acc=FAKE, stride=-1), -5), (dict(acc=FAKE + 2), -3),
    (dict(n=1, ws=None), -1), (dict(n=1, ws=FAKE + 8), -3), (dict(n=1, ws_bytes=16), -5), (dict(scales=FAKE), -2),
    (dict(most=-1), -5), (dict(reqs=None, n=1), -1), (dict(layer=2), -5), (dict(pt=FAKE + 1), -3),
])
def test_attend_refusals(lib, kw, status):
    assert attend(**kw) == status
    assert bool(kvx.kvx_last_error()) == bool(status)


def select(acc=FAKE, acc_len=100, stride=10, rows=10, reqs=FAKE, n=0, most=10, kept=FAKE, kept_len=100, ks=10, out=None,
           out_len=0, os_=0, err=None):
    return kvx.lib().kvx_select_kept(acc, acc_len, stride, rows, reqs, n, most, kept, kept_len, ks, out, out_len, os_, err,
                                     None)


@pytest.mark.parametrize("kw,status", [
    ({}, 0), (dict(rows=0), -5), (dict(rows=(1 << 20) + 1), -5), (dict(acc=None), -1), (dict(acc_len=-1), -5),
    (dict(stride=-1), -5), (dict(acc=FAKE + 2), -3), (dict(kept=None), -1), (dict(kept_len=-1), -5), (dict(ks=-1), -5),
    (dict(out=FAKE, out_len=-1), -5), (dict(out=FAKE + 1), -3), (dict(n=-1), -5), (dict(n=1, reqs=None), -1),
    (dict(most=-1), -5), (dict(err=FAKE + 1), -3),
])
def test_select_refusals(lib, kw, status):
    assert select(**kw) == status
    assert bool(kvx.kvx_last_error()) == bool(status)


def kept(S=KV, D=KV, sl=None, n=0, most=1, kept=FAKE, kept_len=10, stride=1, reqs=FAKE, spt=FAKE):
    x = None if sl is None else kvx._slice_arg(sl)
    return kvx.lib().kvx_transfer_kept(bytes(kvx.pool_desc(S, FAKE)), bytes(kvx.pool_desc(D, FAKE)), x, spt, 1, FAKE, 1, reqs,
                                       n, most, kept, kept_len, stride, None, None)


@pytest.mark.parametrize("kw,status", [
    ({}, 0), (dict(D=ONE), -2), (dict(D=F8), -2), (dict(sl=(0, 0, 3, 0, 0, 1, 0, 0, 1)), -5), (dict(n=-1), -5),
    (dict(sl=(0, 0, 0, 0, 0, 1, 0, 0, 1), n=1), 0), (dict(most=-1), -5), (dict(kept=None), -1), (dict(kept_len=-1), -5),
    (dict(stride=-1), -5), (dict(kept=FAKE + 2), -3), (dict(n=1, reqs=None), -1), (dict(spt=None), -1),
    (dict(S=PoolSpec(1 << 11, 2, 1 << 10, 16, T=1, N=1, e=1), D=PoolSpec(1 << 11, 2, 1 << 10, 16, T=1, N=1, e=1)), -5),
])
def test_transfer_kept_refusals(lib, kw, status):
    assert kept(**kw) == status
    assert bool(kvx.kvx_last_error()) == bool(status)


def test_workspace(lib):
    """Never smaller for more records or positions, so that one for the largest
    call serves all; refused shapes have none."""
    for spec, hq, v in ((KV, 8, 64), (KV, 4, 64), (ONE, 128, 512), (ONE, 20, 512), (PoolSpec(1, 2, 8, 128, T=16, N=1), 32, 128)):
        for acc in (False, True):
            last = 0
            for n in (0, 1, 2, 3, 7, 8, 31, 32, 33, 64, 255, 256, 1000, 4096):
                now = 0
                for most in (0, 1, 31, 32, 33, 100, 127, 129, 1000, 5000, 32768, 40000, 1 << 20):
                    b = kvx.attend_workspace_bytes(spec, n, hq, most, v, acc)
                    assert b >= now, (n, most)
                    now = b
                assert now >= last, n
                last = now
    with pytest.raises(kvx.KvxError):
        kvx.attend_workspace_bytes(KV, 1, 6, 10)
    with pytest.raises(kvx.KvxError):
        kvx.attend_workspace_bytes(KV, 1, 8, -1)
    assert kvx.lib().kvx_attend_workspace(None, 1, 8, 64, 10, 0) == -1


def test_binding_checks():
    import torch
    x = torch.zeros(2, 3, 64)
    for bad in (x, x.to(torch.bfloat16)[0], x.to(torch.bfloat16).transpose(1, 2)):
        with pytest.raises(ValueError):
            kvx._rows_arg(bad, "q")
    with pytest.raises(ValueError):
        kvx._floats(torch.zeros(4, dtype=torch.int32), "acc")
    with pytest.raises(ValueError):
        kvx._floats(torch.zeros(4, 4).t(), "acc")
    with pytest.raises(ValueError):
        kvx._scales(torch.zeros(3), KV)
    with pytest.raises(ValueError):
        kvx._reqs_arg(torch.zeros(33, dtype=torch.uint8), kvx.APPEND_REQ_DTYPE)
    with pytest.raises(ValueError):
        kvx._pack([[0, 0, 2**31, 0, 0]], kvx.APPEND_REQ_DTYPE)
    r = kvx._pack([[1, 2, 3, 4, 5]], kvx.APPEND_REQ_DTYPE)[0]
    assert tuple(r) == (1, 2, 3, 4, 5, 0)
    # strides of single rows and heads are never used and may be anything
    one = torch.zeros(1, 1, 64, dtype=torch.bfloat16).as_strided((1, 1, 64), (3, 5, 1))
    assert kvx._rows_arg(one, "q") == kvx._ROWS_PACK(one.data_ptr(), 1, 0, 0, 1, 64, 0, 0)


def test_rope_frequencies():
    plain = np.array([10000.0 ** (-2 * j / 128) for j in range(64)])
    f, a = kvx.rope_frequencies(128)
    np.testing.assert_allclose(f, plain, rtol=1e-7)
    assert a == 1.0 and f.dtype == np.float32
    f, a = kvx.rope_frequencies(128, factor=8.0)
    np.testing.assert_allclose(f, plain / 8, rtol=1e-7)
    f, a = kvx.rope_frequencies(128, factor=8.0, scaling="base")
    np.testing.assert_allclose([f[0], f[-1]], [1.0, plain[-1] / 8], rtol=1e-6)
    f, a = kvx.rope_frequencies(128, factor=8.0, scaling="ramp", trained=4096)
    turns = 4096 * plain / (2 * math.pi)
    np.testing.assert_allclose(f[turns > 40], plain[turns > 40], rtol=1e-6)
    np.testing.assert_allclose(f[turns < 0.8], plain[turns < 0.8] / 8, rtol=1e-6)
    assert (np.diff(f.astype(np.float64) / plain) <= 1e-6).all() and a == 0.1 * math.log(8) + 1
    for kw in (dict(rot_dim=63), dict(rot_dim=64, factor=0.5), dict(rot_dim=64, scaling="x"),
               dict(rot_dim=64, scaling="ramp"), dict(rot_dim=2, scaling="base"), dict(rot_dim=64, base=1.0)):
        with pytest.raises(ValueError):
            kvx.rope_frequencies(**kw)


@pytest.mark.parametrize("rot_dim,base,trained,factor,fast,slow", [
    (64, 1e4, 131072, 4.0, 32.0, 1.0),          # the slowest pair turns more than `slow` times
    (64, 1e4, 65536, 4.0, 32.0, 1.0),
    (128, 1e4, 131072, 8.0, 32.0, 1.0),
    (128, 1e6, 4096, 8.0, 32.0, 1.0),           # both ends inside
    (64, 100.0, 131072, 2.0, 32.0, 1.0),        # the ramp's end beyond every dimension
    (64, 100.0, 1 << 24, 2.0, 32.0, 1.0),       # every pair turns more than `fast` times: none changes
    (64, 1e4, 100, 4.0, 32.0, 1.0),             # none does: the ramp begins at the first pair
    (64, 1e4, 6, 4.0, 32.0, 1.0),               # no pair turns `slow` times: all are divided
    (2, 1e4, 1000, 4.0, 32.0, 1.0),
])
def test_rope_ramp_pair_by_pair(rot_dim, base, trained, factor, fast, slow):
    """Pair j turns trained * base ** (-2j / rot_dim) / (2 pi) times.  The ramp falls from the last whole
    pair index that turns `fast` times or more (or 0) to the first that turns `slow` times or fewer."""
    def index(turns):
        return rot_dim / 2 * math.log(trained / (2 * math.pi * turns), base)
    lo, hi = max(0, math.floor(index(fast))), math.ceil(index(slow))
    f, _ = kvx.rope_frequencies(rot_dim, base=base, factor=factor, scaling="ramp", trained=trained, fast=fast, slow=slow)
    for j in range(rot_dim // 2):
        plain = base ** (-2 * j / rot_dim)
        turns = trained * plain / (2 * math.pi)
        keep = 1.0 if j <= lo < hi else 0.0 if j >= hi else (hi - j) / (hi - lo)
        if turns > fast:
            assert keep == 1.0
        if turns < slow and lo < hi and j > lo:
            assert keep == 0.0
        assert abs(float(f[j]) / plain - (keep + (1 - keep) / factor)) < 1e-6, (j, turns)


def test_binding_needs_strides():
    """Without a stride several heads' accumulators, or rows' weights, would be the same ones."""
    import torch
    x, f = torch.zeros(1, 8, 64, dtype=torch.bfloat16), torch.zeros(100)
    reqs = torch.zeros(24, dtype=torch.uint8)
    with pytest.raises(ValueError, match="acc_stride"):
        kvx.kvx_attend(x, x, f, KV, 0, None, reqs, 1, f, acc=f)
    with pytest.raises(ValueError, match="acc_out_stride"):
        kvx.kvx_select_kept(f, 10, 2, reqs, 1, f, 10, f)


@pytest.mark.parametrize("n,heads,s_row,s_head,ok", [
    (3, 8, 512, 64, True), (3, 8, 64, 192, True), (3, 8, 0, 64, False), (3, 8, 512, 0, False), (1, 8, 0, 64, True),
    (1, 8, 0, 56, False), (3, 8, 504, 64, False), (3, 8, 56, 512, False), (3, 8, 64, 64, False), (3, 8, 64, 184, False),
    (2, 2, 192, 128, True), (3, 3, 192, 128, True), (3, 4, 192, 128, False), (2, 4, 192, 128, True), (3, 2, 184, 128, False),
])
def test_output_rows_share_nothing(lib, n, heads, s_row, s_head, ok):
    """Outputs whose rows meet would be written by several wavefronts; the rule against every pair of rows."""
    at = [i * s_row + j * s_head for i in range(n) for j in range(heads)]
    assert ok == all(abs(a - b) >= 64 for x, a in enumerate(at) for b in at[:x])
    o = rows(heads, 64, n, s_row=s_row, s_head=s_head)
    status = 0 if ok else -5
    assert append(spec=PoolSpec(2, 2, 1, 64, T=16, N=8, e=2), q=rows(heads, 64, n), q_out=o, k=rows(1, 64, n),
                  v=rows(1, 64, n)) == status
    # without a workspace, so that what passes this check is refused by a later one
    got = attend(spec=PoolSpec(2, 2, 1, 64, T=16, N=8, e=2), q=rows(heads, 64, n), out=o, n=n, ws=None)
    assert got == (-1 if ok else -5)
