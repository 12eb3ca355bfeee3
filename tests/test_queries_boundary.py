"""Host-side checks of the calls for several tokens of a request, without a GPU: records
match the C layout, every kind of bad argument returns its documented status before
anything touches the device, workspaces grow with their arguments."""
import os
import subprocess

import numpy as np
import pytest
import torch

import np_queries as ref
from paper_2606_31093_amd import build_lib, kvx
from paper_2606_31093_amd.workloads import PoolSpec
from test_decode_boundary import F8, FAKE, KV, ONE, ROOT, rows

NULL, SHAPE, ALIGN, RANGE = -1, -2, -3, -5


@pytest.fixture(scope="module", autouse=True)
def lib():
    if build_lib.is_stale():
        build_lib.build()
    return kvx.lib()


def test_records_match_c(tmp_path):
    fields = {"kvx_queries_req": kvx.QUERIES_REQ_DTYPE, "kvx_path_req": kvx.PATH_REQ_DTYPE}
    structs = ("kvx_norm", "kvx_positions", "kvx_scores")
    lines = [f'printf("{t} %zu\\n", sizeof({t}));' for t in (*fields, *structs)]
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
    assert int(got["kvx_norm"]) == len(kvx._NORM_PACK(0, 0, 0, 0.0, 0))
    assert int(got["kvx_positions"]) == len(kvx._POSITIONS_PACK(0, 0, 0, 0, 0))
    assert int(got["kvx_scores"]) == len(kvx._SCORES_PACK(0, 0.0, 0.0, 0, 0))


def pool(spec, base=FAKE):
    return bytes(kvx.pool_desc(spec, base))


def norm(weight=FAKE, dim=64, off=0, eps=1e-6, reserved=0):
    return kvx._NORM_PACK(weight, dim, off, eps, reserved)


def positions(ptr=FAKE, stride=10, axis=0, axes=1, reserved=0):
    return kvx._POSITIONS_PACK(ptr, stride, axis, axes, reserved)


ROPE = kvx._ROPE_PACK(FAKE, 64, 0, 0, 1.0)


def normed(spec=KV, q=rows(8, 64), q_out=rows(8, 64), k=rows(4, 64), v=rows(4, 64), rope=ROPE, q_norm=None, k_norm=None,
           pos=None, n=0, most=1, reqs=FAKE, err=None, layer=0, scales=None, pt=FAKE):
    return kvx.lib().kvx_append_normed(pool(spec), layer, scales, q, q_out, k, v, rope, q_norm, k_norm, pos, pt, 1, reqs, n,
                                       most, err, None)


WIDE = PoolSpec(2, 2, 4, 1032, T=16, N=8, e=2)


@pytest.mark.parametrize("want,args", [
    (0, {}), (0, dict(q_norm=norm(), k_norm=norm(0, 8, 56))), (0, dict(pos=positions())),
    (0, dict(pos=positions(axes=3, axis=FAKE))), (0, dict(k_norm=norm(), q=None, q_out=None)), (0, dict(rope=None, k_norm=norm())),
    (SHAPE, dict(k_norm=norm(dim=0))), (SHAPE, dict(k_norm=norm(dim=-8))), (SHAPE, dict(k_norm=norm(dim=12))),
    (SHAPE, dict(k_norm=norm(dim=64, off=8))), (SHAPE, dict(q_norm=norm(dim=8, off=4))), (SHAPE, dict(q_norm=norm(dim=8, off=-8))),
    (SHAPE, dict(q_norm=norm(dim=72))), (RANGE, dict(q_norm=norm(eps=-1e-9))), (RANGE, dict(q_norm=norm(eps=float("nan")))),
    (RANGE, dict(q_norm=norm(reserved=1))), (ALIGN, dict(k_norm=norm(FAKE + 2))),
    (NULL, dict(q_norm=norm(), q=None, q_out=None)), (NULL, dict(pos=positions(), rope=None)),
    (NULL, dict(pos=positions(), rope=kvx._ROPE_PACK(FAKE, 0, 0, 0, 1.0))), (NULL, dict(pos=positions(0))),
    (RANGE, dict(pos=positions(axes=0))), (RANGE, dict(pos=positions(axes=17, stride=20))), (RANGE, dict(pos=positions(reserved=1))),
    (RANGE, dict(pos=positions(stride=-1))), (RANGE, dict(pos=positions(axes=2, stride=9))),
    (RANGE, dict(pos=positions(axes=2, stride=1 << 60))), (ALIGN, dict(pos=positions(FAKE + 1))),
    (ALIGN, dict(pos=positions(axis=FAKE + 2))),
    (SHAPE, dict(spec=WIDE, q=None, q_out=None, k=rows(4, 1032), v=rows(4, 1032))),
    # what kvx_append refuses
    (RANGE, dict(layer=2)), (SHAPE, dict(scales=FAKE)), (SHAPE, dict(k=rows(3, 64))), (NULL, dict(q_out=None)), (NULL, dict(k=None)),
    (RANGE, dict(q_out=rows(8, 64, s_row=8))), (RANGE, dict(most=-1)), (RANGE, dict(n=-1)), (NULL, dict(n=1, reqs=0)),
    (ALIGN, dict(err=FAKE + 1)), (NULL, dict(pt=0)),
])
def test_append_normed_refuses(want, args):
    assert normed(**args) == want, kvx.kvx_last_error()


def scores(slopes=0, scale=0.1, cap=0.0, window=0, reserved=0):
    return kvx._SCORES_PACK(slopes, scale, cap, window, reserved)


def attend(spec=KV, q=rows(8, 64), out=rows(8, 64), lse=0, s=scores(), n=0, most_q=4, most=100, ws=FAKE, ws_bytes=1 << 40,
           tree=None, layer=0, scales=None, pt=FAKE, reqs=FAKE, err=None, base=FAKE):
    L = kvx.lib()
    head = (pool(spec, base), layer, scales, q, out, lse, s, pt, 1, reqs)
    rest = (n, most_q, most, ws, ws_bytes, err, None)
    if tree is None:
        return L.kvx_attend_prompt(*head, *rest)
    return L.kvx_attend_tree(*head, tree, *rest)


REFUSED = [
    (0, {}), (0, dict(s=scores(FAKE, -1.0, 30.0, 5))), (0, dict(spec=ONE, q=rows(16, 576), out=rows(16, 512))),
    (0, dict(spec=F8, scales=FAKE)),
    (NULL, dict(s=None)), (RANGE, dict(s=scores(reserved=1))), (RANGE, dict(s=scores(cap=-1.0))),
    (RANGE, dict(s=scores(cap=float("inf")))), (RANGE, dict(s=scores(cap=2.0 ** 101))), (RANGE, dict(s=scores(cap=float("nan")))), (RANGE, dict(s=scores(window=-1))),
    (ALIGN, dict(s=scores(FAKE + 2))), (RANGE, dict(most_q=-1)), (RANGE, dict(most_q=(1 << 22) + 1)), (RANGE, dict(most=-1)),
    (RANGE, dict(most=(1 << 22) + 1)), (ALIGN, dict(lse=FAKE + 2)), (SHAPE, dict(out=rows(4, 64))), (SHAPE, dict(out=rows(8, 64, n=9))),
    (SHAPE, dict(out=rows(8, 64, dtype=1))), (SHAPE, dict(out=rows(8, 56))), (SHAPE, dict(q=rows(8, 72), out=rows(8, 64))),
    (SHAPE, dict(q=rows(6, 64), out=rows(6, 64))), (SHAPE, dict(q=rows(1028, 64), out=rows(1028, 64))),
    (RANGE, dict(out=rows(8, 64, s_row=64))), (RANGE, dict(out=rows(8, 64, s_head=8))), (RANGE, dict(layer=-1)),
    (SHAPE, dict(scales=FAKE)), (NULL, dict(base=0)), (NULL, dict(q=None)), (NULL, dict(pt=0)), (RANGE, dict(n=65537)),
    (NULL, dict(n=1, ws=0)), (ALIGN, dict(n=1, ws=FAKE + 8)), (RANGE, dict(n=1, ws_bytes=8)), (NULL, dict(n=1, reqs=0)),
    (RANGE, dict(spec=PoolSpec(1, 2, 1, 64, T=16, N=8, e=2), q=rows(512, 64), out=rows(512, 64), most_q=1 << 22)),
]


@pytest.mark.parametrize("want,args", REFUSED)
@pytest.mark.parametrize("tree", [None, FAKE])
def test_attend_refuses(want, args, tree):
    assert attend(tree=tree, **args) == want, kvx.kvx_last_error()


def test_tree_refuses():
    assert attend(tree=0) == NULL
    assert attend(tree=FAKE + 4) == ALIGN


def test_keep_path_refuses():
    L = kvx.lib()

    def call(spec=KV, pt=FAKE, reqs=FAKE, n=0, most=4, path=FAKE, path_len=4, err=None, base=FAKE):
        return L.kvx_keep_path(pool(spec, base), pt, 1, reqs, n, most, path, path_len, err, None)
    assert call() == 0
    assert call(PoolSpec(1, 1, 1, 8, T=16, N=8, e=8)) == 0
    for want, args in ((RANGE, dict(most=65)), (RANGE, dict(most=-1)), (NULL, dict(path=0)), (ALIGN, dict(path=FAKE + 2)),
                       (RANGE, dict(path_len=-1)), (NULL, dict(pt=0)), (NULL, dict(n=1, reqs=0)), (ALIGN, dict(reqs=FAKE + 4)),
                       (RANGE, dict(n=-1)), (ALIGN, dict(err=FAKE + 1)), (NULL, dict(base=0))):
        assert call(**args) == want, args


def test_workspace_grows():
    """More records, queries or positions never need less, whatever kernel and division they take."""
    for spec, heads, v in ((KV, 8, 64), (ONE, 16, 512), (PoolSpec(1, 2, 2, 128, T=16, N=8, e=2), 8, 128),
                           (PoolSpec(1, 2, 8, 256, T=16, N=8, e=1), 8, 256)):
        def need(n, queries, tokens):
            return kvx.queries_workspace_bytes(spec, n, heads, queries, tokens, v)
        before = 0
        for queries in (0, 1, 2, 4, 8, 9, 16, 33, 64, 128, 129, 1000, 50000):
            per = 0
            for n in (0, 1, 2, 7, 32, 100, 600, 5000):
                last = 0
                for tokens in (0, 1, 31, 200, 256, 300, 3000, 100000):
                    x = need(n, queries, tokens)
                    assert x >= last
                    last = x
                assert last >= per
                per = last
            assert per >= before
            before = per
    L = kvx.lib()
    for args in ((pool(KV, 0), -1, 8, 64, 1, 1), (pool(KV, 0), 1, 7, 64, 1, 1), (pool(KV, 0), 1, 8, 64, -1, 1),
                 (pool(KV, 0), 1, 8, 64, 1, -1), (pool(KV, 0), 1, 8, 64, (1 << 22) + 1, 1), (pool(KV, 0), 1, 8, 64, 1, (1 << 22) + 1)):
        assert L.kvx_queries_workspace(*args) == -1
    with pytest.raises(kvx.KvxError):
        kvx.queries_workspace_bytes(KV, 1, 7, 1, 1)


def test_a_call_needs_no_more_than_its_workspace():
    """A call of any sizes up to those of a workspace takes it: its own check of the bytes passes, and the next
    refusal, of a tree at an odd address, is what returns."""
    for spec, q, out, heads, v in ((KV, rows(8, 64), rows(8, 64), 8, 64), (ONE, rows(16, 576), rows(16, 512), 16, 512)):
        have = kvx.queries_workspace_bytes(spec, 600, heads, 1000, 3000, v)
        for queries in (0, 1, 2, 8, 9, 40, 200, 1000):
            for n in (1, 2, 7, 100, 600):
                for tokens in (0, 300, 3000):
                    assert attend(spec, q, out, n=n, most_q=queries, most=tokens, ws_bytes=have, reqs=FAKE + 4) == ALIGN
                    x = attend(spec, q, out, n=n, most_q=queries, most=tokens, ws_bytes=have, ws=FAKE + 8)
                    assert x == ALIGN and "workspace" in kvx.kvx_last_error()
                    # with enough bytes the call goes on to the pointers, none of which is memory here
                    x = attend(spec, q, out, n=n, most_q=queries, most=tokens, ws_bytes=have)
                    assert x != 0 and "bytes, this call needs" not in kvx.kvx_last_error()


def test_binding_checks():
    spec = PoolSpec(1, 2, 2, 64, T=16, N=4, e=2)
    p, pt = torch.zeros(spec.nbytes, dtype=torch.uint8), torch.zeros(4, dtype=torch.int32)
    q, k = torch.zeros(4, 4, 64, dtype=torch.bfloat16), torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    reqs = kvx.device_append_reqs([[0, 0, 0, 0, 4]], "cpu")
    rope = kvx.Rope(torch.zeros(32))

    def append(**kw):
        kvx.kvx_append_normed(p, spec, 0, k, k, pt, reqs, 4, q=q, q_out=q.clone(), **{"rope": rope, **kw})
    for kw in (dict(axis=torch.zeros(32, dtype=torch.int32)), dict(positions=torch.zeros(3, dtype=torch.int32)),
               dict(positions=torch.zeros(4)), dict(positions=torch.zeros(2, 4, dtype=torch.int64)),
               dict(positions=torch.zeros(4, 2, dtype=torch.int32).t()), dict(positions=torch.zeros(1, 1, 4, dtype=torch.int32)),
               dict(positions=torch.zeros(4, dtype=torch.int32), axis=torch.zeros(31, dtype=torch.int32)),
               dict(q_norm=kvx.Norm(torch.zeros(64, dtype=torch.float16))), dict(q_norm=kvx.Norm(torch.zeros(64), dim=32))):
        with pytest.raises(ValueError):
            append(**kw)
    reqs = kvx.device_queries_reqs([[0, 0, 0, 4, 4, 0]], "cpu")
    ws = torch.zeros(1 << 20, dtype=torch.uint8)

    def attend(**kw):
        tree = kw.pop("tree", False)
        if tree is False:
            kvx.kvx_attend_prompt(q, q.clone(), p, spec, 0, pt, reqs, 4, 4, ws, **kw)
        else:
            kvx.kvx_attend_tree(q, q.clone(), p, spec, 0, pt, reqs, tree, 4, 4, ws, **kw)
    for kw in (dict(tree=None), dict(tree=torch.zeros(4, dtype=torch.int32)), dict(tree=torch.zeros(3, dtype=torch.int64)),
               dict(tree=torch.zeros(4, dtype=torch.float64)), dict(lse=torch.zeros(15)), dict(scores=kvx.Scores(slopes=torch.zeros(3))),
               dict(scales=torch.zeros(3))):
        with pytest.raises(ValueError):
            attend(**kw)
    with pytest.raises(ValueError):
        kvx.device_queries_reqs([[0, 0, 0, 1 << 31, 1, 0]], "cpu")


def test_definitions():
    """The reference's own: a tree of one branch sees what a prompt sees, and a norm leaves a mean square of 1."""
    n = 7
    bits = np.array([(1 << (j + 1)) - 1 for j in range(n)], np.uint64)
    rec = (0, 0, 2, 30, n, 0)
    for window in (0, 1, 4, 12):
        for i in range(n):
            for t in range(30):
                assert ref.sees(rec, i, t, window, bits) == ref.sees(rec, i, t, window, None)
    x = np.random.default_rng(1).standard_normal((3, 64))
    assert np.allclose((ref.norm(x, np.ones(32), 16, 0.0)[:, 16:48] ** 2).mean(axis=-1), 1)


@pytest.mark.parametrize("n", [1 << 57, 1 << 61, 1 << 62, (1 << 63) - 1])
def test_positions_of_more_rows_than_bytes_count(n):
    """Rows that share elements (stride 0) may be any number; their positions' bytes have to fit 63 bits."""
    k = rows(4, 64, n=n, s_row=0)
    assert normed(q=None, q_out=None, k=k, v=k, pos=positions(stride=0)) == RANGE
    assert normed(q=None, q_out=None, k=k, v=k, pos=positions(stride=n, axes=3)) == RANGE
    assert normed(q=None, q_out=None, k=k, v=k) == 0
