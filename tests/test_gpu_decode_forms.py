"""Forms of the decode step's calls that sizes choose and test_gpu_decode.py does
not reach: every kernel of kvx_attend with its split and join, several blocks of
query heads, several launches (the test build starts a new one after 16 records
or 1024 workgroups), pools in pinned host memory, and the two parts that hold
the weights for their product with the values.  Bounds as there, and tighter
where a test says so."""
import numpy as np
import pytest
import torch

import np_decode as ref
import test_gpu_decode as base
from paper_2606_31093_amd import build_lib, kvx
from paper_2606_31093_amd.workloads import LAYOUTS, PoolSpec
from test_gpu_decode import error_word, rows_tensor, rows_values, tensor

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")]


@pytest.fixture
def several_launches(monkeypatch):
    kvx.lib()    # the product library first: raises if it is missing
    monkeypatch.setattr(kvx, "_LIB", kvx.load(build_lib.TEST_LIBRARY))


@pytest.mark.parametrize("kind,cache", TYPES)
@pytest.mark.parametrize("C,H,D,G,v", [
    (1, 1, 576, 48, 512), (1, 1, 576, 64, 512),       # latents: four wavefronts
    (1, 1, 576, 160, 512),                            # latents: two blocks of heads
    (1, 1, 320, 40, 256), (2, 1, 512, 20, 0),         # wide rows of another shape: four wavefronts
    (1, 2, 576, 5, 480), (2, 1, 272, 130, 0),         # and values that end inside, three blocks of heads
    (2, 1, 128, 80, 0), (2, 1, 64, 130, 0)])          # narrow rows: two and three blocks
def test_attend_blocks_of_heads(C, H, D, G, v, kind, cache):
    spec = PoolSpec(2, C, H, D, T=16, N=60, e=1 if cache == "e4m3" else 2, layout=LAYOUTS[(D // 16 + G) % 4])
    base.attend_case(D + G, spec, kind, cache, base.LENGTHS, G, v or None, acc=True, spoil=True)


@pytest.mark.parametrize("kind,cache", TYPES)
@pytest.mark.parametrize("layout", ["LPCTHD", "PLCHTD"])
@pytest.mark.parametrize("C,H,D,G,v", [
    (2, 2, 64, 4, 0), (2, 2, 80, 3, 0), (2, 4, 128, 7, 0), (2, 1, 128, 20, 0), (2, 1, 192, 3, 0), (2, 1, 256, 16, 0),
    (1, 2, 128, 4, 96), (2, 1, 96, 70, 0), (1, 1, 576, 16, 512), (1, 1, 576, 30, 512), (1, 1, 576, 64, 512),
    (1, 1, 576, 130, 512), (1, 1, 448, 6, 384), (2, 1, 320, 24, 0)])
def test_attend_split_and_joined(C, H, D, G, v, layout, kind, cache):
    """One long request and ragged ones, so that units are split among workgroups and joined."""
    spec = PoolSpec(1, C, H, D, T=16, N=420, e=1 if cache == "e4m3" else 2, layout=layout)
    base.attend_case(D + G, spec, kind, cache, [(0, 3001), (77, 2000), (0, 1), (5, 5), (900, 1300)], G, v or None, acc=True,
                     spoil=True)


@pytest.mark.parametrize("C,H,D,G,v", [(2, 2, 64, 4, 0), (1, 1, 576, 20, 512)])
def test_attend_more_records_than_a_launch(C, H, D, G, v):
    """1100 short records, with long ones on both sides of the 1024th."""
    spec = PoolSpec(1, C, H, D, T=16, N=1600, e=2)
    ranges = [(0, 1 + r % 5) for r in range(1100)]
    ranges[3], ranges[1023], ranges[1024], ranges[1090] = (0, 1500), (3, 1700), (0, 1100), (31, 900)
    base.attend_case(1, spec, "bf16", "bf16", ranges, G, v or None, acc=True)


@pytest.mark.parametrize("C,H,D,G,v,most", [(2, 2, 64, 4, 0, 70), (2, 2, 64, 40, 0, 700), (1, 1, 576, 128, 512, 600),
                                            (2, 1, 128, 4, 0, 3000)])
def test_attend_in_several_launches(several_launches, C, H, D, G, v, most):
    spec = PoolSpec(1, C, H, D, T=16, N=800, e=2)
    rng = np.random.default_rng(most)
    ranges = [(0, int(x)) for x in rng.integers(0, 150, 40)]
    ranges[7], ranges[16], ranges[39] = (3, most), (0, most), (most - 1, most)
    base.attend_case(2, spec, "bf16", "bf16", ranges, G, v or None, acc=True, spoil=True)


def test_append_in_several_launches(several_launches):
    spec = PoolSpec(1, 2, 2, 64, T=16, N=300, e=2)
    lens = [200, 0, 1, 17] * 15
    base.append_case(5, spec, "bf16", "bf16", lens, [r % 3 for r in range(60)], list(range(60)), 30, 64, 0, False, 1.0)


def test_select_in_several_launches(several_launches):
    n = 300
    base.select_case(6, [20 + r % 50 for r in range(n)], [10 + r % 20 for r in range(n)], [1] * n, [2] * n, 5,
                     base.WEIGHTS["heavy"])


def test_transfer_kept_in_several_launches(several_launches):
    S = PoolSpec(8, 1, 8, 16, T=16, N=80, e=1)           # 64 lists: 16 pieces of a record in a launch
    base.kept_case(7, S, S, [1150], [1100], [0], [0])
    S = PoolSpec(2, 2, 3, 16, T=16, N=700, e=2)          # 6 lists, 2 pieces, 120 records
    base.kept_case(8, S, S, [60 + r % 9 for r in range(119)] + [200], [30 + r % 30 for r in range(119)] + [100], [0] * 120,
                   [0] * 120)


def split_case(D, G, C):
    """Half of 256 positions of weight 1, the others of a weight that bfloat16 rounds down by nearly half a step, and
    values that nearly cancel: what the rounding leaves decides the result."""
    spec = PoolSpec(1, C, 1, D, T=16, N=16, e=2)
    p = 0.5 + 0.9 * 2.0 ** -9
    scale = float(np.float32(-np.log(p)))
    light = np.arange(256) % 2 == 1
    pool = np.zeros(spec.elems * 2, np.uint8)
    c = ref.canonical(pool, spec)[0].transpose(0, 2, 1, 3, 4).reshape(256, C, D)       # a copy: positions, kv, elements
    c[:, 0, D - 1] = np.where(light, 0xbf80, 0)                                       # a key of -1 or 0 in the last element
    v_dim = D if C == 2 else 512
    c[:, C - 1, :v_dim if C == 1 else D] = np.where(light, 0xbfff, 0x3f80)[:, None]   # -1.9921875 or 1
    ref.canonical(pool, spec)[0] = c.reshape(16, 16, C, 1, D).transpose(0, 2, 1, 3, 4)
    q = np.zeros((1, G, D), np.uint16)
    q[..., D - 1] = 0x3f80
    return spec, pool, q, scale, p, v_dim


@pytest.mark.parametrize("D,G,C", [(64, 8, 2), (128, 1, 2), (256, 4, 2), (576, 8, 1), (320, 3, 2)])
def test_attend_weights_to_twice_bfloat16(D, G, C):
    """Weights are held to twice bfloat16's 8 bits: out is off by u |out| + (u u + 2 ds + 2^-20) sum w |v|.
    (Few heads, where other columns of the products are free.)"""
    spec, pool, qb, scale, p, v_dim = split_case(D, G, C)
    pt, rows = np.arange(16, dtype=np.int32), [[0, 0, 0, 256]]
    want, _, _, mag, dots = ref.attend(ref.values(qb, "bf16"), ref.values(ref.canonical(pool, spec), "bf16"), spec, 0, pt, rows,
                                       scale, v_dim)
    u = base.U["bf16"]
    tol = u * np.abs(want) + (u * u + 2 * (D + 8) * 2.0 ** -24 * dots[0] + 2.0 ** -20) * mag
    # the same with weights rounded once would be outside
    once = (1 - 0.5 * 1.9921875) / (1 + p)
    assert (np.abs(once - want) > 8 * tol).all()
    q = rows_tensor(qb, "bf16")
    out = torch.zeros(1, G, v_dim, dtype=q.dtype, device="cuda")
    for most in (256, 1 << 20):          # a workgroup for the unit, and shares of its steps
        out.fill_(7.0)
        kvx.kvx_attend(q, out, tensor(pool), spec, 0, tensor(pt), kvx.device_attend_reqs(rows), most,
                       kvx.attend_workspace(spec, 1, G, most, v_dim), scale=scale)
        assert (np.abs(rows_values(out, "bf16") - want) <= tol).all()


def test_pinned_host_memory():
    """Kept rows from and to pools in pinned host memory, lists and records there too; attention reads such a pool;
    append writes device memory only."""
    S = PoolSpec(2, 2, 2, 64, T=16, N=8, e=2)
    rng = np.random.default_rng(9)
    src = torch.from_numpy(rng.integers(0, 256, S.nbytes).astype(np.uint8))
    pt, kept = np.arange(8, dtype=np.int32)[::-1].copy(), np.sort(rng.choice(100, (4, 40), replace=True), axis=1).astype(np.int32)
    reqs, err = kvx.device_reqs([[0, 0, 0, 0, 0, 40]], "cpu"), error_word()

    def pinned(x):
        t = torch.empty(x.shape, dtype=x.dtype, pin_memory=True)
        t.copy_(x)
        return t
    lists, table, recs = pinned(torch.from_numpy(kept)), pinned(torch.from_numpy(pt)), pinned(reqs)
    got = []
    for s, d in ((src.cuda(), torch.zeros(S.nbytes, dtype=torch.uint8, device="cuda")),
                 (src.cuda(), pinned(torch.zeros(S.nbytes, dtype=torch.uint8))),
                 (pinned(src), torch.zeros(S.nbytes, dtype=torch.uint8, device="cuda"))):
        kvx.kvx_transfer_kept(s, S, d, S, table, table, recs, 40, lists, 40, None, err)
        torch.cuda.synchronize()
        got.append(d.cpu().numpy())
    want = np.zeros(S.nbytes, np.uint8)
    a, b = ref.canonical(src.numpy(), S), ref.canonical(want, S)
    for l in range(2):
        for h in range(2):
            for i, k in enumerate(kept[2 * l + h]):
                b[l, pt[i // 16], :, i % 16, h] = a[l, pt[k // 16], :, k % 16, h]
    assert int(err.item()) == 0 and all(np.array_equal(x, want) for x in got)

    q = torch.randn(1, 4, 64, device="cuda").to(torch.bfloat16)
    host = pinned(torch.randn(S.elems).to(torch.bfloat16).view(torch.uint8))
    out = [torch.zeros_like(q) for _ in range(2)]
    for o, pool in zip(out, (host, host.cuda())):
        kvx.kvx_attend(q, o, pool, S, 1, table, kvx.device_attend_reqs([[0, 0, 0, 100]]), 100, kvx.attend_workspace(S, 1, 4, 100))
    assert torch.equal(out[0], out[1]) and out[0].any()
    k = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(kvx.KvxError, match="pool base"):
        kvx.kvx_append(host, S, 0, k, k, table, kvx.device_append_reqs([[0, 0, 0, 0, 1]]), 1)


def test_example_attends_over_what_it_keeps(monkeypatch):
    """The example, past an eviction: the lists are those of the accumulated weights, fresh pages hold their rows, the
    weights left are theirs, and the last step's outputs are attention over those rows and the newer ones."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import decode_step
    calls, moves = {}, []

    class Watched(decode_step.Sequences):
        def evict(self, sink=4, recent=32):
            full = [r for r in range(self.n) if self.length[r] == self.limit]
            pool, acc, pages = self.pool.cpu().numpy().copy(), self.acc.cpu().numpy().copy(), [list(p) for p in self.pages]
            freed = super().evict(sink, recent)
            for r in full:
                old, new = ref.canonical(pool, self.spec), ref.canonical(self.pool.cpu().numpy(), self.spec)
                left = self.acc[r].cpu().numpy()
                assert not set(pages[r]) & set(self.pages[r])
                for layer in range(self.spec.L):
                    for h in range(self.spec.H):
                        kept = ref.select(acc[r, layer, h], self.budget, sink, recent)
                        assert np.array_equal(left[layer, h, :self.budget], acc[r, layer, h, kept])
                        assert (left[layer, h, self.budget:] == 0).all()
                        for i, t in enumerate(kept):
                            a, b = pages[r][t // 64], self.pages[r][i // 64]
                            assert np.array_equal(new[layer, b, :, i % 64, h], old[layer, a, :, t % 64, h])
                moves.append(r)
            return freed

    real = kvx.kvx_attend

    def attend(q, out, pool, spec, layer, *rest, **kw):
        real(q, out, pool, spec, layer, *rest, **kw)
        calls[layer] = (q.clone(), out)
    monkeypatch.setattr(decode_step, "Sequences", Watched)
    monkeypatch.setattr(kvx, "kvx_attend", attend)
    s, outs = decode_step.run(steps=105, n=2, budget=64, limit=100, verbose=False)
    assert moves == [0, 1] and s.length == [69, 69] and sorted(calls) == [0, 1, 2]
    values = ref.values(ref.canonical(s.pool.cpu().numpy(), s.spec), "bf16")
    rows, u = [[r * s.slots_per, 0, 0, 69] for r in range(2)], base.U["bf16"]
    for layer, (q, out) in calls.items():
        want, _, _, mag, dots = ref.attend(rows_values(q, "bf16"), values, s.spec, layer, s.pt.cpu().numpy(), rows, 128 ** -0.5,
                                           128)
        tol = u * np.abs(want) + (u + 2 * ((128 + 8) * 2.0 ** -24 * dots)[:, None, None] + 2.0 ** -20) * mag
        assert (np.abs(rows_values(out, "bf16") - want) <= tol).all()


FORMS = [(64, 3, 2), (128, 16, 2), (192, 9, 2), (256, 20, 2), (128, 70, 2), (320, 12, 2), (512, 40, 2), (576, 8, 1), (576, 16, 1),
         (576, 30, 1), (576, 64, 1)]


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("D,G,C", FORMS)
def test_attend_weights_in_two_parts(D, G, C, kind):
    """Any number of query heads up to 64 on rows of more than 256 elements: the weights' rounding is that of their second
    part, 1/256 and 2^-8 of a weight in bfloat16, 1/16 and 2^-11 in half (a rounding of the first part is in the second)."""
    spec, pool, qb, scale, p, v_dim = split_case(D, G, C)
    u = base.U[kind]
    if kind == "f16":
        p = 0.5 + 0.9 * 2.0 ** -12
        scale = float(np.float32(-np.log(p)))
        swap = {0xbf80: 0xbc00, 0x3f80: 0x3c00, 0xbfff: 0xbfff, 0: 0}        # -1, 1, the largest value below 2 (negative), 0
        words = pool.view(np.uint16)
        words[:] = np.vectorize(swap.get)(words)
        qb = np.vectorize(swap.get)(qb).astype(np.uint16)
    pt, rows = np.arange(16, dtype=np.int32), [[0, 0, 0, 256]]
    want, _, _, mag, dots = ref.attend(ref.values(qb, kind), ref.values(ref.canonical(pool, spec), kind), spec, 0, pt, rows,
                                       scale, v_dim)
    part = 2.0 ** -7 if kind == "bf16" else 1 / 16 + 2.0 ** -11
    # a score is one product (the others are zeros): 2^-23 of it
    tol = u * np.abs(want) + (part * u + 2.0 ** -22 * dots[0] + 2.0 ** -20) * mag + (2.0 ** -24 if kind == "f16" else 0)
    last = 1.9921875 if kind == "bf16" else 2 - 2.0 ** -10
    assert (np.abs((1 - 0.5 * last) / (1 + p) - want) > 4 * tol).all()       # weights rounded once would be outside
    q = rows_tensor(qb, kind)
    out = torch.zeros(1, G, v_dim, dtype=q.dtype, device="cuda")
    for most in (256, 1 << 20):
        out.fill_(7.0)
        kvx.kvx_attend(q, out, tensor(pool), spec, 0, tensor(pt), kvx.device_attend_reqs(rows), most,
                       kvx.attend_workspace(spec, 1, G, most, v_dim), scale=scale)
        assert (np.abs(rows_values(out, kind) - want) <= tol).all()


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("D,G,C", FORMS + [(576, 128, 1)])
def test_attend_infinite_values(D, G, C, kind):
    """An infinite value reaches its element as such, also at weights that the rows' type holds exactly (1, 1/2, 2^-9), which
    leave no rest.  With one kv component it is a key's element too, which times the query's 0 makes the score NaN."""
    spec = PoolSpec(1, C, 1, D, T=16, N=16, e=2)
    one, inf = (0x3f80, 0x7f80) if kind == "bf16" else (0x3c00, 0x7c00)
    pool = np.zeros(spec.elems * 2, np.uint8)
    c = ref.canonical(pool, spec)                                 # l, page, kv, slot, h, d
    v_dim = D if C == 2 else 512
    c[0, :, C - 1, :, 0, :v_dim if C == 1 else D] = one
    if C == 2:
        c[0, :, 0] = 0
    # keys: score -k in log2 units by the last element's value times the scale
    key = {"bf16": [0, 0xbf80, 0xc110], "f16": [0, 0xbc00, 0xc880]}[kind]       # 0, -1, -9
    where = {0: (0, 3), 1: (7, 100), 2: (9, 201)}                 # which key: element, position
    c[0, :, 0, :, 0, D - 1] = key[2]
    for k, (d, t) in where.items():
        c[0, t // 16, 0, t % 16, 0, D - 1] = key[k]
        c[0, t // 16, C - 1, t % 16, 0, d] = inf
    qb = np.zeros((1, G, D), np.uint16)
    qb[..., D - 1] = one
    q = rows_tensor(qb, kind)
    out = torch.zeros(1, G, v_dim, dtype=q.dtype, device="cuda")
    for most in (256, 1 << 20):
        out.fill_(7.0)
        kvx.kvx_attend(q, out, tensor(pool), spec, 0, tensor(np.arange(16, dtype=np.int32)),
                       kvx.device_attend_reqs([[0, 0, 0, 256]]), most, kvx.attend_workspace(spec, 1, G, most, v_dim),
                       scale=float(np.log(2)))
        got = rows_values(out, kind)[0]
        if C == 1:
            assert np.isnan(got).all()
            continue
        assert np.isposinf(got[:, [0, 7, 9]]).all()
        rest = np.delete(got, [0, 7, 9], axis=1)
        assert (np.abs(rest - 1) <= base.U[kind] + 2.0 ** -16).all()
