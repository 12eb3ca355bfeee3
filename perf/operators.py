"""The decode step's operators over a paged KV cache, as cases to measure.

A case is a dict of plain values.  ``kind`` says which operator a pass runs:
- ``append``: kvx_append, the new tokens' queries and keys rotated, keys and
  values written into the request's pages of one layer;
- ``attend``: kvx_attend, one query per request over its pages of one layer,
  optionally adding each position's attention weight to its accumulator;
- ``select``: kvx_select_kept, the positions each layer and head keeps of a
  request, by accumulated weight;
- ``kept``: kvx_transfer_kept, the kept rows moved into pages of another pool.

Request lengths follow from the case alone, so every seed has the same work;
the seed gives values, page tables, lists and accumulators.  Pools hold some
pages that belong to nobody.  Where ``own`` is false a pass is computed with
elementary torch operations in 32 bits, else by the library.
"""
import math
import types

import numpy as np
import torch

own = False

# The requests' token counts are drawn with this seed and the case's sizes.
LENGTHS_SEED = 31094

AXES = {"LPCTHD": "lpcthd", "LPCHTD": "lpchtd", "PLCTHD": "plcthd", "PLCHTD": "plchtd"}
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
# The records the library's calls take.
APPEND_REQ = np.dtype([("pt_off", "<i8"), ("row_off", "<i8"), ("start", "<i4"), ("position", "<i4"),
                       ("n_tokens", "<i4"), ("reserved", "<i4")])
ATTEND_REQ = np.dtype([("pt_off", "<i8"), ("acc_off", "<i8"), ("start", "<i4"), ("end", "<i4")])
SELECT_REQ = np.dtype([("acc_off", "<i8"), ("kept_off", "<i8"), ("out_off", "<i8"), ("n_tokens", "<i4"),
                       ("n_keep", "<i4"), ("sink", "<i4"), ("recent", "<i4")])
MOVE_REQ = np.dtype([("src_pt_off", "<i8"), ("dst_pt_off", "<i8"), ("buf_off", "<i8"), ("src_start", "<i4"),
                     ("dst_start", "<i4"), ("n_tokens", "<i4"), ("reserved", "<i4")])


def _case(name, kind, L, C, H, D, T, layout, n, lo, hi, G=1, cache="bf16", q="bf16", rot=0, off=0, pairs="halves",
          v=0, acc=False, keep=0, sink=0, recent=0, Td=0, dst="", start=0):
    c = dict(kind=kind, L=L, C=C, H=H, D=D, T=T, layout=layout, n=n, lo=lo, hi=hi, G=G, cache=cache, q=q, rot=rot,
             off=off, pairs=pairs, v=v or D, acc=acc, keep=keep, sink=sink, recent=recent, Td=Td, dst=dst, start=start)
    return dict(c, name=name) if name else c


def listed():
    return [
        # The newest token of 64 running sequences: 32 query heads on 8 cache heads.
        _case("append_step", "append", 2, 2, 8, 128, 64, "LPCTHD", 64, 1, 1, G=4, rot=128, start=37),
        # Prompts as prefill leaves them, half of each head rotated, into an 8-bit head-major cache.
        _case("append_prompt", "append", 2, 2, 4, 128, 64, "PLCHTD", 4, 1024, 8192, G=7, cache="e4m3", rot=64),
        # Chunks of prompts of an MLA model: one latent of 512 + 64, the 64 rotated.
        _case("append_latent", "append", 2, 1, 1, 576, 64, "LPCTHD", 16, 257, 2048, G=16, rot=64, off=512,
              pairs="interleaved"),
        # The smallest call in earnest: one short sequence of a small model.
        _case("attend_tiny", "attend", 2, 2, 2, 64, 16, "LPCTHD", 1, 100, 100, G=4),
        # One long sequence alone: its length has to fill the device.
        _case("attend_one", "attend", 2, 2, 8, 128, 64, "LPCTHD", 1, 32768, 32768, G=4),
        # A decode batch that keeps account of what each position contributes.
        _case("attend_batch", "attend", 2, 2, 8, 128, 64, "LPCTHD", 32, 1024, 8192, G=4, acc=True),
        # The same from an 8-bit head-major cache with 7 queries to a cache head.
        _case("attend_8bit", "attend", 2, 2, 4, 128, 64, "PLCHTD", 16, 2048, 16384, G=7, cache="e4m3"),
        # MLA with all 128 query heads on one latent.
        _case("attend_latent", "attend", 1, 1, 1, 576, 64, "LPCTHD", 16, 4096, 32768, G=128, v=512),
        # One sequence over its budget: 36 layers x 8 heads choose 1024 of 1500 positions.
        _case("select_one", "select", 36, 2, 8, 128, 64, "LPCTHD", 1, 1500, 1500, keep=1024, sink=4, recent=128),
        # A batch of long sequences brought back to 2048 positions.
        _case("select_batch", "select", 28, 2, 4, 128, 16, "LPCTHD", 16, 2048, 16384, keep=2048, sink=4, recent=256),
        # The rows of the one sequence, into fresh pages of the same shape.
        _case("kept_one", "kept", 36, 2, 8, 128, 64, "LPCTHD", 1, 1500, 1500, keep=1024, Td=64, dst="LPCTHD"),
        # The rows of the batch, handed to a role with larger head-major pages: the largest case.
        _case("kept_batch", "kept", 28, 2, 4, 128, 16, "LPCTHD", 16, 2048, 16384, keep=2048, Td=64, dst="PLCHTD"),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("append", "append", "attend", "attend", "attend", "select", "kept"))
    mla = rng.random() < 0.25
    T, layout = rng.choice((16, 32, 64, 64, 128, 24)), rng.choice(sorted(AXES))
    q = rng.choice(("bf16", "bf16", "f16"))
    cache = "e4m3" if rng.random() < 0.3 else q
    C, H, D = (1, 1, 576) if mla else (2, rng.choice((1, 2, 4, 5, 8, 8)), rng.choice((64, 80, 128, 128, 128, 192, 256)))
    G = rng.choice((8, 16, 16, 32, 64, 128)) if mla else rng.choice((1, 2, 4, 4, 5, 7, 8, 8, 16))
    e = 1 if cache == "e4m3" else 2
    rot, off = (64, 512) if mla else rng.choice(((D, 0), (D, 0), (D // 2 // 8 * 8, 0), (32, D - 32)))
    if kind == "append":
        row = (H * G + C * H) * D * 2
        n = log(1, 256)
        lo = 1 if rng.random() < 0.4 else log(1, 4096)
        hi = 1 if lo == 1 else lo + rng.randrange(lo)
        n = max(1, min(n, int(200e6 / (row * (lo + hi) / 2))))
        return _case("", kind, 2, C, H, D, T, layout, n, lo, hi, G=G, cache=cache, q=q, rot=rot, off=off,
                     pairs=rng.choice(("halves", "interleaved")), start=rng.choice((0, 1, 777)))
    lo = log(16, 32768)
    hi = min(32768, lo + rng.randrange(lo))
    n = log(1, 128)
    if kind == "attend":
        token = max(C * H * D * e / 600e6, 4 * H * G * D / 80e9)      # of the largest pass
        n = max(1, min(n, int(2 / (token * (lo + hi)))))
        return _case("", kind, 1, C, H, D, T, layout, n, lo, hi, G=G, cache=cache, q=q, v=512 if mla else D,
                     acc=rng.random() < 0.4, start=rng.choice((0, 0, 0, 1, lo // 3)))
    L = rng.randint(2, 61)
    keep = max(1, int(lo * rng.uniform(0.2, 1.0)))
    if kind == "select":
        sink = min(4, keep // 4)
        n = max(1, min(n, int(300e6 / (4 * L * H * (lo + hi) / 2))))
        return _case("", kind, L, C, H, D, T, layout, n, lo, hi, keep=keep, sink=sink,
                     recent=min(keep - sink, rng.choice((0, 16, keep // 8))))
    n = max(1, min(n, int(5e9 / (L * C * H * D * e * (lo + hi) / 2))))
    keep = min(keep, int(3e9 / (2 * n * L * C * H * D * e)) + 1)
    return _case("", kind, L, C, H, D, T, layout, n, lo, hi, cache=cache, keep=keep, Td=rng.choice((T, 16, 64, 24)),
                 dst=rng.choice((layout, "LPCTHD", "PLCHTD")))


# ---------------------------------------------------------------------------
# what follows from a case alone
# ---------------------------------------------------------------------------

def _ceil(a, b):
    return -(-a // b)


def _tokens(case):
    rng = np.random.default_rng([LENGTHS_SEED, case["n"], case["lo"], case["hi"]])
    return rng.integers(case["lo"], case["hi"] + 1, size=case["n"])


def _first(n):
    """Offsets of consecutive blocks of n[r] entries."""
    return np.concatenate([[0], np.cumsum(n)[:-1]]).astype(np.int64)


def _size(case):
    return 1 if case["cache"] == "e4m3" else 2


def _begins(case, n):
    """The first position attended of each request (a sliding window)."""
    return np.minimum(case["start"], n - 1)


def work(case):
    n, e = _tokens(case), _size(case)
    H, G, C, D, L = case["H"], case["G"], case["C"], case["D"], case["L"]
    total = int(n.sum())
    if case["kind"] == "append":
        moved = total * (2 * H * G * D * 2 + C * H * D * (2 + e))
        return {"bytes": moved + 32 * len(n) + 4 * int((n + case["T"] - 1).sum() // case["T"]),
                "flops": 10 * total * H * (G + 1) * case["rot"] // 2}
    if case["kind"] == "attend":
        seen = int((n - _begins(case, n)).sum())
        b = seen * C * H * D * e + len(n) * H * G * ((D + case["v"]) * 2 + 4) + 24 * len(n)
        b += 4 * (seen // case["T"] + len(n)) + (8 * seen * H if case["acc"] else 0)
        return {"bytes": b, "flops": 2 * seen * H * G * (D + case["v"])}
    kept = int(np.minimum(n, case["keep"]).sum())
    if case["kind"] == "select":
        return {"bytes": L * H * (4 * total + 8 * kept) + 40 * len(n), "flops": 0}
    return {"bytes": L * H * kept * (2 * C * D * e + 4) + 40 * len(n), "flops": 0}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _spec(L, C, H, D, T, N, e, layout):
    return types.SimpleNamespace(L=L, C=C, H=H, D=D, T=T, N=N, e=e, layout=layout)


def _records(dtype, dev, **columns):
    a = np.zeros(len(next(iter(columns.values()))), dtype)
    for k, x in columns.items():
        a[k] = x
    cols = {k: torch.from_numpy(a[k].astype(np.int64)).to(dev) for k in columns}
    return torch.from_numpy(a.view(np.uint8).copy()).to(dev), cols


def _pages(rng, T, ends):
    """Pages of a pool for requests of `ends` positions, their table and its offsets."""
    count = -(-ends // T)
    used = int(count.sum())
    N = used + used // 8 + 3
    return N, rng.permutation(N)[:used].astype(np.int32), _first(count)


def _fill(n, kind, g, dev):
    """n cache values of a pool: roughly normal, as keys and values are."""
    x = torch.randn(n, generator=g, device=dev, dtype=torch.bfloat16 if kind == "bf16" else torch.float16)
    return x.to(DTYPES[kind]).view(torch.uint8)


def prepare(case, seed):
    dev = torch.device("cuda")
    rng = np.random.default_rng([seed, 2])
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    n, e, kind = _tokens(case), _size(case), case["kind"]
    L, C, H, D, G, T = (case[k] for k in ("L", "C", "H", "D", "G", "T"))
    dt = DTYPES[case["q"]]
    st = dict(case=case, kind=kind, layer=L - 1, most=int(n.max()), total=int(n.sum()),
              err=torch.zeros(1, dtype=torch.int32, device=dev))
    if kind == "select":
        cap, kcap = _ceil(st["most"], 64) * 64, case["keep"]
        # sums of softmax weights: a few positions hold most, many hold next to nothing or nothing
        acc = torch.randn(len(n), L * H, cap, generator=g, device=dev).mul_(2.5).exp_().mul_(1e-3)
        acc.mul_(acc > 2e-5)
        r = np.arange(len(n), dtype=np.int64)
        st["reqs"], st["cols"] = _records(SELECT_REQ, dev, acc_off=r * (L * H * cap), kept_off=r * (L * H * kcap),
                                          out_off=r * (L * H * kcap), n_tokens=n, n_keep=np.full_like(n, case["keep"]),
                                          sink=np.full_like(n, case["sink"]), recent=np.full_like(n, case["recent"]))
        st.update(acc=acc, kept=torch.full((len(n), L * H, kcap), -1, dtype=torch.int32, device=dev),
                  out=torch.zeros(len(n), L * H, kcap, device=dev))
        return st

    ends = n + case["start"] if kind == "append" else n
    N, pt, off = _pages(rng, T, ends)
    st.update(spec=_spec(L, C, H, D, T, N, e, case["layout"]), pt=torch.from_numpy(pt).to(dev))
    st["pool"] = _fill(L * N * C * T * H * D, case["cache"], g, dev)
    st["scales"] = torch.rand(C, H, generator=g, device=dev) * 0.05 + 0.02 if e == 1 and kind != "kept" else None
    if kind == "append":
        st["reqs"], st["cols"] = _records(APPEND_REQ, dev, pt_off=off, row_off=_first(n),
                                          start=np.full_like(n, case["start"]),
                                          position=rng.integers(0, 1 << 17, size=len(n)), n_tokens=n)
        # queries, keys and values as one projection leaves them, side by side in a row
        rows = torch.randn(st["total"], (H * G + C * H) * D, generator=g, device=dev).to(dt)
        q, k, v = rows.split([H * G * D, H * D, (C - 1) * H * D], dim=1)
        st.update(q=q.unflatten(1, (H * G, D)), k=k.unflatten(1, (H, D)),
                  v=v.unflatten(1, (H, D)) if C == 2 else None)
        # frequencies stretched for a context 4 times as long
        j = np.arange(0, case["rot"], 2)
        st["freq"] = torch.from_numpy((10000.0 ** (-j / case["rot"]) / 4).astype(np.float32)).to(dev)
        st["amplitude"] = 0.1 * math.log(4) + 1
        st["q_out"] = torch.zeros(st["total"], H * G, D, dtype=dt, device=dev)
        return st
    if kind == "attend":
        cap = _ceil(st["most"], 64) * 64
        b = _begins(case, n)
        st["reqs"], st["cols"] = _records(ATTEND_REQ, dev, pt_off=off, acc_off=np.arange(len(n)) * (H * cap), start=b,
                                          end=n)
        st.update(q=(torch.randn(len(n), H * G, D, generator=g, device=dev) * 2).to(dt), seen=int((n - b).max()),
                  scale=(192 if C == 1 else D) ** -0.5,
                  out=torch.zeros(len(n), H * G, case["v"], dtype=dt, device=dev),
                  lse=torch.zeros(len(n), H * G, device=dev))
        if e == 1:      # queries as large as meets keys of that scale
            st["q"] = st["q"] * 8
        if case["acc"]:
            st["acc"] = torch.rand(len(n), H, cap, generator=g, device=dev) * 0.01
        return st

    m = np.minimum(n, case["keep"])
    kcap = int(m.max())
    key = torch.rand(len(n), L * H, st["most"], generator=g, device=dev)
    key.masked_fill_(torch.arange(st["most"], device=dev) >= torch.from_numpy(n).to(dev)[:, None, None], 2.0)
    kept = key.topk(kcap, largest=False, dim=2).indices
    kept.masked_fill_(torch.arange(kcap, device=dev) >= torch.from_numpy(m).to(dev)[:, None, None], 1 << 30)
    st["kept"] = kept.sort(dim=2).values.to(torch.int32)
    Nd, dpt, doff = _pages(rng, case["Td"], m)
    st.update(dspec=_spec(L, C, H, D, case["Td"], Nd, e, case["dst"]), dpt=torch.from_numpy(dpt).to(dev), most=kcap,
              total=int(m.sum()), dst=torch.zeros(L * Nd * C * case["Td"] * H * D * e, dtype=torch.uint8, device=dev))
    st["reqs"], st["cols"] = _records(MOVE_REQ, dev, src_pt_off=off, dst_pt_off=doff,
                                      buf_off=np.arange(len(n)) * (L * H * kcap), n_tokens=m)
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def _axes(pool, spec, order, dtype):
    """A pool's elements with its axes in the order of the letters l p c t h d."""
    size = dict(l=spec.L, p=spec.N, c=spec.C, t=spec.T, h=spec.H, d=spec.D)
    have = AXES[spec.layout]
    return pool.view(dtype).view([size[a] for a in have]).permute([have.index(a) for a in order])


def _bits(case):
    return torch.uint8 if case["cache"] == "e4m3" else torch.int16


def _outputs(st):
    """What a pass returns: the buffers it has written."""
    case, kind = st["case"], st["kind"]
    if kind == "append":
        return [st["q_out"], st["pool"].view(DTYPES[case["cache"]])]
    if kind == "attend":
        return [st["out"], st["lse"]] + ([st["acc"]] if case["acc"] else [])
    if kind == "select":
        return [st["kept"], st["out"].view(torch.int32)]
    return [st["dst"].view(_bits(case))]


def run(st):
    {"append": _append, "attend": _attend, "select": _select, "kept": _kept}[st["kind"]](st)
    return _outputs(st)


def _append(st):
    case, spec, cols, layer = st["case"], st["spec"], st["cols"], st["layer"]
    if own:
        from paper_2606_31093_amd import kvx
        kvx.kvx_append(st["pool"], spec, layer, st["k"], st["v"], st["pt"], st["reqs"], st["most"], q=st["q"],
                       q_out=st["q_out"], scales=st["scales"], dev_err=st["err"],
                       rope=kvx.Rope(st["freq"], case["off"], case["pairs"] == "interleaved", st["amplitude"]))
        return
    rec = torch.arange(case["n"], device=st["pt"].device).repeat_interleave(cols["n_tokens"], output_size=st["total"])
    i = torch.arange(st["total"], device=rec.device) - cols["row_off"][rec]
    slot = cols["start"][rec] + i
    page = st["pt"][cols["pt_off"][rec] + slot // spec.T].long()
    # whole turns are taken off in 64 bits: a long position times a frequency has no exact 32-bit form
    turns = (cols["position"][rec] + i).double()[:, None] * st["freq"].double() / (2 * math.pi)
    angle = ((turns - turns.floor()) * (2 * math.pi)).float()[:, None]
    cos, sin = angle.cos() * st["amplitude"], angle.sin() * st["amplitude"]

    def rotated(x):
        x = x.float()
        y = x.clone()
        o, h = case["off"], case["rot"] // 2
        at = (slice(o, o + 2 * h, 2), slice(o + 1, o + 2 * h, 2)) if case["pairs"] == "interleaved" else \
            (slice(o, o + h), slice(o + h, o + 2 * h))
        a, b = x[..., at[0]], x[..., at[1]]
        y[..., at[0]], y[..., at[1]] = a * cos - b * sin, b * cos + a * sin
        return y

    st["q_out"].copy_(rotated(st["q"]))
    kv = torch.stack([rotated(st["k"])] + ([st["v"].float()] if st["v"] is not None else []), dim=1)
    if st["scales"] is not None:
        kv = (kv / st["scales"][:, :, None]).clamp(-448, 448)
    bits = _bits(case)
    _axes(st["pool"], spec, "lptchd", bits)[layer][page, slot % spec.T] = kv.to(DTYPES[case["cache"]]).view(bits)


def _attend(st):
    case, spec, cols = st["case"], st["spec"], st["cols"]
    if own:
        from paper_2606_31093_amd import kvx
        if "workspace" not in st:     # a serving program makes it once, for its largest batch
            st["workspace"] = kvx.attend_workspace(spec, case["n"], case["H"] * case["G"], st["seen"], case["v"],
                                                   accumulate=case["acc"], device=st["q"].device)
        kvx.kvx_attend(st["q"], st["out"], st["pool"], spec, st["layer"], st["pt"], st["reqs"], st["seen"],
                       st["workspace"], scale=st["scale"], scales=st["scales"], lse=st["lse"], acc=st.get("acc"),
                       acc_stride=st["acc"].shape[2] if case["acc"] else 0, dev_err=st["err"])
        return
    n, H, G, v = case["n"], case["H"], case["G"], case["v"]
    pos = torch.arange(st["most"], device=st["pt"].device)[None]
    seen = (pos >= cols["start"][:, None]) & (pos < cols["end"][:, None])
    at = torch.minimum(pos, cols["end"][:, None] - 1)
    page = st["pt"][cols["pt_off"][:, None] + at // spec.T].long()
    bits, dt = _bits(case), DTYPES[case["cache"]]
    kv = _axes(st["pool"], spec, "lpthcd", bits)[st["layer"]][page, at % spec.T].view(dt).float()   # n, most, H, C, D
    if st["scales"] is not None:
        kv = kv * st["scales"].t()[:, :, None]
    k, val = kv[:, :, :, 0].transpose(1, 2), kv[:, :, :, -1, :v].transpose(1, 2)
    s = st["q"].float().view(n, H, G, -1) @ k.transpose(2, 3).contiguous() * st["scale"]
    s = s.masked_fill(~seen[:, None, None], -math.inf)
    m = s.max(dim=3, keepdim=True).values
    p = (s - m).exp()
    l = p.sum(dim=3, keepdim=True)
    p = p / l
    st["out"].copy_((p @ val.contiguous()).view(n, H * G, v))
    st["lse"].copy_((m + l.log()).view(n, H * G))
    if case["acc"]:
        st["acc"][:, :, :st["most"]] += p.sum(dim=2)


def _select(st):
    case, cols = st["case"], st["cols"]
    if own:
        from paper_2606_31093_amd import kvx
        kvx.kvx_select_kept(st["acc"], st["acc"].shape[2], case["L"] * case["H"], st["reqs"], st["most"], st["kept"],
                            st["kept"].shape[2], acc_out=st["out"], acc_out_stride=st["out"].shape[2],
                            dev_err=st["err"])
        return
    n, sink, recent = (cols[k][:, None, None] for k in ("n_tokens", "sink", "recent"))
    kept = torch.minimum(n, cols["n_keep"][:, None, None])
    acc = st["acc"][:, :, :st["most"]]
    pos = torch.arange(st["most"], device=acc.device)
    key = acc.masked_fill((pos < sink) | (pos >= n - recent), math.inf).masked_fill(pos >= n, -math.inf)
    order = key.sort(dim=2, descending=True, stable=True).indices
    room = min(st["kept"].shape[2], st["most"])
    order = order.masked_fill(pos >= kept, st["most"]).sort(dim=2).values[:, :, :room]
    valid = order < st["most"]
    st["kept"][:, :, :room] = torch.where(valid, order.to(torch.int32), st["kept"][:, :, :room])
    st["out"][:, :, :room] = torch.where(valid, acc.gather(2, order.clamp(max=st["most"] - 1)), st["out"][:, :, :room])


def _kept(st):
    case, spec, dspec, cols = st["case"], st["spec"], st["dspec"], st["cols"]
    if own:
        from paper_2606_31093_amd import kvx
        kvx.kvx_transfer_kept(st["pool"], spec, st["dst"], dspec, st["pt"], st["dpt"], st["reqs"], st["most"],
                              st["kept"], st["kept"].shape[2], dev_err=st["err"])
        return
    dev = st["pt"].device
    rec = torch.arange(case["n"], device=dev).repeat_interleave(cols["n_tokens"], output_size=st["total"])
    first = cols["n_tokens"].cumsum(0) - cols["n_tokens"]
    i = torch.arange(st["total"], device=dev) - first[rec]
    l, h = torch.arange(spec.L, device=dev)[:, None, None], torch.arange(spec.H, device=dev)[:, None]
    row = st["kept"].view(case["n"], spec.L, spec.H, -1)[rec, l, h, i].long()           # L, H, total
    page = st["pt"][cols["src_pt_off"][rec] + row // spec.T].long()
    to = st["dpt"][cols["dst_pt_off"][rec] + i // dspec.T].long()
    bits = _bits(case)
    _axes(st["dst"], dspec, "lpthcd", bits)[l, to, i % dspec.T, h] = \
        _axes(st["pool"], spec, "lpthcd", bits)[l, page, row % spec.T, h]


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    """Request by request from the definitions; None for what is moved or
    chosen and not computed."""
    if case["kind"] not in ("append", "attend"):
        return None
    st = prepare(case, seed)
    n = _tokens(case)
    C, H, D, G, T = (case[k] for k in ("C", "H", "D", "G", "T"))
    first = _first(-(-(n + (case["start"] if case["kind"] == "append" else 0)) // T))
    stored = st["pool"].view(DTYPES[case["cache"]]).double()
    size = dict(l=case["L"], p=st["spec"].N, c=C, t=T, h=H, d=D)
    have = AXES[case["layout"]]
    cache = stored.view([size[a] for a in have]).permute([have.index(a) for a in "lptchd"])[st["layer"]]
    unit = torch.ones(C, H, 1, dtype=torch.float64, device=stored.device)
    if st["scales"] is not None:
        unit = st["scales"].double()[:, :, None]
    if case["kind"] == "append":
        half, o = case["rot"] // 2, case["off"]
        a = torch.arange(half, device=stored.device)
        ia, ib = (o + 2 * a, o + 2 * a + 1) if case["pairs"] == "interleaved" else (o + a, o + half + a)
        row = 0
        queries = st["q"].double()
        for r, tokens in enumerate(n.tolist()):
            i = torch.arange(tokens, device=stored.device)
            z = torch.polar(torch.full((tokens, 1, half), st["amplitude"], dtype=torch.float64, device=stored.device),
                            ((st["cols"]["position"][r] + i).double()[:, None] * st["freq"].double())[:, None])

            def turn(x):
                x = x.double()
                w = torch.complex(x[..., ia], x[..., ib]) * z
                x[..., ia], x[..., ib] = w.real, w.imag
                return x
            queries[row:row + tokens] = turn(st["q"][row:row + tokens])
            new = [turn(st["k"][row:row + tokens])] + ([st["v"][row:row + tokens].double()] if C == 2 else [])
            slot = case["start"] + i
            pages = st["pt"][first[r] + slot // T].long()
            new = torch.stack(new, dim=1) / unit
            cache[pages, slot % T] = new.clamp(-448, 448) if st["scales"] is not None else new
            row += tokens
        return [queries, stored]
    begin = _begins(case, n)
    out = torch.zeros(len(n), H * G, case["v"], dtype=torch.float64, device=stored.device)
    lse = torch.zeros(len(n), H * G, dtype=torch.float64, device=stored.device)
    acc = st["acc"].double() if case["acc"] else None
    for r, tokens in enumerate(n.tolist()):
        t = torch.arange(int(begin[r]), tokens, device=stored.device)
        kv = cache[st["pt"][first[r] + t // T].long(), t % T] * unit                    # tokens, C, H, D
        for h in range(H):
            heads = slice(h * G, (h + 1) * G)
            s = st["q"][r, heads].double() @ kv[:, 0, h].t().contiguous() * st["scale"]
            lse[r, heads] = torch.logsumexp(s, dim=1)
            w = torch.exp(s - lse[r, heads, None])
            out[r, heads] = w @ kv[:, C - 1, h, :case["v"]].contiguous()
            if acc is not None:
                acc[r, h, int(begin[r]):tokens] += w.sum(dim=0)
    return [out, lse] + ([acc] if acc is not None else [])
