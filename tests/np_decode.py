"""The decode step's operators from their definitions, in 64 bits and element
by element of the page tables, in numpy.  Shares no code with the library."""
import numpy as np

ORDER = {"LPCTHD": "lpcthd", "LPCHTD": "lpchtd", "PLCTHD": "plcthd", "PLCHTD": "plchtd"}


def e4m3_values():
    """The value of each of the 256 e4m3 codes: 1 sign, 4 exponent (bias 7) and 3
    mantissa bits, no infinities, 0x7f and 0xff NaN."""
    out = np.zeros(256)
    for code in range(256):
        sign, exp, man = -1.0 if code & 128 else 1.0, code >> 3 & 15, code & 7
        if exp == 15 and man == 7:
            out[code] = np.nan
        elif exp == 0:
            out[code] = sign * man / 8 * 2.0 ** -6
        else:
            out[code] = sign * (1 + man / 8) * 2.0 ** (exp - 7)
    return out


E4M3 = e4m3_values()


def bf16_bits(x):
    """float64 -> bfloat16 bits, nearest even (through float32, whose own rounding of
    these inputs is exact enough: they are made as float32)."""
    b = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return ((b + 0x7FFF + ((b >> 16) & 1)) >> 16).astype(np.uint16)


def bits(x, kind):
    return bf16_bits(x) if kind == "bf16" else np.asarray(x, np.float16).view(np.uint16)


def values(b, kind):
    """Stored bits as float64."""
    if kind == "e4m3":
        return E4M3[np.asarray(b, np.uint8)]
    b = np.asarray(b, np.uint16)
    if kind == "f16":
        return b.view(np.float16).astype(np.float64)
    return (b.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def canonical(pool, spec):
    """A view of a pool's elements with axes l, p, c, t, h, d."""
    size = dict(l=spec.L, p=spec.N, c=spec.C, t=spec.T, h=spec.H, d=spec.D)
    have = ORDER[spec.layout]
    a = pool.view(np.uint8 if spec.e == 1 else np.uint16).reshape([size[x] for x in have])
    return a.transpose([have.index(x) for x in "lpcthd"])


def resolve(pt, pt_off, pos, T, N):
    """(page, slot), or None where the table or the page is out of range."""
    i = pt_off + pos // T
    if not 0 <= i < len(pt) or not 0 <= pt[i] < N:
        return None
    return int(pt[i]), pos % T


def rotate(x, position, freq, off, interleaved, amplitude):
    """x[..., d] in float64, rotated for a position."""
    y = x.copy()
    half = len(freq)
    for j in range(half):
        a, b = (off + 2 * j, off + 2 * j + 1) if interleaved else (off + j, off + j + half)
        ang = float(position) * float(freq[j])
        c, s = amplitude * np.cos(ang), amplitude * np.sin(ang)
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y


def attend(q, cache, spec, layer, pt, rows, scale, v_dim, scales=None):
    """q [n, Hq, D] float64, cache the canonical values in float64.  For every
    record (pt_off, acc_off, start, end): out, lse, the weights [H, positions]
    summed over the group, and the size of the sums that rounding acts on:
    sum w |v| (as out), and the largest sum |q k| * scale."""
    n, Hq, D = q.shape
    G = Hq // spec.H
    out, lse = np.zeros((n, Hq, v_dim)), np.full((n, Hq), -np.inf)
    mag, dots, weights = np.zeros((n, Hq, v_dim)), np.zeros(n), []
    for r, (pt_off, _, start, end) in enumerate(rows):
        at = [resolve(pt, pt_off, t, spec.T, spec.N) for t in range(start, end)]
        use = [i for i, a in enumerate(at) if a is not None]
        w_all = np.zeros((spec.H, end - start))
        if use:
            k = np.stack([cache[layer, at[i][0], 0, at[i][1]] for i in use])                 # t, H, D
            v = np.stack([cache[layer, at[i][0], spec.C - 1, at[i][1]] for i in use])[..., :v_dim]
            if scales is not None:
                k, v = k * scales[0][:, None], v * scales[spec.C - 1][:, None]
            for hq in range(Hq):
                h = hq // G
                s = scale * (k[:, h] @ q[r, hq])
                dots[r] = max(dots[r], scale * float((np.abs(k[:, h]) @ np.abs(q[r, hq])).max()))
                m = s.max()
                p = np.exp(s - m)
                l = p.sum()
                out[r, hq], lse[r, hq] = p @ v[:, h] / l, m + np.log(l)
                mag[r, hq] = p @ np.abs(v[:, h]) / l
                w_all[h, use] += p / l
        weights.append(w_all)
    return out, lse, weights, mag, dots


def select(w, n_keep, sink, recent):
    """Kept positions of one list, ascending."""
    n = len(w)
    if n <= n_keep:
        return list(range(n))
    mid = range(sink, n - recent)
    key = [(-np.inf, 1) if np.isnan(x) else (float(x), 0) for x in w]
    # NaN below -inf; ties to the lower position
    best = sorted(mid, key=lambda t: (-key[t][0] if key[t][0] != -np.inf else np.inf, key[t][1], t))
    return sorted(list(range(sink)) + best[:n_keep - sink - recent] + list(range(n - recent, n)))
