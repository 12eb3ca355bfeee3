"""Several tokens of a request over a paged cache, from the definitions, in 64
bits and element by element of the page tables, in numpy.  Shares no code with the
library."""
import numpy as np

from np_decode import resolve


def norm(x, weight, off, eps):
    """x[..., d] in float64 with elements off .. normed."""
    y = x.copy()
    n = slice(off, off + len(weight))
    y[..., n] = x[..., n] * weight / np.sqrt((x[..., n] ** 2).mean(axis=-1, keepdims=True) + eps)
    return y


def rotate(x, positions, freq, off, interleaved, amplitude):
    """x[..., d] in float64, pair j rotated for positions[j]."""
    y = x.copy()
    half = len(freq)
    for j in range(half):
        a, b = (off + 2 * j, off + 2 * j + 1) if interleaved else (off + j, off + j + half)
        ang = float(positions[j]) * float(freq[j])
        c, s = amplitude * np.cos(ang), amplitude * np.sin(ang)
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y


def depths(bits, n):
    return [max(0, bin(int(b) & ((1 << n) - 1)).count("1") - 1) for b in bits[:n]]


def sees(rec, i, t, window, tree):
    """Whether query i of (pt_off, row_off, start, end, n, prefix) sees position t, and
    their distance."""
    _, row, start, end, n, prefix = rec
    base = end - n
    if tree is None:
        p, at, ok = base + i, t, t <= base + i or t < prefix
    else:
        d = depths(tree[row:row + n], n)
        p = base + d[i]
        at = t if t < base else base + d[t - base]
        ok = t < base or bool(int(tree[row + i]) >> (t - base) & 1)
    return ok and start <= t < end and (not window or p - at < window), abs(p - at)


def attend(q, cache, spec, layer, pt, recs, scale, v_dim, scales=None, cap=0.0, slopes=None, window=0, tree=None):
    """q [rows, Hq, D] float64, cache the canonical values in float64.  Returns out,
    lse, whether a row belongs to a record, and the sizes that rounding acts on: sum w
    |v| (as out), by row the largest sum |q k| * scale and |s| + bias, and sum |v| of the
    positions seen (as out)."""
    rows, Hq, D = q.shape
    G = Hq // spec.H
    out, lse = np.zeros((rows, Hq, v_dim)), np.full((rows, Hq), -np.inf)
    mag, dots, size = np.zeros((rows, Hq, v_dim)), np.zeros(rows), np.zeros(rows)
    mine, sums = np.zeros(rows, bool), np.zeros((rows, Hq, v_dim))
    for rec in recs:
        pt_off, row, start, end, n, prefix = rec
        at = [resolve(pt, pt_off, t, spec.T, spec.N) for t in range(start, end)]
        here = [t for t, a in zip(range(start, end), at) if a is not None]
        mine[row:row + n] = True
        if not here:
            continue
        k = np.stack([cache[layer, at[t - start][0], 0, at[t - start][1]] for t in here])                    # t, H, D
        v = np.stack([cache[layer, at[t - start][0], spec.C - 1, at[t - start][1]] for t in here])[..., :v_dim]
        if scales is not None:
            k, v = k * scales[0][:, None], v * scales[spec.C - 1][:, None]
        for i in range(n):
            pairs = [sees(rec, i, t, window, tree) for t in here]
            use = np.array([a for a, _ in pairs])
            far = np.array([d for _, d in pairs], np.float64)
            if not use.any():
                continue
            for hq in range(Hq):
                h = hq // G
                ku, vu = k[use][:, h], v[use][:, h]
                s = scale * (ku @ q[row + i, hq])
                dots[row + i] = max(dots[row + i], abs(scale) * float((np.abs(ku) @ np.abs(q[row + i, hq])).max()))
                if cap:
                    s = cap * np.tanh(s / cap)
                size[row + i] = max(size[row + i], float(np.abs(s).max()))
                if slopes is not None:
                    s = s - float(slopes[hq]) * far[use]
                    size[row + i] = max(size[row + i], float(np.abs(s).max()), abs(float(slopes[hq])) * far[use].max())
                m = s.max()
                p = np.exp(s - m)
                l = p.sum()
                out[row + i, hq], lse[row + i, hq] = p @ vu / l, m + np.log(l)
                mag[row + i, hq] = p @ np.abs(vu) / l
                sums[row + i, hq] = np.abs(vu).sum(axis=0)
    return out, lse, mine, mag, dots, size, sums
