"""The attention sublayer's operators in fp64 (numpy): rotary positions, the
append to a paged cache, and attention of new tokens over it.

Section 4.1's far-skip window runs the next layer's attention; these are its
parts, from their definitions.
"""

import math

import numpy as np

from .layer import checkpoint, restore


def frequencies(rot, base=10000.0, scaling="plain", factor=1.0, trained=0.0, low=1.0, high=4.0):
    """Radians a position of each of the rot / 2 pairs."""
    out = []
    for i in range(rot // 2):
        b = base * factor ** (rot / (rot - 2)) if scaling == "base" else base
        f = math.exp(-2 * i / rot * math.log(b))
        if scaling == "linear":
            f = f / factor
        if scaling == "parts":
            turns = trained / (2 * math.pi / f)
            g = (turns - low) / (high - low)
            g = 0.0 if g < 0 else 1.0 if g > 1 else g
            f = f * g + f / factor * (1 - g)
        out.append(f)
    return np.array(out, np.float64)


def pairs(rot, layout, first=0):
    """Columns (a, b) of each pair."""
    i = np.arange(rot // 2)
    return (first + i, first + i + rot // 2) if layout == "halves" else (first + 2 * i, first + 2 * i + 1)


def rotary(x, positions, freqs, layout="halves", first=0, mscale=1.0, back=False):
    """x [tokens, heads, d] with its pairs turned."""
    a, b = pairs(2 * len(freqs), layout, first)
    t = np.asarray(positions, np.float64)[:, None] * np.asarray(freqs)
    c, s = mscale * np.cos(t)[:, None], mscale * np.sin(t)[:, None] * (-1 if back else 1)
    out = np.array(x, np.float64)
    out[..., a], out[..., b] = c * x[..., a] - s * x[..., b], s * x[..., a] + c * x[..., b]
    return out


def place(table, pages, page_size, seq, pos):
    """(page, place) of a token, or None where there is a hole."""
    slot = pos // page_size
    if slot >= table.shape[1] or not 0 <= table[seq, slot] < pages:
        return None
    return int(table[seq, slot]), int(pos % page_size)


def append(cache, rows, seqs, positions, table):
    """cache [pages, heads, page_size, d] with rows [tokens, heads, d] put in their
    places (a new array)."""
    out = np.array(cache)
    for t, (b, p) in enumerate(zip(seqs, positions)):
        if p < 0 or not 0 <= b < table.shape[0]:
            continue
        at = place(table, cache.shape[0], cache.shape[2], b, p)
        if at is not None:
            out[at[0], :, at[1]] = rows[t]
    return out


def coded(rows):
    """Codes and scale bytes of rows [..., d]."""
    c, s = checkpoint(rows.reshape(-1, rows.shape[-1]))
    return c.reshape(rows.shape), s.reshape(*rows.shape[:-1], -1)


def decoded(codes, scales):
    """The values that codes [..., d] stand for."""
    return restore(codes.reshape(-1, codes.shape[-1]), scales.reshape(-1, scales.shape[-1])).reshape(codes.shape)


def attention(q, k, v, lengths, table, new=1, scale=1.0, window=0):
    """out, lse, and for error bounds the sums of |weight v| and of |q k| (the
    largest over a row's tokens), of queries [sequences * new, heads, d] over
    caches k, v [pages, kv_heads, page_size, d]."""
    tokens, heads, d = q.shape
    pages, kv, size = k.shape[:3]
    group = heads // kv
    out, lse = np.zeros((tokens, heads, d)), np.full((tokens, heads), -np.inf)
    mass, reach = np.zeros((tokens, heads, d)), np.zeros((tokens, heads))
    for b in range(tokens // new):
        n = min(max(int(lengths[b]), 0), table.shape[1] * size)
        for i in range(new):
            at = n - new + i
            first = max(0, at - window + 1) if window else 0
            places = [place(table, pages, size, b, j) for j in range(first, at + 1)]
            places = [p for p in places if p is not None]
            if not places:
                continue
            pg, pl = (np.array(x) for x in zip(*places))
            for h in range(heads):
                kk, vv = k[pg, h // group, pl], v[pg, h // group, pl]
                t = b * new + i
                s = scale * (kk @ q[t, h])
                top = s.max()
                with np.errstate(invalid="ignore"):
                    e = np.exp(s - top)
                w = e / e.sum()
                out[t, h], lse[t, h] = w @ vv, top + math.log(e.sum()) if top > -np.inf else -np.inf
                mass[t, h] = w @ np.abs(vv)
                reach[t, h] = abs(scale) * (np.abs(kk) @ np.abs(q[t, h])).max()
    return out, lse, mass, reach
