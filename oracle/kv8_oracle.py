"""ORACLE -- test infrastructure only (tests/ may use it; the product never does).  Plain NumPy, slow and obvious.

Serving a batch from a paged 8-bit key/value cache, written out from the definitions in include/aq.h:

    plan          lengths, tables and row maps of a step, from the requests' lengths
    rope_rows     rotary positions of rows: both pairings, part of a head, the forms for long contexts (float64)
    append        the quantising append, one block of 32 positions after another (binary32 steps as defined, so codes are exact)
    gather        a request's cached values (float64)
    attn          attention of one query row over its positions (float64), and what its tolerance is made of

Cache: codes int8 [n_pages][Hkv][page][D], scales float32 [n_pages][Hkv][page / 32].
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 32


def plan(lens, new, table, free, page, n_rows, free_cap):
    """Lists; table a list of lists (a copy is returned), free the stack.  Returns (lens, table, free, row_start, pos), or None where
    the step does not fit."""
    lens, table, free = list(lens), [list(r) for r in table], list(free)
    before, pos, row_start = list(lens), [], [0]
    if any(n < -1 or m < 0 for n, m in zip(new, lens)) or any(m > len(r) * page for m, r in zip(lens, table)):
        return None
    for b, n in enumerate(new):
        if n < 0:
            free += table[b][: -(-lens[b] // page)]
            lens[b] = 0
    if len(free) > free_cap:
        return None
    for b, n in enumerate(new):
        if n < 0:
            row_start.append(row_start[-1])
            continue
        if lens[b] + n > len(table[b]) * page:
            return None
        for i in range(-(-lens[b] // page), -(-(lens[b] + n) // page)):
            if not free:
                return None
            table[b][i] = free.pop()
        pos += range(lens[b], lens[b] + n)
        lens[b] += n
        row_start.append(row_start[-1] + n)
    if len(pos) > n_rows:
        return None
    assert all(l >= 0 for l in lens) and len(before) == len(lens)
    return lens, table, free, row_start, pos + [-1] * (n_rows - len(pos))


def rope_frequencies(rot, theta=10000.0, scaling="none", factor=1.0, trained=0.0, low=1.0, high=32.0):
    f = []
    for i in range(rot // 2):
        base = theta * factor ** (rot / (rot - 2)) if scaling == "base" and rot > 2 else theta
        x = base ** (-2.0 * i / rot)
        if scaling == "linear":
            x /= factor
        elif scaling == "parts":
            turns = trained * x / (2 * math.pi)
            keep = 1.0 if turns >= high else 0.0 if turns <= low else (turns - low) / (high - low)
            x = x * keep + x / factor * (1 - keep)
        f.append(x)
    return np.array(f)


def rope_rows(x, pos, f, layout, magnitude=1.0):
    """x [T][H][D] -> float64; rows with a negative position as they are."""
    x = np.array(x, dtype=np.float64)
    out = x.copy()
    for t, p in enumerate(pos):
        if p < 0:
            continue
        for i, w in enumerate(f):
            a, b = (i, i + len(f)) if layout == "half" else (2 * i, 2 * i + 1)
            c, s = magnitude * math.cos(p * w), magnitude * math.sin(p * w)
            out[t, :, a] = x[t, :, a] * c - x[t, :, b] * s
            out[t, :, b] = x[t, :, b] * c + x[t, :, a] * s
    return out


def up11(y):
    """The next number of 11 significant bits not below y >= 0 (float32 in, float32 out)."""
    m, e = math.frexp(float(y))
    return np.float32(math.ldexp(math.ceil(m * 2048), e - 11))


def _rint(x):
    return np.rint(x)   # ties to even


def append_block(codes, scale, at, x):
    """One block of one head: codes int8 [32][D], its scale, the place of the first new row, the new rows float32 [n][D].
    Returns (codes, scale)."""
    codes, x = codes.copy(), np.asarray(x, dtype=np.float32)
    n = x.shape[0]
    old = np.float32(0 if at == 0 else scale)
    if not np.all(np.isfinite(x)) or np.isnan(old):
        codes[at: at + n] = 0
        return codes, np.float32(np.nan)
    need = up11(np.float32(np.max(np.abs(x))) / np.float32(127))
    s = old if need <= old else max(need, up11(np.float32(1.25) * old))
    codes[at: at + n] = _rint(x / s).astype(np.int8) if s > 0 else 0
    if at > 0 and s > old:
        codes[:at] = _rint((codes[:at].astype(np.float32) * old) / s).astype(np.int8)
    return codes, np.float32(s)


def append(k, ks, v, vs, lens, row_start, table, new_k, new_v):
    """Arrays as in the cache; returns the cache's four arrays after the step."""
    k, ks, v, vs = k.copy(), ks.copy(), v.copy(), vs.copy()
    page = k.shape[2]
    for b, L in enumerate(lens):
        row, p = row_start[b], L - (row_start[b + 1] - row_start[b])
        while p < L:
            upto = min(L, (p // BLOCK + 1) * BLOCK)
            n = upto - p
            if p >= 0:
                pg, j, at = table[b][p // page], p % page // BLOCK, p % BLOCK
                for codes, scales, x in ((k, ks, new_k), (v, vs, new_v)):
                    for h in range(k.shape[1]):
                        here = slice(j * BLOCK, (j + 1) * BLOCK)
                        codes[pg, h, here], scales[pg, h, j] = append_block(codes[pg, h, here], scales[pg, h, j], at, x[row: row + n, h])
            row, p = row + n, upto
    return k, ks, v, vs


def gather(codes, scales, pages, L):
    """[Hkv][L][D] float64 of a request."""
    page = codes.shape[2]
    n = -(-L // page)
    c = codes[pages[:n]].astype(np.float64) * np.repeat(scales[pages[:n]].astype(np.float64), BLOCK, axis=2)[..., None]
    return np.moveaxis(c, 0, 1).reshape(codes.shape[1], n * page, codes.shape[3])[:, :L]


def attn(q, K, V, scale):
    """q [D]; K, V [L][D] float64, the positions that the row sees.  Returns (out, sum_p w|V|, weights)."""
    if K.shape[0] == 0:
        z = np.zeros(V.shape[1])
        return z, z, np.zeros(0)
    s = (K @ q) * scale
    w = np.exp(s - s.max())
    w /= w.sum()
    return w @ V, w @ np.abs(V), w
