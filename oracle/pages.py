"""Paged 8-bit caches from their definitions, in 64 bits: codes, scales, tables, attention.

Plain numpy, one token, page or row after the other.  A cache is a dict with k, v (uint8 codes [L][pages][Hkv][ps][hd]), k_scale,
v_scale (float32 [L][pages][Hkv]), table (int32 [sequences][blocks]) and ref (int32 [pages]).
"""
from __future__ import annotations

import math

import numpy as np

# the 256 values of e4m3: sign, 4 bits of exponent (bias 7), 3 of mantissa, no infinities, 0x7F and 0xFF not numbers
_c = np.arange(256)
_e, _m = (_c >> 3) & 15, _c & 7
VALUES = np.where(_e == 0, _m / 8.0 * 2.0 ** -6, (1 + _m / 8.0) * 2.0 ** (_e - 7.0)) * np.where(_c < 128, 1.0, -1.0)
VALUES[[0x7F, 0xFF]] = np.nan
LARGEST = 448.0


def decode(codes):
    return VALUES[codes]


def encode(x):
    """The nearest code (ties to the even mantissa), saturating; NaN becomes 0x7F."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(x)
    pos = VALUES[:0x7F]                                         # ascending
    hi = np.clip(np.searchsorted(pos, a), 1, 0x7E)
    lo = hi - 1
    mid = (pos[lo] + pos[hi]) / 2
    up = (a > mid) | ((a == mid) & (hi % 2 == 0))
    code = np.where(up, hi, lo)
    code = np.where(a >= LARGEST, 0x7E, code)
    code = np.where(np.isnan(x), 0x7F, code)
    return np.where(np.signbit(x), code | 0x80, code).astype(np.uint8)


def least_scale(amax):
    """The least 2^e, -126 <= e <= 120, with amax <= 448 2^e."""
    e = -126
    while e < 120 and LARGEST * 2.0 ** e < amax:
        e += 1
    return 2.0 ** e


def rotate(x, positions, sections, theta):
    """x [tokens][heads][hd]; positions [axes][tokens].  Pair (i, i + hd/2) turns by positions[axis of i] theta^(-2i/hd)."""
    x = np.asarray(x, dtype=np.float64)
    hd = x.shape[-1]
    half = hd // 2
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    out = np.empty_like(x)
    for i in range(half):
        ang = np.asarray(positions)[axis[i]].astype(np.float64) * float(theta) ** (-2.0 * i / hd)
        c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
        out[..., i] = x[..., i] * c - x[..., i + half] * s
        out[..., i + half] = x[..., i + half] * c + x[..., i] * s
    return out


def append(cache, layer, k, v, seq, first, start):
    """k, v [tokens][Hkv][hd] in 64 bits, rotated already."""
    ps = cache["k"].shape[3]
    for e, s in enumerate(seq):
        t, pos = first[e], start[e]
        while t < first[e + 1]:
            off = pos % ps
            n = min(ps - off, first[e + 1] - t)
            page = cache["table"][s, pos // ps]
            for x, name in ((k, "k"), (v, "v")):
                codes, scale = cache[name][layer, page], cache[name + "_scale"][layer, page]
                for h in range(codes.shape[0]):
                    new = np.where(np.isnan(x[t:t + n, h]), 0.0, x[t:t + n, h])
                    sc = least_scale(np.abs(np.where(np.isinf(new), 0.0, new)).max())
                    if off:
                        sc = max(sc, float(scale[h]))
                        codes[h, :off] = encode(decode(codes[h, :off]) * (float(scale[h]) / sc))
                    codes[h, off:off + n] = encode(new / sc)
                    scale[h] = sc
            t, pos = t + n, pos + n


def gather(cache, layer, seq, length, name):
    """[Hkv][length][hd]"""
    ps = cache["k"].shape[3]
    got = [decode(cache[name][layer, cache["table"][seq, j // ps], :, j % ps]) * cache[name + "_scale"][layer, cache["table"][seq, j // ps]].astype(np.float64)[:, None]
           for j in range(length)]
    return np.stack(got, axis=1) if got else np.zeros((cache["k"].shape[2], 0, cache["k"].shape[4]))


def seen(rows, length, prefix=0, tree=None):
    """[rows][length]: which positions a row sees."""
    i, j = np.arange(rows)[:, None], np.arange(length)[None]
    base = length - rows
    if tree is None:
        ok = j <= base + i
    else:
        ok = (j < base) | ((j >= base) & ((np.asarray([int(b) & (2 ** 64 - 1) for b in tree], dtype=object)[:, None] >> np.maximum(j - base, 0).astype(object)) % 2 == 1))
        ok = ok.astype(bool)
    return ok | (j < prefix)


def attention(q, K, V, scale, mask, softcap=0.0, slopes=None):
    """q [rows][H][hd], K, V [Hkv][length][hd], mask [rows][length].  Returns the output, the weighted mean of |V|, and a bound of
    the terms of the scores (both [rows][H][...]) for what depends on their sizes."""
    rows, H, hd = q.shape
    length = K.shape[1]
    out, size, terms = np.zeros((rows, H, hd)), np.zeros((rows, H, hd)), np.zeros((rows, H, 1))
    here = length - rows + np.arange(rows)
    for h in range(H):
        kh, vh = K[h // (H // K.shape[0])], V[h // (H // K.shape[0])]
        for i in range(rows):
            at = np.flatnonzero(mask[i])
            if at.size == 0:
                continue
            s = kh[at] @ q[i, h] * scale
            big = (np.abs(kh[at]) @ np.abs(q[i, h])).max() * scale
            if softcap:
                s = softcap * np.tanh(s / softcap)
                big += softcap
            if slopes is not None:
                d = float(slopes[h]) * np.abs(here[i] - at)
                s, big = s - d, big + d.max()
            w = np.exp(s - s.max())
            w /= w.sum()
            out[i, h], size[i, h], terms[i, h] = w @ vh[at], w @ np.abs(vh[at]), big
    return out, size, terms


def fork(cache, src, dst, keep, length):
    """Returns whether the pages sufficed."""
    table, ref, ps = cache["table"], cache["ref"], cache["k"].shape[3]
    old, was = table.copy(), {x: cache[x].copy() for x in ("k", "v", "k_scale", "v_scale")}
    named = np.zeros(len(ref), dtype=np.int64)                  # references after the sharing and the giving back
    named += ref
    for s, d, n in zip(src, dst, keep):
        for b in range(n // ps):
            named[old[s, b]] += 1
        for page in old[d]:
            if page >= 0:
                named[page] -= 1
    stays, claimed = [], set()                                  # of several that nobody but they named, the first entry keeps the page
    for s, d, n in zip(src, dst, keep):
        tail = int(old[s, n // ps]) if n % ps else -1
        stays.append(tail >= 0 and s == d and named[tail] == 0 and tail not in claimed)
        if stays[-1]:
            claimed.add(tail)
    pinned = {int(old[s, n // ps]) for s, d, n in zip(src, dst, keep) if n % ps}
    free = [p for p in range(len(ref)) if named[p] == 0 and p not in pinned]
    enough = True
    for s, d, n, m, stay in zip(src, dst, keep, length, stays):
        full = n // ps
        row = [int(old[s, b]) for b in range(full)]
        if stay:
            row.append(int(old[s, full]))
            named[row[-1]] += 1
        for b in range(full + stay, -(-m // ps)):
            if not free:
                enough = False
                row.append(-1)
                continue
            page = free.pop(0)
            named[page] += 1
            row.append(page)
            if b == full and n % ps:
                for x in ("k", "v"):
                    cache[x][:, page, :, :n % ps] = was[x][:, old[s, full], :, :n % ps]
                    cache[x + "_scale"][:, page] = was[x + "_scale"][:, old[s, full]]
        table[d] = -1
        table[d, :len(row)] = row
    ref[:] = named
    return enough


def compact(cache, seq, start, count, index):
    ps = cache["k"].shape[3]
    table = cache["table"]
    for e, s in enumerate(seq):
        i = 0
        while i < count[e]:
            to = start[e] + i
            off = to % ps
            n = min(ps - off, count[e] - i)
            page = table[s, to // ps]
            of = [(table[s, x // ps], x % ps) for x in index[e][i:i + n]]
            for name in ("k", "v"):
                codes, scale = cache[name], cache[name + "_scale"]
                for layer in range(codes.shape[0]):
                    for h in range(codes.shape[2]):
                        sc = max(float(scale[layer, p, h]) for p, _ in of)
                        if off:
                            sc = max(sc, float(scale[layer, page, h]))
                        new = [encode(decode(codes[layer, p, h, r]) * (float(scale[layer, p, h]) / sc)) for p, r in of]
                        if off:
                            codes[layer, page, h, :off] = encode(decode(codes[layer, page, h, :off]) * (float(scale[layer, page, h]) / sc))
                        codes[layer, page, h, off:off + n] = new
                        scale[layer, page, h] = sc
            i += n
