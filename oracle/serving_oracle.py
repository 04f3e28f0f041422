"""What surrounds a decoder's attention in a server, in numpy and 64 bits, written from the formulas: rows in 4 bits, rotary
positions, the life of a cache's pages. Test infrastructure, CPU only."""
from __future__ import annotations

import math
from fractions import Fraction

import numpy as np

GROUP = 32


def scale4(amax: float) -> float:
    """The least number of 4 significant bits s with amax <= 7 s, within 2^-126 and 1.125 * 2^125."""
    least, most = 2.0 ** -126, 1.125 * 2.0 ** 125
    if amax <= 7 * least:
        return least
    e = math.frexp(amax / 7)[1] - 4                 # amax / 7 is 8 to 16 times 2^e
    for m in (7.5, 8, 9, 10, 11, 12, 13, 14, 15, 16, 18):
        s = m * 2.0 ** e
        if amax <= 7 * s:
            return min(max(s, least), most)
    raise AssertionError(amax)


def quantise4(x: np.ndarray):
    """Rows [..., D] -> (bytes [..., D / 2], scales [..., ceil(D / 32)], values [..., D])."""
    x = np.asarray(x, np.float64)
    D = x.shape[-1]
    rows = x.reshape(-1, D)
    codes, scales = np.zeros(rows.shape, np.int64), np.zeros((rows.shape[0], -(-D // GROUP)))
    values = np.zeros(rows.shape)
    for r, row in enumerate(rows):
        for g in range(scales.shape[1]):
            part = row[g * GROUP: (g + 1) * GROUP]
            to = slice(g * GROUP, g * GROUP + len(part))
            if not np.isfinite(part).all():
                scales[r, g] = values[r, to] = np.nan
                continue
            s = scale4(float(np.abs(part).max()))
            c = np.clip(np.rint(part / s), -7, 7)          # a 24-bit number over a 4-bit one: no quotient lies within 2^-30 of a half
            codes[r, to], scales[r, g], values[r, to] = c, s, c * s
    packed = (codes[:, 0::2] + 8) | (codes[:, 1::2] + 8) << 4
    return (packed.astype(np.uint8).reshape(x.shape[:-1] + (D // 2,)), scales.reshape(x.shape[:-1] + (-1,)), values.reshape(x.shape))


def bf16_bits(x: np.ndarray) -> np.ndarray:
    """Bits of numbers that bf16 holds exactly; NaN as 0x7fff."""
    b = (np.asarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7FFF), b)


def frequencies(rot, base=10000.0, scaling="none", factor=1.0, original_len=0.0, low=1.0, high=32.0, divisors=None):
    """f_i of rotary positions."""
    out = []
    for i in range(rot // 2):
        t = base ** (-2.0 * i / rot)
        if scaling == "none":
            f = t
        elif scaling == "linear":
            f = t / factor
        else:
            if scaling == "by_turns":
                g = (original_len * t / (2 * math.pi) - low) / (high - low)
            else:
                def index(turns):
                    return rot * math.log(original_len / (2 * math.pi * turns)) / (2 * math.log(base))
                a, z = max(math.floor(index(high)), 0), min(math.ceil(index(low)), rot - 1)
                g = 1 - (i - a) / ((z if z != a else a + 0.001) - a)
            g = min(max(g, 0.0), 1.0)
            f = t * (g + (1 - g) / factor)
        out.append(f / (divisors[i] if divisors is not None else 1.0))
    return np.array(out)


PI = Fraction("3.14159265358979323846264338327950288419716939937510")


def rotate(x, positions, freq, layout="half", magnitude=1.0, inverse=False):
    """Rows [T, H, D] turned; angles without their whole turns by exact fractions, so that far positions lose nothing."""
    x = np.array(x, np.float64)
    R = 2 * len(freq)
    angle = np.array([[float((int(p) * Fraction(float(f)) / (2 * PI)) % 1) for f in freq] for p in positions]) * 2 * math.pi
    c, s = np.cos(angle)[:, None] * magnitude, np.sin(angle)[:, None] * magnitude * (-1 if inverse else 1)
    a, b = (slice(0, R // 2), slice(R // 2, R)) if layout == "half" else (slice(0, R, 2), slice(1, R, 2))
    u, w = x[..., a].copy(), x[..., b].copy()
    x[..., a], x[..., b] = u * c - w * s, u * s + w * c
    return x


def fork(table, lens, parents, refs, page):
    """(new table, new lens, new refs), row by row."""
    refs = refs.copy()
    new, new_lens = np.full((len(parents), table.shape[1]), -1, np.int32), np.zeros(len(parents), np.int32)
    for row in table:
        for x in row[row >= 0]:
            refs[x] -= 1
    for b, p in enumerate(parents):
        if p >= 0:
            n = -(-int(lens[p]) // page)
            new[b, :n], new_lens[b] = table[p, :n], lens[p]
            for x in new[b, :n]:
                refs[x] += 1
    return new, new_lens, refs


def reserve(table, lens, grow, refs, page):
    """(table, refs, missing, moves): request after request, as the free pages are at the beginning; moves are (from, to, rows)."""
    new, now, moves = table.copy(), refs.copy(), []
    free = [int(x) for x in np.nonzero(refs == 0)[0]]
    asked = 0

    def take():
        nonlocal asked
        asked += 1
        return free[asked - 1] if asked <= len(free) else None
    for b in range(len(lens)):
        if grow[b] == 0:
            continue
        first, end = -(-int(lens[b]) // page), -(-int(lens[b] + grow[b]) // page)
        if lens[b] % page:
            x = new[b, first - 1]
            if now[x] > 1:
                y = take()
                now[x] -= 1
                if y is not None:
                    moves.append((int(x), y, int(lens[b] % page)))
                    new[b, first - 1], now[y] = y, 1
        for i in range(first, end):
            if new[b, i] < 0:
                y = take()
                if y is not None:
                    new[b, i], now[y] = y, 1
    if asked > len(free):
        return table.copy(), refs.copy(), asked - len(free), []
    return new, now, 0, moves


def compact(table, refs):
    """(table, refs, pages in use, their places, moves)."""
    n = int((refs > 0).sum())
    high = [x for x in range(n, len(refs)) if refs[x] > 0]
    low = [x for x in range(n) if refs[x] == 0]
    at = np.where(refs > 0, np.arange(len(refs)), -1).astype(np.int32)
    refs = refs.copy()
    for a, b in zip(high, low):
        at[a], refs[b], refs[a] = b, refs[a], 0
    return np.where(table >= 0, at[table], -1).astype(np.int32), refs, n, at, list(zip(high, low))
