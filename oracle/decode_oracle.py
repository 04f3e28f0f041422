"""The speculative decode step's operators in numpy and 64 bits, written from their formulas: the fp8 rows of
the cache, attention for trees of drafted tokens, verification. Test infrastructure, CPU only."""
from __future__ import annotations

import numpy as np


def e4m3_values() -> np.ndarray:
    """The value of each of the 256 e4m3 codes: sign, 4 exponent bits (bias 7), 3 of mantissa; 0x7f is NaN."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * 2.0 ** (e - 7.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c >> 7 == 1, -v, v)


def quantise_rows(x: np.ndarray):
    """Rows [..., D] -> (codes, scale bytes, values): e the smallest integer >= -126 with max finite |x| <= 448 * 2^e,
    codes of x * 2^-e rounded to nearest even, NaN for what is not finite."""
    x = np.asarray(x, np.float64)
    fine = np.isfinite(x)
    amax = np.where(fine, np.abs(x), 0.0).max(-1)
    e = np.full(amax.shape, -126)
    while (over := amax > 448.0 * np.ldexp(1.0, e)).any():
        e = np.where(over, e + 1, e)
    y = np.where(fine, x, 0.0) * np.ldexp(1.0, -e)[..., None]
    pos = e4m3_values()[:127]                       # ascending
    a = np.abs(y)
    hi = np.clip(np.searchsorted(pos, a), 0, 126)
    lo = np.clip(hi - 1, 0, 126)
    d_hi, d_lo = np.abs(pos[hi] - a), np.abs(a - pos[lo])
    code = np.where((d_lo < d_hi) | ((d_lo == d_hi) & (lo % 2 == 0)), lo, hi)
    code = np.where(np.signbit(x), code | 128, code)
    code = np.where(fine, code, 127)
    return code.astype(np.uint8), (e + 127).astype(np.uint8), e4m3_values()[code] * np.ldexp(1.0, e)[..., None]


def ancestors(parents) -> np.ndarray:
    """[n, n] bool: node i sees itself and its ancestors; a parent that is not below its node is none."""
    n = len(parents)
    sees = np.zeros((n, n), bool)
    for i in range(n):
        j = i
        while j >= 0:
            sees[i, j] = True
            p = int(parents[j])
            j = p if 0 <= p < j else -1
    return sees


def mask_words(sees: np.ndarray, words: int) -> np.ndarray:
    """[n, m] bool -> [n, words] uint64."""
    out = np.zeros((sees.shape[0], words), np.uint64)
    for i, j in zip(*np.nonzero(sees)):
        out[i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return out


def tree_attention(q, k, v, length: int, sees, scale: float):
    """One request: q [n, Hq, D], k and v [length + n, H, D], sees [n, n] -> (out [n, Hq, D], lse [n, Hq]).
    Only the rows that a node sees are read."""
    n, Hq, D = q.shape
    G = Hq // k.shape[1]
    out, lse = np.zeros((n, Hq, D)), np.full((n, Hq), -np.inf)
    for i in range(n):
        at = np.concatenate([np.arange(length), length + np.nonzero(sees[i])[0]])
        if not len(at):
            continue
        for h in range(Hq):
            s = k[at, h // G] @ q[i, h] * scale
            top = s.max()
            p = np.exp(s - top)
            lse[i, h] = top + np.log(p.sum())
            out[i, h] = p @ v[at, h // G] / p.sum()
    return out, lse


def verify(logits, tokens, parents, draft, temperature: float, u, noise):
    """One request: (path, next token). draft [n, V] or None."""
    n = len(tokens)
    if n == 0:
        return [], -1
    V = logits.shape[1]
    node, path = 0, []
    while True:
        path.append(node)
        z = np.asarray(logits[node], np.float64)
        if np.isnan(z).any() or (z == np.inf).any() or not np.isfinite(z).any():
            return path, -1
        kids = [c for c in range(node + 1, n) if parents[c] == node]
        if temperature == 0:
            best = int(z.argmax())
            taken = next((c for c in kids if tokens[c] == best), None)
            if taken is None:
                return path, best
            node = taken
            continue
        r = np.exp((z - z.max()) / temperature)
        r /= r.sum()
        q = np.asarray(draft[node], np.float64).copy() if draft is not None else None
        taken = None
        for c in kids:
            x = int(tokens[c])
            if not 0 <= x < V:
                continue
            qx = q[x] if q is not None else 1.0
            if r[x] > 0 and u[c] * qx <= r[x]:
                taken = c
                break
            less = np.maximum(r - q, 0) if q is not None else np.where(np.arange(V) == x, 0.0, r)
            if less.sum() > 0:
                r = less / less.sum()
            if q is not None:
                q[x] = 0.0
                q = q / (1 - qx) if 1 - qx > 0 else np.zeros(V)
        if taken is None:
            with np.errstate(divide="ignore", invalid="ignore"):
                return path, int(np.where(r > 0, r / noise, -1.0).argmax())
        node = taken
