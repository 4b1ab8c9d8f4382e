"""fp64 oracle of the compact cache (test infrastructure): 8-bit pages with powers of
two as scales, the append of rotated keys and values, the attention over page lists,
and the retention of tokens one at a time.

Codes are bit patterns (uint8). A page's values are code * 2^e. For a magnitude a, e(a) is
the least whole number in [-32, 32] with a <= qmax 2^e (qmax 127 for "int8", 448 for
"e4m3"). Everything is evaluated list by list and page by page from these definitions.

The budget s + w + k per KV head is the paper's (Sec. 3 eq. kv_budget); which tokens a
list holds is the running top-k mask (App. C.1 eq. running_topk_mask_app), brought
forward one query at a time.
"""
from __future__ import annotations

import math

import numpy as np

__all__ = ["E_MIN", "E_MAX", "QMAX", "code_values", "code_of", "needed_exponent", "rotate", "append", "list_values",
           "attend", "retain_step"]

E_MIN, E_MAX = -32, 32
QMAX = {"int8": 127.0, "e4m3": 448.0}


def code_values(fmt: str) -> np.ndarray:
    """The value of each of the 256 bit patterns."""
    bits = np.arange(256)
    if fmt == "int8":
        return np.where(bits < 128, bits, bits - 256).astype(np.float64)
    e, m = (bits >> 3) & 15, bits & 7
    v = np.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * 2.0 ** (e - 7.0))
    v = np.where((bits & 127) == 127, np.nan, v)
    return np.where(bits >= 128, -v, v)


_VALUES = {f: code_values(f) for f in QMAX}


def code_of(y, fmt: str) -> np.ndarray:
    """Bit patterns of the nearest codes of y, ties to even, saturated; NaN gives 0."""
    y = np.asarray(y, dtype=np.float64)
    y = np.where(np.isnan(y), 0.0, y)
    if fmt == "int8":
        return np.clip(np.rint(np.clip(y, -127, 127)), -127, 127).astype(np.int64).astype(np.uint8)
    v = _VALUES["e4m3"][:127]  # ascending; the low bit of the pattern is that of the mantissa
    a = np.minimum(np.abs(y), 448.0)
    hi = np.minimum(np.searchsorted(v, a), 126)
    lo = np.maximum(hi - 1, 0)
    below, above = a - v[lo], v[hi] - a
    up = (above < below) | ((above == below) & (hi % 2 == 0)) | (v[hi] == a)
    return (np.where(up, hi, lo) + np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def needed_exponent(x, fmt: str) -> int:
    """The least e in [E_MIN, E_MAX] with |x| <= qmax 2^e for every finite x."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(x[np.isfinite(x)]).max(initial=0.0)
    e = E_MIN
    while e < E_MAX and a > QMAX[fmt] * 2.0 ** e:
        e += 1
    return e


def rotate(x, cos, sin, adjacent: bool) -> np.ndarray:
    """R(p) x for rows x [..., D] and their table rows cos, sin [..., R / 2]."""
    y = np.array(x, dtype=np.float64)
    R = 2 * cos.shape[-1]
    a, b = (y[..., 0:R:2], y[..., 1:R:2]) if adjacent else (y[..., :R // 2], y[..., R // 2:R])
    with np.errstate(invalid="ignore", over="ignore"):
        a2, b2 = a * cos - b * sin, b * cos + a * sin
    if adjacent:
        y[..., 0:R:2], y[..., 1:R:2] = a2, b2
    else:
        y[..., :R // 2], y[..., R // 2:R] = a2, b2
    return y


def append(pages, exps, table, fmt, rows, held: int, start: int):
    """Writes rows [n, D] (64 bits) to the slots start .. start + n - 1 of one list, in
    place. pages: uint8 [n_pages, P, D]; exps: int8 [n_pages]; table: the list's pages."""
    P = pages.shape[1]
    n = len(rows)
    if start < 0:
        return
    for p in range(start // P, min(len(table), -(-(start + n) // P))):
        lo, hi = max(start, p * P), min(start + n, (p + 1) * P)
        if lo >= hi or not 0 <= table[p] < len(pages):
            continue
        page = table[p]
        new = rows[lo - start:hi - start]
        old = [j - p * P for j in range(p * P, min(held, (p + 1) * P)) if not lo <= j < hi]
        e = needed_exponent(new, fmt)
        if old:
            was = int(exps[page])
            e = max(e, was)
            if e > was:
                pages[page, old] = code_of(_VALUES[fmt][pages[page, old]] * 2.0 ** (was - e), fmt)
        exps[page] = e
        pages[page, lo - p * P:hi - p * P] = code_of(new * 2.0 ** -e, fmt)


def list_values(pages, exps, table, fmt, held: int):
    """(values [n, D], codes' values [n, D], exponents [n]) of one list's slots, n = held
    taken into the list's room, and which of them have a page [n]."""
    P, D = pages.shape[1:]
    n = min(max(held, 0), len(table) * P)
    codes, e, ok = np.zeros((n, D)), np.zeros(n), np.zeros(n, dtype=bool)
    for p in range(-(-n // P)):
        m = min(P, n - p * P)
        if 0 <= table[p] < len(pages):
            codes[p * P:p * P + m] = _VALUES[fmt][pages[table[p], :m]]
            e[p * P:p * P + m] = float(exps[table[p]])
            ok[p * P:p * P + m] = True
    return codes * 2.0 ** e[:, None], codes, e, ok


def attend(q, k, v, seen, scale: float):
    """Softmax attention of rows q [n, D] over keys k [L, D] of which row i sees seen[i]
    (bool [n, L]): (o [n, D], lse [n], p [n, L]); rows that see nothing get 0 and -inf."""
    l = scale * (np.asarray(q, dtype=np.float64) @ k.T)
    l = np.where(seen, l, -np.inf)
    m = np.where(seen.any(1), l.max(1, initial=-np.inf), 0.0)
    p = np.exp(l - m[:, None])
    z = p.sum(1)
    with np.errstate(divide="ignore"):
        lse = m + np.log(z)
    p = p / np.where(z > 0, z, 1.0)[:, None]
    return p @ v, lse, p


def _order(prio: float):
    """A number that orders priorities as kvpop_running_topk does (-0 = +0, NaN by its bits)."""
    u = int(np.float32(prio).view(np.uint32))
    u = 0 if u == 0x80000000 else u
    return -(u & 0x7FFFFFFF) - 1 if u & 0x80000000 else u


def retain_step(state: dict, q: int, score: float, log_gamma: float, s: int, w: int, k: int) -> int:
    """The token at position q arrives at one list. state: {slot: [position, priority]}.
    Returns its slot, or -1."""
    if q < 0:
        return -1
    t = q - w
    mine = np.float32(np.float32(score) - np.float32(np.float32(t) * np.float32(log_gamma)))
    for x in state.values():
        if x[0] == t:
            x[1] = mine
    if len(state) < s + w + k:
        slot = len(state)
    else:
        can = [(_order(x[1]), -x[0], i) for i, x in state.items() if s <= x[0] <= t]
        if w == 0 and t >= s:
            can.append((_order(mine), -t, -1))
        slot = min(can)[2] if can else -1
    if slot >= 0:
        state[slot] = [q, mine if w == 0 else np.float32(0.0)]
    return slot
