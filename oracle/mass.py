"""Eviction by accumulated attention weight, from its definition in 64 bits (plain NumPy and Python).

* a slot's new mass: ``decay * mass`` plus the probabilities that the queries which see it give it;
* what a prompt keeps: sinks, the newest window, and the largest masses of the others;
* the slot for a new token: the least mass that is neither a sink nor new.
"""
import numpy as np


def order_key(x):
    """float32 values as integers that grow as they do, -0 as +0, NaN above +inf."""
    x = np.asarray(x, np.float32)
    u = np.where(x == 0, np.float32(0), x).view(np.uint32).astype(np.int64)
    return np.where(np.isnan(x), 1 << 31, np.where(u >> 31 == 1, -(u & 0x7FFFFFFF) - 1, u))


def add_mass(mass, q, k, seen, lse, scale, decay):
    """mass [L]; q [rows, D], k [L, D], seen [rows, L], lse [rows], all in 64 bits."""
    if not len(q):
        return decay * mass if decay else np.zeros_like(mass)
    with np.errstate(over="ignore", invalid="ignore"):
        x = scale * (q @ k.T) - np.where(np.isneginf(lse), np.inf, lse)[:, None]
        p = np.where(seen, np.exp(x), 0.0)
    return (decay * mass if decay else 0.0) + p.sum(0)


def group_mass(mass):
    """mass [G, T] float32: summed in 64 bits head after head, rounded to 32."""
    s = np.zeros(mass.shape[1])
    for row in mass.astype(np.float64):
        s = s + row
    return s.astype(np.float32)


def prompt_keeps(a, sinks, window, topk):
    """Ascending positions that a prompt with masses a [n] (float32) keeps."""
    n = len(a)
    lo = min(sinks, n)
    hi = max(lo, n - window)
    key = order_key(a)
    middle = sorted(range(lo, hi), key=lambda t: (-key[t], t))[:topk]
    return sorted(list(range(lo)) + middle + list(range(hi, n)))


def step(state, q, sinks, window, topk):
    """state {slot: [position, mass]}, updated; the slot of the token at q, or -1."""
    if q < 0:
        return -1
    slot = len(state)
    if slot >= sinks + window + topk:
        can = [(order_key(m).item(), -p, s) for s, (p, m) in state.items() if sinks <= p <= q - window]
        if not can:
            return -1
        slot = min(can)[2]
    state[slot] = [q, np.float32(0)]
    return slot
