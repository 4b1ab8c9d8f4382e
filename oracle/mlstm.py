"""The mLSTM scorer's recurrence from its definition in 64 bits (plain NumPy), head by head.

``log_weights`` are the logarithms of the weight that token t has in what is held at time u,
ig_t + sum_{t < s <= u} log sigmoid(fg_s), built row after row, so that no infinities are
subtracted. ``read`` is the read-out, ``grads`` the gradients for a given o and lse by their
formulas, ``recur`` the recurrence itself, token by token.
"""
import numpy as np


def log_sigmoid(x):
    x = np.asarray(x, np.float64)
    with np.errstate(over="ignore"):
        return -(np.maximum(-x, 0) + np.log1p(np.exp(-np.abs(x))))


def log_weights(ig, fg):
    """[T, T], -inf above the diagonal."""
    T = len(ig)
    lf = log_sigmoid(fg)
    L = np.full((T, T), -np.inf)
    for u in range(T):
        if u:
            L[u, :u] = L[u - 1, :u] + lf[u]
        L[u, u] = ig[u]
    return L


def clean(x, off):
    """Rows that have no weight, as zeros."""
    return np.where(off[:, None], 0.0, x)


def read(q, k, v, ig, fg, scale, delay, normalize, state=None):
    """(o [T, D], lse [T], weights [T, T] of the tokens in each row's read-out, absolute sums of the
    terms of o and of the normaliser, divided as o is). state: (C, z, m) held before. Rows that are
    not read: 0 and -inf."""
    T, D = q.shape
    k, v = clean(k, np.isneginf(ig)), clean(v, np.isneginf(ig))
    L = log_weights(ig, fg)
    old = np.full(T, -np.inf)
    if state is not None:
        old = state[2] + np.cumsum(log_sigmoid(fg))
    o, lse, W = np.zeros((T, D)), np.full(T, -np.inf), np.zeros((T, T))
    terms, den_terms = np.zeros((T, D)), np.zeros(T)
    for t in range(T - delay):
        u = t + delay
        top = max(L[u].max(), old[u])
        if top == -np.inf:
            lse[t] = -np.inf if normalize else 0.0
            continue
        w, f = np.exp(L[u] - top), np.exp(old[u] - top)
        x = scale * q[t]
        s, sa = k @ x, np.abs(k) @ np.abs(x)
        num, den, a, b = (w * s) @ v, (w * s).sum(), (w * sa) @ np.abs(v), (w * sa).sum()
        if state is not None and f > 0:
            num, den = num + f * (x @ state[0]), den + f * (x @ state[1])
            a, b = a + f * (np.abs(x) @ np.abs(state[0])), b + f * (np.abs(x) @ np.abs(state[1]))
        if normalize and not den > 0:
            continue
        lse[t] = top + np.log(den) if normalize else 0.0
        c = 1 / den if normalize else np.exp(top)
        o[t], W[t], terms[t], den_terms[t] = num * c, w * c, a * c, b * c
    return o, lse, W, terms, den_terms


def held(k, v, ig, fg, state=None):
    """(C, z, m) after the last token."""
    T, D = k.shape
    k, v = clean(k, np.isneginf(ig)), clean(v, np.isneginf(ig))
    w = np.full(T, -np.inf)
    C0, z0, m0 = state if state is not None else (np.zeros((D, D)), np.zeros(D), -np.inf)
    m = old = m0
    lf = log_sigmoid(fg)
    for t in range(T):
        w[:t] += lf[t]
        w[t] = ig[t]
        old += lf[t]
        m = max(m + lf[t], ig[t])
    if m == -np.inf:
        return np.zeros((D, D)), np.zeros(D), m
    e, f = np.exp(w - m), np.exp(old - m)
    C, z = (k * e[:, None]).T @ v, e @ k
    return (C + f * C0, z + f * z0, m) if f > 0 else (C, z, m)


def recur(q, k, v, ig, fg, scale, normalize):
    """o and the last (C, z), token by token without a common factor (small gates only)."""
    T, D = q.shape
    C, z, o = np.zeros((D, D)), np.zeros(D), np.zeros((T, D))
    for t in range(T):
        f, i = np.exp(log_sigmoid(fg[t])), np.exp(ig[t])
        C, z = f * C + i * np.outer(k[t], v[t]), f * z + i * k[t]
        x = scale * q[t]
        o[t] = x @ C / (x @ z if normalize else 1.0)
    return o, C, z


def grads(do, q, k, v, ig, fg, o, lse, scale, delay, normalize):
    """(dq, dk, dv, dig, dfg) for this o and lse, and of each the absolute sums of its terms: what
    a rounding of each term by a share of itself can change at most by that share."""
    T, D = q.shape
    off = np.isneginf(ig)
    k, v = clean(k, off), clean(v, off)
    n = max(0, T - delay)
    got = np.zeros(T, bool)
    got[:n] = ~np.isneginf(lse[:n])
    q, do, o = (clean(x, ~got) for x in (q, do, o))
    L = log_weights(ig, fg)
    W = np.zeros((T, T))  # by time
    X, G, d = np.zeros((T, D)), np.zeros((T, D)), np.zeros(T)
    for t in np.flatnonzero(got):
        W[t + delay] = np.exp(L[t + delay] - lse[t])
        X[t + delay], G[t + delay] = scale * q[t], do[t]
        d[t + delay] = -(do[t] @ o[t]) if normalize else 0.0
    A = np.abs
    S, Sa = X @ k.T, A(X) @ A(k).T
    dS, dSa = W * (G @ v.T + d[:, None]), W * (A(G) @ A(v).T + A(d)[:, None])
    dx, dxa = dS @ k, dSa @ A(k)
    dk, dka = dS.T @ X, dSa.T @ A(X)
    dv, dva = (W * S).T @ G, (W * Sa).T @ A(G)
    dq, dqa = np.zeros((T, D)), np.zeros((T, D))
    dq[:n], dqa[:n] = scale * dx[delay:], scale * dxa[delay:]
    dig, diga = (k * dk).sum(1), (A(k) * dka).sum(1)
    dfg, dfga = np.zeros(T), np.zeros(T)
    P = dS * S
    sig = np.exp(log_sigmoid(-np.asarray(fg, np.float64)))
    for t in range(T):  # pairs that t lies between
        dfg[t] = sig[t] * P[t:, :t].sum()
        dfga[t] = sig[t] * diga.sum()
    return (dq, dk, dv, dig, dfg), (dqa, dka, dva, diga, dfga)
