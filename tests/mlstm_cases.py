"""Inputs and comparisons that the tests of the mLSTM recurrence share (no test of its own)."""
import numpy as np
import torch

from oracle import mlstm as om

U = 2.0 ** -8  # half a step of bf16, relative
NAMES = ("dq", "dk", "dv", "dig", "dfg")


def features(rng, shape, signed=False):
    x = rng.standard_normal(shape) * 1.5
    if signed:
        return x * 0.3
    x = np.exp(x - x.max(-1, keepdims=True))
    return x / x.sum(-1, keepdims=True)


def b16(x):
    """x rounded to bf16 on the GPU, and its exact values."""
    t = torch.as_tensor(np.asarray(x), dtype=torch.float64).to(torch.bfloat16)
    return t.cuda(), t.double().numpy()


def inputs(rng, B, H, T, D, signed=False, ig=(0.0, 1.0), fg=(4.0, 1.5)):
    return dict(q=features(rng, (B, H, T, D), signed), k=features(rng, (B, H, T, D), signed),
                v=rng.standard_normal((B, H, T, D)) + 0.3, ig=ig[0] + ig[1] * rng.standard_normal((B, H, T)),
                fg=fg[0] + fg[1] * rng.standard_normal((B, H, T)), do=rng.standard_normal((B, H, T, D)))


def on_gpu(x, tokens=False):
    """The arrays on the GPU (as views of [B, T, H, ...] with `tokens`) and their exact values."""
    gpu, ref = {}, {}
    for n, y in x.items():
        t, ref[n] = b16(y)
        gpu[n] = t.transpose(1, 2).contiguous().transpose(1, 2) if tokens else t
    return gpu, ref


def check(name, got, want, bound):
    got = got.double().cpu().numpy() if isinstance(got, torch.Tensor) else got
    err = np.abs(got - want)
    bad = ~(err <= bound)
    assert not bad.any(), "%s: %d of %d out of bound, worst ratio %.3g at %s: %s for %s" % (
        name, bad.sum(), bad.size, np.nanmax(np.where(bad, err / np.maximum(bound, 1e-300), 0)), np.argwhere(bad)[:3].tolist(),
        got[bad][:4], want[bad][:4])


def check_read(ref, lens, scale, delay, normalize, o, lse, state=None, after=None):
    """Tolerance, from the arithmetic (u = 2^-8): a weight times <x, k> is rounded to bf16 before it meets v, or an
    element of what is held before it meets x: u of each term; o is rounded: u of itself. What is held carries
    16 bits of each token's weighted value (two bf16 parts) and fp32 sums, exponents 2^-17 at most
    (150 log2 units in fp32), products fp32 sums over D and 64 terms: together below 2^-14 of each term, also
    of the normaliser's."""
    o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    B, H, T, D = ref["q"].shape
    for b in range(B):
        n = T if lens is None else min(max(int(lens[b]), 0), T)
        for h in range(H):
            x = {y: ref[y][b, h, :n] for y in ("q", "k", "v", "ig", "fg")}
            s = None if state is None else [y[b, h] for y in state]
            with np.errstate(invalid="ignore"):
                ro, rl, _, terms, dens = om.read(x["q"], x["k"], x["v"], x["ig"], x["fg"], scale, delay, normalize, s)
            assert (o[b, h, n:] == 0).all() and np.isneginf(lse[b, h, n:]).all()
            off = np.isneginf(rl)
            assert np.array_equal(np.isneginf(lse[b, h, :n]), off), (b, h)
            assert (o[b, h, :n][off] == 0).all()
            tiny = 2.0 ** -14
            rel = dens[:, None] * tiny if normalize else 0.0
            check("o b%d h%d" % (b, h), o[b, h, :n], ro, 1.01 * (U * np.abs(ro) + (U + tiny) * terms + rel * np.abs(ro)) + 1e-30)
            if normalize and n:
                check("lse b%d h%d" % (b, h), lse[b, h, :n][~off], rl[~off], (dens * tiny + 2.0 ** -21 * (np.abs(np.where(off, 0, rl)) + 1))[~off])
            if after is not None:
                rs = om.held(x["k"], x["v"], x["ig"], x["fg"], s) if n else s
                ra = om.held(np.abs(x["k"]), np.abs(x["v"]), x["ig"], x["fg"], None if s is None else [np.abs(s[0]), np.abs(s[1]), s[2]]) if n else s
                for y, got, want, most in zip("Cz", after, rs, ra):
                    check("%s b%d h%d" % (y, b, h), got[b, h].double().cpu().numpy(), want, tiny * np.abs(most) + 1e-37)
                m = float(after[2][b, h])
                assert m == rs[2] or abs(m - rs[2]) <= 2.0 ** -20 * (abs(rs[2]) + 1), (m, rs[2])


def check_grads(ref, lens, scale, delay, normalize, o, lse, grads):
    """Tolerance, from the arithmetic (u = 2^-8): a gradient's terms are rounded once each before their product (the
    weighted product of the chunk, or the element of what is held), and the gradient itself: u of the terms' absolute
    sum and of itself; 2^-14 for the rest as in check_read. dig sums k times dk unrounded; dfg is a running sum of
    dig and of do . o from an exact edge, which may be off by what all the terms may, twice (its start's and its end's)."""
    o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    grads = [x.double().cpu().numpy() for x in grads]
    B, H, T, D = ref["q"].shape
    for b in range(B):
        n = T if lens is None else min(max(int(lens[b]), 0), T)
        for h in range(H):
            x = {y: ref[y][b, h, :n] for y in ("q", "k", "v", "ig", "fg", "do")}
            with np.errstate(invalid="ignore"):
                want, terms = om.grads(x["do"], x["q"], x["k"], x["v"], x["ig"], x["fg"], o[b, h, :n], lse[b, h, :n], scale, delay, normalize)
            for name, g, w, t in zip(NAMES, grads, want, terms):
                assert (g[b, h, n:] == 0).all(), name
                loose = 2.0 if name == "dfg" else 1.0
                check("%s b%d h%d" % (name, b, h), g[b, h, :n], w, 1.01 * (U * np.abs(w) + loose * (U + 2.0 ** -13) * t) + 1e-30)


def norm_error(got, want):
    got = got.double().cpu().numpy() if isinstance(got, torch.Tensor) else got
    return float(np.linalg.norm(got - want) / max(np.linalg.norm(want), 1e-300))


def partial_sums(x, o, lse, scale, delay, normalize):
    """Of one head, by token t: G, the sum over the pairs of a token s < t and a read-out at u >= t of
    W(u, s) (x_u . k_s) (do_u . v_s + d_u), which sigmoid(-fg_t) makes dfg_t; and R, the root of the sum of the squares of
    W |x . k| times the root of the sum of the squares of what do . v + d adds up. own: that of a token's pair with itself, which
    is in neither but in both of the terms that a running sum subtracts."""
    q, k, v, ig, fg, do = (x[n] for n in ("q", "k", "v", "ig", "fg", "do"))
    T, D = q.shape
    off = np.isneginf(ig)
    k, v = om.clean(k, off), om.clean(v, off)
    n = max(0, T - delay)
    got = np.zeros(T, bool)
    got[:n] = ~np.isneginf(lse[:n])
    L = om.log_weights(ig, fg)
    P, Q = np.zeros((T, T)), np.zeros((T, T))
    u = np.flatnonzero(got)
    if len(u):
        W = np.exp(L[u + delay] - lse[u][:, None])
        s = scale * q[u] @ k.T
        d = -(do[u] * o[u]).sum(1) if normalize else np.zeros(len(u))
        P[u + delay] = W * s * (do[u] @ v.T + d[:, None])
        squares = (do[u] ** 2) @ (v.T ** 2) + (((do[u] * o[u]) ** 2).sum(1) if normalize else np.zeros(len(u)))[:, None]
        Q[u + delay] = (W * s) ** 2 * squares
    G, R = np.zeros(T), np.zeros(T)
    forgets = np.asarray(fg) < -2.0 ** 24
    for y, sums in ((P, G), (Q, R)):  # a token's pairs as a key begin behind it, those as a query end there
        step = y.sum(0) - y.sum(1)
        for t in range(1, T):
            sums[t] = 0.0 if forgets[t] else sums[t - 1] + step[t - 1]
    return G, np.sqrt(np.maximum(R, 0)), np.sqrt(np.diag(Q))


def check_forget(name, got, fg, G, R, own, D):
    """The forget gates' gradients of one head. Their error is that of sums, relative to the largest of the partial sums since
    the last gate that forgets everything (or to R where those cancel): in the 2-norm over these tokens, four of at most
    2^-8 / sqrt(3): the pairs' rounded weights, the read state's elements in dk, o in do . o, the result. Beside it what fp32 leaves
    where a token's own pair cancels in x . dx - k . dk, sums of D products that are sums of up to 64 terms: (D + 64) 2^-24 of it
    on each side, independent from token to token. (With f = e^-20 that is more than all other pairs are.)"""
    sig = np.exp(om.log_sigmoid(-np.asarray(fg, np.float64)))
    group = np.cumsum(np.asarray(fg) < -2.0 ** 24)
    for i in range(group[-1] + 1 if len(group) else 0):
        t = np.flatnonzero(group == i)
        if not len(t):
            continue
        most = max(np.abs(G[t]).max(), R[t].max())
        most = 4 * U / 3 ** 0.5 * most + 2 * (D + 64) * 2.0 ** -24 * np.linalg.norm(own[t])
        err, bound = np.linalg.norm(got[t] - sig[t] * G[t]), most * np.linalg.norm(sig[t])
        assert err <= bound + 1e-30, "%s: tokens %d to %d: error %.3g, bound %.3g, size %.3g" % (
            name, t[0], t[-1], err, bound, np.linalg.norm(sig[t] * G[t]))
