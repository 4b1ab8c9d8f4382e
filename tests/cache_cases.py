"""Inputs and comparisons that the tests of the compact cache share (no test of its own)."""
import numpy as np
import torch

import paper_2607_05061_amd as kv
from oracle import compact_cache as cc

DTYPE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def bf16(x):
    """x rounded to bf16, on the GPU, and its exact values."""
    t = torch.as_tensor(np.asarray(x), dtype=torch.float64).to(torch.bfloat16)
    return t.cuda(), t.double().numpy()


def i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda().contiguous()


class HostCache:
    """A pool with random codes in every byte, lists of `per` pages each in a shuffled order, and
    a copy on the GPU."""

    def __init__(self, rng, B, H, per, P, D, fmt, spare=2, exps=(-6, 3)):
        n = B * H * per + spare
        self.fmt, self.P, self.D = fmt, P, D
        self.side = {}
        for s in "kv":
            codes = rng.integers(0, 256, (n, P, D)).astype(np.uint8)
            if fmt == "int8":
                codes[codes == 128] = 0
            else:
                codes[(codes & 127) == 127] = 0
            self.side[s] = [codes, rng.integers(exps[0], exps[1] + 1, n).astype(np.int8)]
        self.table = rng.permutation(n)[:B * H * per].reshape(B, H, per).astype(np.int32)

    def gpu(self):
        k, ke = self.side["k"]
        v, ve = self.side["v"]
        up = lambda x: torch.from_numpy(x.copy()).cuda()  # noqa: E731
        return kv.KvpopCache(up(k.view(np.int8)).view(DTYPE[self.fmt]), up(v.view(np.int8)).view(DTYPE[self.fmt]),
                             up(ke), up(ve), up(self.table))

    def append(self, side, x, held, start, b, h):
        codes, exps = self.side[side]
        cc.append(codes, exps, self.table[b, h].tolist(), self.fmt, x, int(held), int(start))

    def check(self, cache):
        """The GPU's pool is this one, byte for byte."""
        for s, pages, exps in (("k", cache.k_pages, cache.k_exp), ("v", cache.v_pages, cache.v_exp)):
            np.testing.assert_array_equal(exps.cpu().numpy(), self.side[s][1], err_msg=s)
            np.testing.assert_array_equal(pages.view(torch.uint8).cpu().numpy(), self.side[s][0], err_msg=s)


def attention_check(q64, host, held, scale, o, lse, q_lens=None, where=None):
    """o and lse of kvpop_cache_attn against the oracle.

    Tolerance, from the arithmetic. A logit's D products are exact in fp32 up to its sums, each
    off by at most 2^-24 of what is summed: dl = (D + 8) 2^-24 scale sum_d |q_d k_d|. The
    exponent's argument, of size up to X = |l| + |lse| + 32 (a value's exponent is added) in units of
    log2, is rounded three times, and 2^x is good to 2 ulp: dx = 2^-22 (1.45 X + 2). So a probability is off
    by eps = 1.01 (dl + 2^-22 (1.45 X + 2) + n 2^-24) of itself, the last for the sum of n. Before
    the product with v it is rounded to 11 bits, 2^-11 of itself, or 2^-25 below 2^-14 of the
    largest numerator, which is at most 2^-25 sum_j |code_j| 2^ve of the largest's key; o is rounded to
    bf16, 2^-8 of itself. A query's elements below 2^-28 of its largest may vanish: below dl."""
    o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    B, Hq, N, D = q64.shape
    H = host.table.shape[1]
    G = Hq // H
    for b in range(B):
        n = N if q_lens is None else min(max(int(q_lens[b]), 0), N)
        for h in range(H):
            k, _, _, ok = cc.list_values(*host.side["k"], host.table[b, h], host.fmt, int(held[b][h]))
            v, code, ve, _ = cc.list_values(*host.side["v"], host.table[b, h], host.fmt, int(held[b][h]))
            L = len(k)
            live = np.ones(L, bool) if where is None else where(b, h, L)
            seen = (np.arange(L)[None] <= L - n + np.arange(n)[:, None]) & (ok & live)[None]
            for g in range(h * G, h * G + G):
                assert (o[b, g, n:] == 0).all() and np.isneginf(lse[b, g, n:]).all(), (b, g)
                if not n:
                    continue
                ro, rl, p = cc.attend(q64[b, g, :n], k, v, seen, scale)
                some = seen.any(1)
                assert (o[b, g, :n][~some] == 0).all() and np.isneginf(lse[b, g, :n][~some]).all(), (b, g)
                if not some.any():
                    continue
                dl = np.where(seen, (D + 8) * 2.0 ** -24 * scale * (np.abs(q64[b, g, :n]) @ np.abs(k).T), 0).max(1)
                X = np.where(seen, np.abs(scale * (q64[b, g, :n] @ k.T)), 0).max(1) + np.abs(np.where(some, rl, 0)) + 32
                eps = 1.01 * (dl + 2.0 ** -22 * (1.45 * X + 2) + L * 2.0 ** -24)
                top = np.where(p > 0, np.log2(np.maximum(p, 1e-300)) + ve, -np.inf).argmax(1)
                tiny = 2.0 ** -25 * (seen[:, :, None] * np.abs(code)[None]).sum(1) * 2.0 ** ve[top][:, None] * \
                    p[np.arange(n), top][:, None]
                bound = (2.0 ** -8 * np.abs(ro) + (2.0 ** -11 + 2 * eps)[:, None] * (p @ np.abs(v)) + tiny) * 1.01 + 1e-30
                err = np.abs(o[b, g, :n] - ro)
                bad = ~(err <= bound)[some]
                assert not bad.any(), "b%d qh%d: %d of %d out of bound, worst ratio %.3g, (query, dim) %s: %s for %s" % (
                    b, g, bad.sum(), bad.size, np.nanmax((err / bound)[some]), np.argwhere(bad)[:4].tolist(),
                    o[b, g, :n][some][bad][:4], ro[some][bad][:4])
                lerr = np.abs(lse[b, g, :n][some] - rl[some])
                lb = (eps + 2.0 ** -22 * (np.abs(rl) + 1))[some]
                assert (lerr <= lb).all(), "b%d qh%d lse: %.3g of bound" % (b, g, np.max(lerr / lb))
