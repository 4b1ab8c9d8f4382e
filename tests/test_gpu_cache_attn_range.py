"""kvpop_cache_attn where much of the answer comes from keys whose numerators, probability times their
page's 2^e, are far below the largest one: a sink that takes nearly all the mass and has no value, and a page
with a large scale beside others."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2607_05061_amd as kv  # noqa: E402
from cache_cases import HostCache, bf16, i32  # noqa: E402
from oracle import compact_cache as cc  # noqa: E402

pytestmark = pytest.mark.gpu


def _check(q64, host, L, scale, o, lse):
    """One list, all of whose queries see it whole but for the last ones' own tokens.

    Tolerance, from the arithmetic: eps, dl and X as in cache_cases.attention_check; numerators are rounded to 11
    bits, 2^-11 of themselves, down to 2^-21 of the largest one, and below that to 2^-32 of it; o
    is rounded to bf16, 2^-8 of itself."""
    o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    _, Hq, N, D = q64.shape
    k, _, _, _ = cc.list_values(*host.side["k"], host.table[0, 0], host.fmt, L)
    v, code, ve, _ = cc.list_values(*host.side["v"], host.table[0, 0], host.fmt, L)
    seen = np.arange(L)[None] <= L - N + np.arange(N)[:, None]
    for g in range(Hq):
        ro, rl, p = cc.attend(q64[0, g], k, v, seen, scale)
        dl = (D + 8) * 2.0 ** -24 * scale * (np.abs(q64[0, g]) @ np.abs(k).T).max(1)
        X = np.abs(scale * (q64[0, g] @ k.T)).max(1) + np.abs(rl) + 32
        eps = 1.01 * (dl + 2.0 ** -22 * (1.45 * X + 2) + L * 2.0 ** -24)
        top = (p * 2.0 ** ve).max(1)
        tiny = 2.0 ** -32 * (seen[:, :, None] * np.abs(code)[None]).sum(1) * top[:, None]
        bound = (2.0 ** -8 * np.abs(ro) + (2.0 ** -11 + 2 * eps)[:, None] * (p @ np.abs(v)) + tiny) * 1.01 + 1e-30
        worst = (np.abs(o[0, g] - ro) / bound).max()
        assert worst <= 1, "head %d: error %.3g of its bound" % (g, worst)
        assert (np.abs(lse[0, g] - rl) <= eps + 2.0 ** -22 * (np.abs(rl) + 1)).all()


@pytest.mark.parametrize("fmt,D", [("int8", 64), ("e4m3", 128)])
@pytest.mark.parametrize("N", [1, 40, 100])
@pytest.mark.parametrize("L", [500, 6000])
@pytest.mark.parametrize("at", [0, 250])
def test_a_sink_without_a_value(fmt, D, N, L, at):
    """Key `at` has 2^27 times the probability of each other key, and a value of zeros."""
    P, rng = 32, np.random.default_rng(N + L)
    host = HostCache(rng, 1, 1, -(-L // P), P, D, fmt, exps=(0, 0))
    k, v = host.side["k"][0], host.side["v"][0]
    k[:, :, 0] = 0
    page, row = host.table[0, 0, at // P], at % P
    k[page, row], v[page, row] = 0, 0
    k[page, row, 0] = 64 if fmt == "int8" else 0x68  # 64
    q = np.zeros((1, 2, N, D))
    q[..., 0] = 1.0
    q[..., 1:] = rng.standard_normal((1, 2, N, D - 1)) * 2.0 ** -12
    qg, q64 = bf16(q)
    scale = float(np.float32(27 * math.log(2) / 64))
    o, lse = kv.kvpop_cache_attn(qg, host.gpu(), i32([[L]]), scale)
    _check(q64, host, L, scale, o, lse)


@pytest.mark.parametrize("fmt,D", [("int8", 128), ("e4m3", 64)])
@pytest.mark.parametrize("N", [1, 40, 100])
@pytest.mark.parametrize("above", [14, 20, 24])
def test_a_page_with_a_large_scale(fmt, D, N, above):
    """A page's scale is 2^above times the others', for one element of one of its tokens."""
    P, L, rng = 16, 176, np.random.default_rng(N + above)
    host = HostCache(rng, 1, 1, L // P, P, D, fmt, exps=(-7, -7))
    codes, exps = host.side["v"]
    big = host.table[0, 0, 3]
    codes[big] = 0
    codes[big, 5, 7] = 100 if fmt == "int8" else 0x6C
    exps[big] += above
    q, q64 = bf16(rng.standard_normal((1, 2, N, D)))
    scale = 0.01
    o, lse = kv.kvpop_cache_attn(q, host.gpu(), i32([[L]]), scale)
    _check(q64, host, L, float(np.float32(scale)), o, lse)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N", [1, 40, 100])
@pytest.mark.parametrize("size", [0, 14, 17, 18, 19, 20, 21, 22, 25])
def test_logits_of_any_size(D, N, size):
    """Logits of up to 127 2^size, past what 32 bits tell apart by less than 2^(size - 17): two keys share
    all of the probability, since the others' logits lie 20 2^size below, and nothing becomes NaN or infinite."""
    P, L, rng = 32, 300, np.random.default_rng(D + N + size)
    host = HostCache(rng, 1, 1, -(-L // P), P, D, "int8", exps=(0, 0))
    k, v = host.side["k"][0].view(np.int8), host.side["v"][0].view(np.int8)
    k[:] = 0
    k[:, :, 0] = rng.integers(-127, 107, k.shape[:2])
    at = [(host.table[0, 0, j // P], j % P) for j in (70, 150)]
    for x in at:
        k[x][0] = 127
    q = np.zeros((1, 1, N, D))
    q[..., 0] = 1.0
    o, lse = kv.kvpop_cache_attn(bf16(q)[0], host.gpu(), i32([[L]]), 2.0 ** size)
    va, vb = (v[x].astype(np.float64) for x in at)
    want = (va + vb) / 2
    top = 127 * 2.0 ** size + math.log(2)
    # The two logits are alike, but each numerator's argument is off by up to eps = 2^-22 (1.45 X + 2) (as in
    # cache_cases.attention_check, X = |l| + |lse| + 32), differently where the reference is: their ratio is
    # within e^(2 eps), and a share within tanh(eps) / 2 of a half. The others together are below 300 e^-20
    # of them; a bf16 half step, and a sum's rounding.
    eps = 2.0 ** -22 * (1.45 * (2 * top + 32) + 2)
    bound = math.tanh(eps) / 2 * np.abs(va - vb) + 2.0 ** -8 * (np.abs(want) + np.abs(va - vb) * math.tanh(eps)) + \
        300 * math.exp(-20) * 254 + 2.0 ** -11
    assert (np.abs(o[0, 0].double().cpu().numpy() - want) <= bound).all()
    assert (np.abs(lse[0, 0].double().cpu().numpy() - top) <= 2.0 ** -21 * top + math.tanh(eps)).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N", [1, 40, 100])
@pytest.mark.parametrize("size", [17, 18, 19, 20, 21, 22])
@pytest.mark.parametrize("step", [1, 2, 4])
def test_large_logits_that_grow(D, N, size, step):
    """Logits around 127 2^size that grow along the list by steps of what 32 bits tell apart there, so that
    the reference is behind by each small multiple of that. All values are 100, and so is every answer,
    whatever the weights."""
    P, L = 32, 300
    host = HostCache(np.random.default_rng(D), 1, 1, -(-L // P), P, D, "int8", exps=(0, 0))
    k = host.side["k"][0].view(np.int8)
    host.side["v"][0][:] = 100
    k[:] = 0
    for j in range(L):
        k[host.table[0, 0, j // P], j % P, :2] = 127, -127 + 254 * j // L
    q = np.zeros((1, 1, N, D))
    q[..., 0], q[..., 1] = 1.0, 2.0 ** -21 * step
    o, lse = kv.kvpop_cache_attn(bf16(q)[0], host.gpu(), i32([[L]]), 2.0 ** size)
    # numerators are rounded to 11 bits each, and o to bf16
    assert ((o.double() - 100).abs() <= 100 * (2.0 ** -8 + 2.0 ** -11)).all()
    # the largest logit that a query sees, and the log of at most L like it
    c = -127 + 254 * (L - N + np.arange(N)) // L
    top = torch.as_tensor((127 + c * q[0, 0, 0, 1]) * 2.0 ** size).cuda()
    assert ((lse[0, 0].double() - top).abs() <= 2.0 ** -20 * top + math.log(L)).all()
