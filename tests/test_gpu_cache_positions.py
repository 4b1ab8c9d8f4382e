"""kvpop_cache_append at positions outside the table of angles, and how attention sees such tokens: a key of
zeros, and the value as it is. Queries turn in 32 bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2607_05061_amd as kv  # noqa: E402
from cache_cases import HostCache, attention_check, bf16, i32  # noqa: E402
from oracle import compact_cache as cc  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("pos0", [-3, 6, 2 ** 31 - 4, -2 ** 31])
def test_positions_outside_the_table(fmt, pos0):
    rng = np.random.default_rng(abs(pos0) % 1000)
    B, H, G, N, P, D, n_pos = 1, 2, 2, 8, 16, 64, 10
    k, k64 = bf16(rng.standard_normal((B, H, N, D)))
    v, v64 = bf16(rng.standard_normal((B, H, N, D)))
    q, q64 = bf16(rng.standard_normal((B, H * G, N, D)))
    ang = rng.standard_normal((n_pos, D // 2)) * 3
    c, s = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
    host = HostCache(rng, B, H, 1, P, D, fmt)
    cache = host.gpu()
    held = np.full((B, H), N)
    got = kv.kvpop_cache_append(cache, k, v, i32(held), q=q, rotary=(torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()),
                                pos0=i32([pos0]))
    at = pos0 + np.arange(N, dtype=np.int64)
    ok = (at >= 0) & (at < n_pos)
    cs, sn = (x[np.clip(at, 0, n_pos - 1)].astype(np.float64) for x in (c, s))
    turned = lambda x: np.where(ok[:, None], cc.rotate(x, cs, sn, False), 0.0)  # noqa: E731
    for h in range(H):
        host.append("k", turned(k64[0, h]), N, 0, 0, h)
        host.append("v", v64[0, h], N, 0, 0, h)
    host.check(cache)
    want = turned(q64[0])
    # two products and a sum in 32 bits, each 2^-24 of what it rounds, and bf16's half step
    size = 2 * np.abs(q64[0]).max(-1, keepdims=True)
    assert (np.abs(got[0].double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 3 * 2.0 ** -24 * size).all()
    o, lse = kv.kvpop_cache_attn(got, cache, i32(held), 0.125)
    attention_check(got.double().cpu().numpy(), host, held, 0.125, o, lse)
