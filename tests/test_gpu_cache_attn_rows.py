"""kvpop_cache_attn, one query beside others: what it gets is its own list's answer, bit for bit,
whatever the other queries of the call are."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2607_05061_amd as kv  # noqa: E402
from cache_cases import HostCache, attention_check, bf16, i32  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,D,P", [("int8", 128, 64), ("e4m3", 128, 16), ("int8", 64, 32), ("e4m3", 64, 128)])
@pytest.mark.parametrize("N", [1, 7, 40, 150])
def test_a_query_does_not_depend_on_the_others(fmt, D, P, N):
    """Flat logits over a list of many tiles, and the same with queries among them that are not finite, that are
    sharp, or that see their largest logits last."""
    rng = np.random.default_rng(D + P + N)
    H, G, L = 2, 2, 2500
    host = HostCache(rng, 1, H, -(-L // P), P, D, fmt, exps=(-2, -1))
    held = np.array([[L, L - 700]])
    cache = host.gpu()
    q, q64 = bf16(rng.standard_normal((1, H * G, N, D)))
    scale = 1.0 / (D ** 0.5 * (32 if fmt == "int8" else 50))
    o, lse = kv.kvpop_cache_attn(q, cache, i32(held), scale)
    attention_check(q64, host, held, float(np.float32(scale)), o, lse)
    for gain in (float("nan"), float("inf"), 30.0, 1000.0, 0.0):
        other = torch.zeros(H * G, N, dtype=torch.bool)
        other[rng.integers(0, H * G), N // 2] = True
        other[1, ::5] = True
        other[2, N - 1] = True
        q2 = q.clone()
        q2[0, other.cuda()] *= gain
        o2, lse2 = kv.kvpop_cache_attn(q2, cache, i32(held), scale)
        mine = ~other
        assert torch.equal(o2[0].cpu()[mine], o[0].cpu()[mine]), gain
        assert torch.equal(lse2[0].cpu()[mine], lse[0].cpu()[mine]), gain
