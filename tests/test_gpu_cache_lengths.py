"""kvpop_cache_append with lengths (held) of any value beside a first slot of its own: only the
slots that they make others' tokens of are moved, and nothing outside the page."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2607_05061_amd as kv  # noqa: E402
from cache_cases import HostCache, bf16, i32  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("start", [0, 20, 45])
def test_lengths_of_any_value(fmt, start):
    rng = np.random.default_rng(start)
    lengths = np.array([[-2 ** 31, -2 ** 31 + 15, -2 ** 31 + 50, -2 ** 31 + 2 ** 24],
                        [-1, 0, 2 ** 31 - 1, 2 ** 31 - 50]])
    B, H, N, P, D = 2, 4, 6, 16, 64
    k, k64 = bf16(rng.standard_normal((B, H, N, D)) * 4096)  # every page's exponent grows
    host = HostCache(rng, B, H, 4, P, D, fmt)
    cache = host.gpu()
    kv.kvpop_cache_append(cache, k, k, i32(lengths), start=i32(np.full((B, H), start)))
    for b in range(B):
        for h in range(H):
            for s in "kv":
                host.append(s, k64[b, h], lengths[b, h], start, b, h)
    host.check(cache)
