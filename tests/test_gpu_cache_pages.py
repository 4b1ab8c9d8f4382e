"""kvpop_cache_attn over lists of many pages: a wave's share of a list, and a part of it for chunks of queries,
take page numbers 64 at a time. Lists here cross that several times, end at it, begin their shares
inside pages, and have entries without a page beside it. Lists share pages, so that the pool stays small."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2607_05061_amd as kv  # noqa: E402
from cache_cases import HostCache, attention_check, bf16, i32  # noqa: E402

pytestmark = pytest.mark.gpu


def _run(rng, fmt, D, P, B, H, G, N, held, holes=()):
    """holes: (list, entry) pairs without a page."""
    held = np.asarray(held).reshape(B, H)
    host = HostCache(rng, 1, 1, 150, P, D, fmt)
    n = len(host.side["k"][0])
    host.table = rng.integers(0, n, (B, H, -(-int(held.max()) // P))).astype(np.int32)
    for i, (lst, entry) in enumerate(holes):
        host.table.reshape(B * H, -1)[lst, entry] = (-1, n, -2 ** 31, 2 ** 31 - 1)[i % 4]
    scale = 1.0 / (D ** 0.5 * (64 if fmt == "int8" else 100))
    q, q64 = bf16(rng.standard_normal((B, H * G, N, D)))
    o, lse = kv.kvpop_cache_attn(q, host.gpu(), i32(held), scale)
    attention_check(q64, host, held, float(np.float32(scale)), o, lse)


# More than 256 lists (512 for D = 64) are not split: 4 waves share a list in runs of ceil(tiles / 4) tiles
# of 32 keys, so a wave crosses 64 pages of P tokens in lists of more than 4 * 64 P.
@pytest.mark.parametrize("fmt,D", [("int8", 128), ("e4m3", 64)])
@pytest.mark.parametrize("P,longest", [(16, 9100), (32, 17001), (64, 33333), (128, 66000)])
def test_single_tokens_over_long_lists_that_are_not_split(fmt, D, P, longest):
    rng = np.random.default_rng(P + D)
    B, H = (65, 4) if D == 128 else (129, 4)
    held = rng.integers(0, 3 * P, (B, H))
    held[3, 1], held[B - 1, 3] = longest, longest - 4 * 31
    _run(rng, fmt, D, P, B, H, 1, 1, held, holes=[(13, e) for e in (0, 62, 63, 64, 65, 127, 128, 129)])


@pytest.mark.parametrize("fmt,D", [("int8", 128), ("e4m3", 128)])
def test_lists_that_end_where_page_numbers_do(fmt, D):
    """Shares of 31 to 34 tiles of 32 keys, 64 pages of 16 tokens being 32 tiles."""
    rng = np.random.default_rng(1)
    held = rng.integers(0, 40, (66, 4))
    held[0] = [4 * 1024 - 32, 4 * 1024 - 1, 4 * 1024, 4 * 1024 + 1]
    held[1] = [4 * 1024 + 31, 4 * 1024 + 33, 4 * 1024 + 128, 4 * 1024 + 129]
    held[2] = [1023, 1024, 1025, 2 * 4 * 1024 + 1]
    _run(rng, fmt, D, 16, 66, 4, 1, 1, held, holes=[(2, 63), (3, 64), (5, 64), (5, 65), (7, 66)])


@pytest.mark.parametrize("N,G", [(1, 3), (3, 2)])
def test_several_rows_over_a_long_list(N, G):
    rng = np.random.default_rng(N)
    held = rng.integers(0, 100, (65, 4))
    held[7, 2] = 13000
    _run(rng, "int8", 128, 16, 65, 4, G, N, held)


# 130 lists and more are not split for chunks either; a tile is 64 keys (128 for D = 64).
@pytest.mark.parametrize("fmt,D", [("int8", 128), ("e4m3", 128), ("e4m3", 64), ("int8", 64)])
@pytest.mark.parametrize("P,longest", [(16, 5003), (32, 6500), (64, 9100), (128, 25001)])
def test_chunks_over_long_lists_that_are_not_split(fmt, D, P, longest):
    rng = np.random.default_rng(P + D)
    held = rng.integers(0, 3 * P, (66, 2))
    held[0, 1], held[40, 0] = longest, longest // 2 + 1
    held[50] = [64 * P, 64 * P + 1]
    _run(rng, fmt, D, P, 66, 2, 2, 20, held, holes=[(1, e) for e in (0, 63, 64, 67, 128)] + [(101, 64)])


def test_a_chunk_of_many_rows_in_few_parts():
    rng = np.random.default_rng(5)
    _run(rng, "int8", 64, 16, 1, 1, 2, 300, [[20000]], holes=[(0, 63), (0, 64), (0, 700)])
