"""kvpop_cache_append against the fp64 oracle. Codes and exponents have to be equal bit for
bit: a code is the one rounding of a value that the kernel has in 64 bits, where a
rotation's products of bf16 and fp32 numbers are exact and its sums rounded to 2^-53, so that
only a sum within 2^-53 of the border between two codes could differ. Bytes that no token of the
call uses have to stay."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2607_05061_amd as kv  # noqa: E402
from cache_cases import HostCache, bf16, i32  # noqa: E402
from oracle import compact_cache as cc  # noqa: E402

pytestmark = pytest.mark.gpu


def _table(rng, n, R):
    a = rng.standard_normal((n, R // 2)) * 10
    c, s = np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)
    return torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda(), c.astype(np.float64), s.astype(np.float64)


def _strided(x):
    """The same [B, heads, N, D] as a slice of a token-major array with more heads."""
    B, H, N, D = x.shape
    big = torch.zeros(B, N, H + 3, D, dtype=x.dtype, device=x.device)
    big[:, :, 2:2 + H] = x.permute(0, 2, 1, 3)
    return big.permute(0, 2, 1, 3)[:, 2:2 + H]


def _wild(rng, shape):
    """Values of many sizes."""
    return rng.standard_normal(shape) * 2.0 ** rng.integers(-12, 6, shape[:-1] + (1,))


CASES = [
    # fmt, P, D, R, adjacent, N
    ("int8", 16, 64, 64, False, 1),
    ("e4m3", 16, 128, 128, True, 1),
    ("int8", 64, 128, 128, False, 77),
    ("e4m3", 64, 64, 32, False, 130),
    ("int8", 128, 128, 0, False, 300),
    ("e4m3", 128, 128, 96, True, 129),
    ("int8", 32, 64, 16, True, 33),
    ("e4m3", 32, 128, 128, False, 64),
    ("int8", 128, 64, 64, False, 5),
    ("e4m3", 16, 64, 48, False, 15),
]


@pytest.mark.parametrize("fmt,P,D,R,adjacent,N", CASES)
def test_ragged_chunks_behind_what_lists_hold(fmt, P, D, R, adjacent, N):
    rng = np.random.default_rng(N + P + D + R)
    B, H, Hq = 3, 2, 6
    k, k64 = bf16(_wild(rng, (B, H, N, D)))
    v, v64 = bf16(_wild(rng, (B, H, N, D)))
    q, q64 = bf16(_wild(rng, (B, Hq, N, D)))
    count = rng.integers(0, N + 1, (B, H))
    count[0, 0], count[1, 1] = N, 0
    held = count + rng.integers(0, 3 * P, (B, H))
    held[0, 1] = count[0, 1]  # an empty list before
    host = HostCache(rng, B, H, -(-(N + 3 * P) // P), P, D, fmt)
    pos0 = rng.integers(0, 50, B)
    cos, sin, c64, s64 = _table(rng, 50 + N, R) if R else (None, None, np.zeros((50 + N, 0)), np.zeros((50 + N, 0)))
    cache = host.gpu()
    got = kv.kvpop_cache_append(cache, _strided(k), _strided(v), i32(held), count=i32(count), q=_strided(q),
                                rotary=(cos, sin) if R else None, pos0=i32(pos0), adjacent=adjacent)
    for b in range(B):
        at = pos0[b] + np.arange(N)
        for h in range(H):
            n = count[b, h]
            host.append("k", cc.rotate(k64[b, h], c64[at], s64[at], adjacent)[:n], held[b, h], held[b, h] - n, b, h)
            host.append("v", v64[b, h, :n], held[b, h], held[b, h] - n, b, h)
    host.check(cache)
    at = pos0[:, None] + np.arange(N)
    want = cc.rotate(q64, c64[at][:, None], s64[at][:, None], adjacent)
    size = np.abs(q64)
    size = cc.rotate(size, np.abs(c64[at][:, None]), -np.abs(s64[at][:, None]), adjacent)  # |a c| + |b s| in its first half
    bound = 2.0 ** -8 * np.abs(want) + 3 * 2.0 ** -24 * (np.abs(size) + 2 * np.abs(q64).max(-1, keepdims=True))
    assert got.is_contiguous() and (np.abs(got.double().cpu().numpy() - want) <= bound).all()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("P,D", [(16, 64), (64, 128)])
def test_token_by_token_into_any_slot(fmt, P, D):
    """Lists grow, are full, and slots are taken over; scales grow by the way; idle lists (start
    -1) stay."""
    rng = np.random.default_rng(P)
    B, H, S = 2, 3, 2 * P + 5
    host = HostCache(rng, B, H, 3, P, D, fmt)
    cache = host.gpu()
    held = np.zeros((B, H), dtype=np.int64)
    for step in range(S + 30):
        k, k64 = bf16(_wild(rng, (B, H, 1, D)))
        v, v64 = bf16(_wild(rng, (B, H, 1, D)) * 2.0 ** (step / 20))
        start = np.where(held < S, held, rng.integers(-1, S, (B, H)))
        start[0, 1] = -1 if step % 3 == 0 else start[0, 1]
        held = np.where((start >= 0) & (held < S), held + 1, held)
        kv.kvpop_cache_append(cache, k, v, i32(held), start=i32(start))
        for b in range(B):
            for h in range(H):
                host.append("k", k64[b, h], held[b, h], start[b, h], b, h)
                host.append("v", v64[b, h], held[b, h], start[b, h], b, h)
    host.check(cache)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_gathered_tokens(fmt):
    """Each head its own tokens of a prompt, one token twice, some outside of it or of the table."""
    rng = np.random.default_rng(5)
    B, H, N, M, P, D = 2, 2, 90, 41, 32, 128
    k, k64 = bf16(_wild(rng, (B, H, N, D)))
    v, v64 = bf16(_wild(rng, (B, H, N, D)))
    src = rng.integers(0, N, (B, H, M))
    src[0, 0, 3] = src[0, 0, 30]
    src[0, 1, 5], src[0, 1, 6], src[1, 0, 0] = -1, N, 2 ** 31 - 1
    count = np.array([[M, M - 1], [1, 200]])
    cos, sin, c64, s64 = _table(rng, 80, D)  # positions 80 .. 89 lie outside
    host = HostCache(rng, B, H, 2, P, D, fmt)
    cache = host.gpu()
    held = np.minimum(count, M)
    kv.kvpop_cache_append(cache, k, v, i32(held), count=i32(count), src=i32(src), rotary=(cos, sin))
    for b in range(B):
        for h in range(H):
            n = held[b, h]
            x, y = np.zeros((n, D)), np.zeros((n, D))
            for i in range(n):
                t = src[b, h, i]
                if 0 <= t < N:
                    y[i] = v64[b, h, t]
                    x[i] = cc.rotate(k64[b, h, t], c64[t], s64[t], False) if t < 80 else 0
            host.append("k", x, n, 0, b, h)
            host.append("v", y, n, 0, b, h)
    host.check(cache)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_not_finite_values_and_the_range_of_scales(fmt):
    rng = np.random.default_rng(6)
    B, H, N, P, D = 1, 5, 20, 16, 64
    x = rng.standard_normal((B, H, N, D))
    x[0, 0, 3, 5], x[0, 0, 4, 6], x[0, 0, 5, 7] = np.nan, np.inf, -np.inf
    x[0, 1] *= 1e-12
    x[0, 2] *= 1e15   # beyond the largest scale
    x[0, 3] = 0.0
    x[0, 4, :, 0] = [127.0, 254.0, 448.0, 896.0, 63.5] * 4  # the borders themselves
    k, k64 = bf16(x)
    host = HostCache(rng, B, H, 2, P, D, fmt, exps=(-32, 32))
    cache = host.gpu()
    held = np.full((B, H), N)
    kv.kvpop_cache_append(cache, k, k, i32(held))
    for h in range(H):
        host.append("k", k64[0, h], N, 0, 0, h)
        host.append("v", k64[0, h], N, 0, 0, h)
    host.check(cache)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("adjacent", [False, True])
def test_not_finite_values_that_turn(fmt, adjacent):
    """An infinity or NaN reaches its pair's two codes and no other, whatever the angle (0 among
    them), and moves no scale."""
    rng = np.random.default_rng(12)
    B, H, N, P, D = 1, 3, 20, 16, 64
    x = rng.standard_normal((B, H, N, D))
    x[0, 0, 1, 5], x[0, 0, 2, 6], x[0, 0, 3, 40], x[0, 0, 16, 2] = np.nan, np.inf, -np.inf, np.inf
    k, k64 = bf16(x)
    cos, sin, c64, s64 = _table(rng, N, 32)
    c64[2], s64[2] = 1.0, 0.0
    c64[16, 2], s64[7, 3] = 0.0, np.inf
    cos, sin = torch.from_numpy(c64.astype(np.float32)).cuda(), torch.from_numpy(s64.astype(np.float32)).cuda()
    host = HostCache(rng, B, H, 2, P, D, fmt)
    cache = host.gpu()
    kv.kvpop_cache_append(cache, k, k, i32(np.full((B, H), N)), rotary=(cos, sin), adjacent=adjacent)
    for h in range(H):
        host.append("k", cc.rotate(k64[0, h], c64, s64, adjacent), N, 0, 0, h)
        host.append("v", k64[0, h], N, 0, 0, h)
    host.check(cache)


def test_rounding_borders_through_a_rotation():
    """Angles of 0, 90 and 45 degrees put sums on the borders between codes, exactly."""
    D, P = 64, 16
    rng = np.random.default_rng(7)
    x = (rng.integers(-254, 255, (1, 1, P, D)) / 2.0)
    x[..., 0] = 127.0
    for fmt in ("int8", "e4m3"):
        k, k64 = bf16(x)
        c = np.where(np.arange(P)[:, None] % 3 == 0, 1.0, np.where(np.arange(P)[:, None] % 3 == 1, 0.0, 0.5))
        c = np.broadcast_to(c, (P, D // 2)).astype(np.float32).copy()
        s = np.where(c == 1, 0, np.where(c == 0, 1, 0.5)).astype(np.float32)
        host = HostCache(rng, 1, 1, 1, P, D, fmt)
        cache = host.gpu()
        kv.kvpop_cache_append(cache, k, k, i32([[P]]), rotary=(torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()))
        host.append("k", cc.rotate(k64[0, 0], c.astype(np.float64), s.astype(np.float64), False), P, 0, 0, 0)
        host.append("v", k64[0, 0], P, 0, 0, 0)
        host.check(cache)


def test_entries_without_a_page_and_past_the_room():
    rng = np.random.default_rng(8)
    B, H, N, P, D = 1, 3, 40, 16, 64
    k, k64 = bf16(rng.standard_normal((B, H, N, D)))
    host = HostCache(rng, B, H, 2, P, D, "int8")
    host.table[0, 0, 1], host.table[0, 1, 0] = -1, 1 << 30
    cache = host.gpu()
    start = np.array([[0, 0, 25]])
    kv.kvpop_cache_append(cache, k, k, i32([[40, 40, 40]]), start=i32(start))  # 32 slots of room
    for h in range(H):
        for s in "kv":
            host.append(s, k64[0, h], 40, start[0, h], 0, h)
    host.check(cache)


def test_negative_default_start_and_idle_counts_write_nothing():
    rng = np.random.default_rng(9)
    k, _ = bf16(rng.standard_normal((1, 2, 4, 64)))
    host = HostCache(rng, 1, 2, 1, 16, 64, "e4m3")
    cache = host.gpu()
    kv.kvpop_cache_append(cache, k, k, i32([[3, 2]]))                       # fewer held than written
    kv.kvpop_cache_append(cache, k, k, i32([[9, 9]]), count=i32([[0, -5]]))
    host.check(cache)


def test_queries_alone_rotate_and_stay_zero_outside_the_table():
    rng = np.random.default_rng(10)
    cos, sin, c64, s64 = _table(rng, 10, 64)
    q, q64 = bf16(rng.standard_normal((2, 3, 4, 64)))
    k, _ = bf16(rng.standard_normal((2, 1, 4, 64)))
    host = HostCache(rng, 2, 1, 1, 16, 64, "int8")
    cache = host.gpu()
    out = kv.kvpop_cache_append(cache, k, k, i32([[4], [4]]), start=i32([[-1], [-1]]), q=q, rotary=(cos, sin),
                                pos0=i32([8, -2]))
    host.check(cache)
    out = out.double().cpu().numpy()
    assert (out[0, :, 2:] == 0).all() and (out[1, :, :2] == 0).all()
    for b, n, p in ((0, 0, 8), (0, 1, 9), (1, 2, 0), (1, 3, 1)):
        want = cc.rotate(q64[b, :, n], c64[p], s64[p], False)
        assert (np.abs(out[b, :, n] - want) <= 2.0 ** -8 * np.abs(want) + 3 * 2.0 ** -24 * 2 * np.abs(q64[b, :, n]).max()).all()


def test_a_pool_past_two_to_the_31_bytes():
    """Pages at byte offsets past 2^31 and 2^32."""
    P, D, n = 128, 128, (1 << 32) // (128 * 128) + 5
    pages = torch.zeros(n, P, D, dtype=torch.int8, device="cuda")
    exps = torch.zeros(n, dtype=torch.int8, device="cuda")
    table = i32([[[n - 1], [n // 2 + 3]]])
    v_pages = torch.zeros(n, P, D, dtype=torch.int8, device="cuda")
    cache = kv.KvpopCache(pages, v_pages, exps, exps.clone(), table)
    k, k64 = bf16(np.random.default_rng(11).standard_normal((1, 2, 3, D)))
    held = i32([[3, 3]])
    kv.kvpop_cache_append(cache, k, k, held)
    o, _ = kv.kvpop_cache_attn(k, cache, held, 0.1)
    for h, page in ((0, n - 1), (1, n // 2 + 3)):
        e = cc.needed_exponent(k64[0, h], "int8")
        want = cc.code_of(k64[0, h] * 2.0 ** -e, "int8").view(np.int8)
        for x in (pages, v_pages):
            np.testing.assert_array_equal(x[page, :3].cpu().numpy(), want)
        # the first query sees one token: its value is that token's
        np.testing.assert_allclose(o[0, h, 0].double().cpu().numpy(), want[0] * 2.0 ** e, rtol=2.0 ** -8)
    assert int((pages != 0).any(-1).sum()) <= 6
