"""kvpop_cache_attn against the fp64 oracle on the same codes (tolerance: derived in
cache_cases.attention_check)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2607_05061_amd as kv  # noqa: E402
from cache_cases import HostCache, attention_check, bf16, i32  # noqa: E402

pytestmark = pytest.mark.gpu


def _run(rng, B, Hq, H, N, D, P, fmt, held, q_lens=None, room=None, exps=(-6, 3), scale=None, q_gain=1.0):
    held = np.asarray(held).reshape(B, H)
    per = max(1, -(-max(int(held.max()), room or 0) // P))
    host = HostCache(rng, B, H, per, P, D, fmt, exps=exps)
    # codes of ordinary size: logits of a few units
    scale = (1.0 / (D ** 0.5 * (64 if fmt == "int8" else 100))) if scale is None else scale
    q, q64 = bf16(rng.standard_normal((B, Hq, N, D)) * q_gain)
    o, lse = kv.kvpop_cache_attn(q, host.gpu(), i32(held), scale, q_lens=None if q_lens is None else i32(q_lens))
    attention_check(q64, host, held, float(np.float32(scale)), o, lse, q_lens)
    return o, lse


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
def test_single_tokens_over_ragged_lists(fmt, D, P):
    rng = np.random.default_rng(P + D)
    _run(rng, 4, 8, 2, 1, D, P, fmt, [[0, 1], [31, 32], [33, 500], [P, 2 * P + 1]])


@pytest.mark.parametrize("Hq,H", [(1, 1), (3, 1), (7, 1), (16, 1), (17, 1), (40, 2), (8, 8)])
@pytest.mark.parametrize("N", [1, 3, 5])
def test_head_groups_and_drafts(Hq, H, N):
    rng = np.random.default_rng(Hq + 100 * N)
    held = rng.integers(0, 300, (2, H))
    held[0, 0] = 2  # fewer tokens than queries: the first ones see nothing
    _run(rng, 2, Hq, H, N, 64, 32, "int8", held)


@pytest.mark.parametrize("fmt,D,P,G", [("int8", 128, 64, 4), ("e4m3", 128, 16, 1), ("int8", 64, 128, 3), ("e4m3", 64, 32, 8)])
@pytest.mark.parametrize("N,held", [(9, 9), (64, 200), (65, 64), (130, 777), (257, 1025)])
def test_chunks(fmt, D, P, G, N, held):
    rng = np.random.default_rng(N + held + P)
    _run(rng, 2, 2 * G, 2, N, D, P, fmt, [[held, max(0, held - 70)], [held // 2, held + 5]])


def test_ragged_queries():
    rng = np.random.default_rng(1)
    _run(rng, 5, 4, 2, 33, 128, 64, "int8", rng.integers(30, 400, (5, 2)), q_lens=[33, 0, 1, 17, 90])
    _run(rng, 5, 4, 2, 2, 128, 64, "e4m3", rng.integers(0, 400, (5, 2)), q_lens=[2, 0, 1, -3, 2])


def test_long_list_in_many_parts():
    """More parts than one workgroup takes, and a list that fills only a few of them."""
    rng = np.random.default_rng(2)
    _run(rng, 1, 4, 2, 1, 128, 64, "int8", [[40000, 70]])
    _run(rng, 1, 4, 2, 1, 64, 128, "e4m3", [[9000, 0]], room=100000)
    _run(rng, 1, 2, 1, 200, 64, 64, "int8", [[20000]])


@pytest.mark.parametrize("N", [1, 40, 120])
def test_scales_of_every_size(N):
    """Exponents over their whole range: a few pages hold all the mass, or values of any size."""
    rng = np.random.default_rng(3)
    for fmt in ("int8", "e4m3"):
        host = HostCache(rng, 2, 2, 12, 16, 64, fmt)
        host.side["v"][1][:] = rng.integers(-32, 33, len(host.side["v"][1]))
        host.side["k"][1][:] = rng.integers(-12, -3, len(host.side["k"][1]))
        q, q64 = bf16(rng.standard_normal((2, 4, N, 64)))
        held = rng.integers(100, 192, (2, 2))
        o, lse = kv.kvpop_cache_attn(q, host.gpu(), i32(held), 0.125)
        attention_check(q64, host, held, 0.125, o, lse)


@pytest.mark.parametrize("N", [1, 40, 120])
def test_sharp_and_flat_logits_and_queries_of_any_size(N):
    rng = np.random.default_rng(4)
    _run(rng, 1, 4, 2, N, 128, 64, "int8", [[900, 333]], scale=0.5)      # one key takes nearly all
    _run(rng, 1, 4, 2, N, 128, 64, "int8", [[900, 333]], q_gain=0.0)     # all keys alike
    _run(rng, 1, 4, 2, N, 64, 64, "e4m3", [[500, 64]], scale=1e-6, q_gain=1e5)
    _run(rng, 1, 4, 2, N, 64, 64, "e4m3", [[500, 64]], scale=1e3, q_gain=1e-9)


@pytest.mark.parametrize("N", [1, 6, 40, 120])
def test_growing_logits_move_the_maximum(N):
    """Each key's logit is above all before it: the running maximum moves in every step."""
    D, P, L = 64, 16, 640
    rng = np.random.default_rng(5)
    host = HostCache(rng, 1, 1, L // P, P, D, "int8", exps=(0, 0))
    for j in range(L):
        row = host.side["k"][0][host.table[0, 0, j // P], j % P].view(np.int8)
        row[:] = 0
        row[:6] = np.clip(j - 127 * np.arange(6), 0, 127)
    q = np.zeros((1, 1, N, D))
    q[..., :6] = 1.0
    qg, q64 = bf16(q)
    for scale in (0.05, 1.0):
        o, lse = kv.kvpop_cache_attn(qg, host.gpu(), i32([[L]]), scale)
        attention_check(q64, host, [[L]], float(np.float32(scale)), o, lse)


@pytest.mark.parametrize("N", [1, 40, 120])
def test_bytes_that_are_not_seen_do_not_matter(N):
    """Slots past a list's end hold NaN codes; entries without a page are left out; spare pages too."""
    rng = np.random.default_rng(6)
    held = np.array([[70, 33], [200, 5]])
    host = HostCache(rng, 2, 2, 8, 32, 128, "e4m3")
    host.table[1, 0, 2], host.table[1, 0, 4] = -1, len(host.side["k"][0])
    for b in range(2):
        for h in range(2):
            for p in range(8):
                t = host.table[b, h, p]
                if 0 <= t < len(host.side["k"][0]):
                    for s in "kv":
                        host.side[s][0][t, max(0, held[b, h] - 32 * p):] = 0x7F
    q, q64 = bf16(rng.standard_normal((2, 4, N, 128)))
    scale = 0.001
    o, lse = kv.kvpop_cache_attn(q, host.gpu(), i32(held), scale)
    attention_check(q64, host, held, float(np.float32(scale)), o, lse)
    host.table[:] = -1
    o, lse = kv.kvpop_cache_attn(q, host.gpu(), i32(held), scale)
    assert (o == 0).all() and torch.isneginf(lse).all()


def test_lists_share_pages():
    rng = np.random.default_rng(7)
    host = HostCache(rng, 3, 2, 4, 16, 64, "int8")
    host.table[:, :, :2] = host.table[0, 0, :2]
    q, q64 = bf16(rng.standard_normal((3, 2, 1, 64)))
    held = rng.integers(20, 64, (3, 2))
    o, lse = kv.kvpop_cache_attn(q, host.gpu(), i32(held), 0.01)
    attention_check(q64, host, held, float(np.float32(0.01)), o, lse)


@pytest.mark.parametrize("N", [1, 50, 120])
def test_a_query_that_is_not_finite_stays_by_itself(N):
    rng = np.random.default_rng(8)
    host = HostCache(rng, 1, 2, 10, 16, 64, "int8")
    held = np.array([[150, 150]])
    q, q64 = bf16(rng.standard_normal((1, 4, N, 64)))
    ref, rl = kv.kvpop_cache_attn(q, host.gpu(), i32(held), 0.01)
    q2 = q.clone()
    q2[0, 1, N // 2, 3] = float("nan")
    q2[0, 2, 0, 0] = float("inf")
    o, lse = kv.kvpop_cache_attn(q2, host.gpu(), i32(held), 0.01)
    same = torch.ones(4, N, dtype=torch.bool)
    same[1, N // 2], same[2, 0] = False, False
    assert torch.equal(o[0].cpu()[same], ref[0].cpu()[same]) and torch.equal(lse[0].cpu()[same], rl[0].cpu()[same])
    assert not torch.isfinite(o[0, 1, N // 2]).any()


def test_held_beyond_the_room_and_strided_queries():
    rng = np.random.default_rng(9)
    host = HostCache(rng, 2, 1, 3, 16, 64, "int8")
    q, q64 = bf16(rng.standard_normal((2, 5, 4, 64)))
    big = torch.zeros(2, 4, 9, 64, dtype=torch.bfloat16, device="cuda")
    big[:, :, 3:8] = q.permute(0, 2, 1, 3)
    held = np.array([[1 << 30], [-7]])
    o, lse = kv.kvpop_cache_attn(big.permute(0, 2, 1, 3)[:, 3:8], host.gpu(), i32(held), 0.01)
    attention_check(q64, host, held, float(np.float32(0.01)), o, lse)


@pytest.mark.parametrize("N", [1, 100])
def test_results_do_not_depend_on_the_run(N):
    rng = np.random.default_rng(10)
    host = HostCache(rng, 2, 4, 40, 64, 128, "int8")
    cache, held = host.gpu(), i32(rng.integers(1000, 2560, (2, 4)))
    q, _ = bf16(rng.standard_normal((2, 16, N, 128)))
    a = kv.kvpop_cache_attn(q, cache, held, 0.01)
    for _ in range(3):
        b = kv.kvpop_cache_attn(q, cache, held, 0.01)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("fmt,D", [("int8", 128), ("e4m3", 64)])
@pytest.mark.parametrize("B,H,G,N", [(1, 8, 4, 20), (1, 8, 4, 21), (4, 8, 4, 8), (4, 8, 4, 9), (1, 31, 3, 11), (1, 32, 3, 11)])
def test_both_sides_of_the_line_between_the_kernels(fmt, D, B, H, G, N):
    rng = np.random.default_rng(B * H * G * N)
    _run(rng, B, H * G, H, N, D, 32, fmt, rng.integers(0, 700, (B, H)))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,H", [(32, 8), (33, 8), (64, 8), (65, 8), (1, 255)])
def test_as_many_lists_as_workgroups_fit(B, H, D):
    rng = np.random.default_rng(B * H + D)
    _run(rng, B, H, H, 1, D, 64, "int8", rng.integers(0, 600, (B, H)), room=600)
