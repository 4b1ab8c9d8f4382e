"""kvpop_retain_step and kvpop_retain_prompt against the running top-k mask: what a list
holds has to be exactly what the mask keeps, and slots, positions and priorities exactly the
oracle's."""
import numpy as np
import pytest

import oracle
from oracle import compact_cache as cc

torch = pytest.importorskip("torch")
import paper_2607_05061_amd as kv  # noqa: E402
from cache_cases import i32  # noqa: E402

pytestmark = pytest.mark.gpu


def _scores(rng, shape):
    r = np.round(rng.standard_normal(shape), 1).astype(np.float32)  # with ties
    flat = r.reshape(-1)
    for x in (-0.0, 0.0, -np.inf, np.inf, np.nan):
        flat[rng.integers(0, flat.size, max(1, flat.size // 50))] = x
    return r


def _empty(B, H, S):
    return (torch.full((B, H, S), 77, dtype=torch.int32, device="cuda"), torch.full((B, H, S), 7.0, device="cuda"),
            torch.zeros(B, H, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("s,w,k,S", [(2, 3, 4, 9), (0, 1, 2, 3), (0, 0, 3, 3), (2, 0, 1, 5), (5, 2, 1, 8),
                                     (4, 16, 300, 333), (0, 300, 5, 305)])
@pytest.mark.parametrize("decay", [False, True])
def test_tokens_one_at_a_time(s, w, k, S, decay):
    B, H, T = 3, 2, s + w + k + 60
    rng = np.random.default_rng(s + 10 * w + k)
    r = _scores(rng, (B, H, T))
    lg = np.array([-0.01, -0.2], dtype=np.float32) if decay else np.zeros(2, dtype=np.float32)
    dev_lg = torch.from_numpy(lg).cuda() if decay else None
    pos, prio, held = _empty(B, H, S)
    states = [[{} for _ in range(H)] for _ in range(B)]
    now = [0, 0, 0]
    for step in range(T):
        q = np.array([now[0], now[1] if step % 4 else -1, now[2]])
        sc = np.array([[r[b, h, q[b] - w] if q[b] >= w else 0.5 for h in range(H)] for b in range(B)], dtype=np.float32)
        slot = kv.kvpop_retain_step(torch.from_numpy(sc).cuda(), i32(q), pos, prio, held, s, w, k, log_gamma=dev_lg)
        want = np.array([[cc.retain_step(states[b][h], int(q[b]), sc[b, h], float(lg[h]), s, w, k) for h in range(H)]
                         for b in range(B)])
        np.testing.assert_array_equal(slot.cpu().numpy(), want)
        now = [n + 1 if x >= 0 else n for n, x in zip(now, q)]
    gp, gr, gh = pos.cpu().numpy(), prio.cpu().numpy(), held.cpu().numpy()
    for b in range(B):
        for h in range(H):
            st = states[b][h]
            assert gh[b, h] == len(st)
            np.testing.assert_array_equal(gp[b, h, :len(st)], [st[i][0] for i in range(len(st))])
            np.testing.assert_array_equal(gr[b, h, :len(st)], [st[i][1] for i in range(len(st))])
            assert (gp[b, h, len(st):] == 77).all()
            # the list is what the mask keeps at its last query
            n = now[b]
            rank = oracle.ranks_from_priority(oracle.static_priority_f32(r[b, h, :n], lg[h])) if not np.isnan(
                r[b, h, :n]).any() else None
            if rank is not None:
                tau = oracle.running_cutoff_fenwick(rank, s, w, k)
                mask = oracle.running_topk_mask_rows(rank, tau, s, w, [n - 1])[0]
                assert sorted(gp[b, h, :len(st)].tolist()) == np.flatnonzero(mask).tolist()


@pytest.mark.parametrize("T", [1, 2, 63, 64, 65, 1000, 1024, 1025, 5000])
@pytest.mark.parametrize("lens", [False, True])
def test_prompt_keeps_what_the_last_query_keeps(T, lens):
    B, H, s, w, k = 3, 2, 4, 16, 100
    S = s + w + k + 3
    rng = np.random.default_rng(T)
    r = _scores(rng, (B, H, T))
    r = np.where(np.isnan(r), np.float32(0.25), r)
    lg = np.array([-1e-3, -0.1], dtype=np.float32)
    sc = torch.from_numpy(r).cuda()
    ev = kv.kvpop_running_topk(sc, s, w, k, log_gamma=torch.from_numpy(lg).cuda(), evict=True)["evict"]
    n = np.array([T, T // 2, -1 if T > 2 else T + 5])
    pos, prio, held = kv.kvpop_retain_prompt(ev, sc, S, log_gamma=torch.from_numpy(lg).cuda(),
                                             lens=i32(n) if lens else None)
    pos, prio, held = pos.cpu().numpy(), prio.cpu().numpy(), held.cpu().numpy()
    n = np.clip(n, 0, T) if lens else np.full(B, T)
    for b in range(B):
        for h in range(H):
            want = []
            if n[b]:
                rank = oracle.ranks_from_priority(oracle.static_priority_f32(r[b, h, :n[b]], lg[h]))
                tau = oracle.running_cutoff_fenwick(rank, s, w, k)
                want = np.flatnonzero(oracle.running_topk_mask_rows(rank, tau, s, w, [n[b] - 1])[0])
            m = len(want)
            assert held[b, h] == m
            np.testing.assert_array_equal(pos[b, h, :m], want)
            np.testing.assert_array_equal(prio[b, h, :m], oracle.static_priority_f32(r[b, h], lg[h])[want] if m else [])
            assert (pos[b, h, m:] == -1).all() and np.isneginf(prio[b, h, m:]).all()


def test_prompt_then_tokens_is_tokens_alone():
    """From a prompt's lists on, the same tokens are held as when every token came alone."""
    B, H, s, w, k, T, n = 2, 2, 2, 5, 20, 90, 50
    rng = np.random.default_rng(1)
    r = torch.from_numpy(np.round(rng.standard_normal((B, H, T)), 1).astype(np.float32)).cuda()
    ev = kv.kvpop_running_topk(r[..., :n].contiguous(), s, w, k, evict=True)["evict"]
    a = kv.kvpop_retain_prompt(ev, r[..., :n].contiguous(), s + w + k)
    b = _empty(B, H, s + w + k)
    for q in range(T):
        sc = r[..., max(0, q - w)].contiguous()
        kv.kvpop_retain_step(sc, i32([q] * B), *b, s, w, k)
        if q >= n:
            kv.kvpop_retain_step(sc, i32([q] * B), *a, s, w, k)
        if q >= n - 1:
            assert torch.equal(a[2], b[2])
            assert torch.equal(a[0].sort(-1).values, b[0].sort(-1).values)


def test_budget_smaller_than_what_is_kept_drops_the_last():
    T = 2000
    ev = torch.full((1, 1, T), T, dtype=torch.int32, device="cuda")
    r = torch.arange(T, dtype=torch.float32, device="cuda").view(1, 1, T)
    pos, prio, held = kv.kvpop_retain_prompt(ev, r, 1300)
    assert held.item() == 1300 and torch.equal(pos[0, 0].cpu(), torch.arange(1300, dtype=torch.int32))
    assert torch.equal(prio[0, 0], r[0, 0, :1300])


def test_a_list_without_an_eligible_token_gives_no_slot():
    """Full of tokens that are all sinks or newer than the one that leaves the window."""
    pos = i32([[[0, 9, 10, 8]]])
    prio = torch.zeros(1, 1, 4, device="cuda")
    held = i32([[4]])
    slot = kv.kvpop_retain_step(torch.zeros(1, 1, device="cuda"), i32([11]), pos, prio, held, 1, 2, 1)
    assert slot.item() == 1  # position 9 leaves the window and competes with 8, the latest of equals goes
    pos = i32([[[0, 10, 11, 12]]])
    slot = kv.kvpop_retain_step(torch.zeros(1, 1, device="cuda"), i32([11]), pos, prio, held, 1, 2, 1)
    assert slot.item() == -1 and pos.flatten().tolist() == [0, 10, 11, 12] and held.item() == 4
