"""kvpop_retain_prompt over prompts of many parts and of different lengths, and kvpop_retain_step's lists against
the running mask also where scores are NaN."""
import numpy as np
import pytest

import oracle
from oracle import compact_cache as cc

torch = pytest.importorskip("torch")
import paper_2607_05061_amd as kv  # noqa: E402
from cache_cases import i32  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("S", [1, 700, 6000])
@pytest.mark.parametrize("decay", [False, True])
def test_prompts_of_many_parts(S, decay):
    """Any lifetimes, prompts of up to five parts of 4096 positions: the kept tokens in order, then the empty slots."""
    T, H = 20001, 3
    n = np.array([T, 3 * 4096, 2 * 4096 + 1, 4096, 4095, 0, -5, 17, T + 9])
    rng = np.random.default_rng(S)
    ev = np.where(rng.random((len(n), H, T)) < 0.1, T + 5, rng.integers(0, T, (len(n), H, T))).astype(np.int32)
    ev[0, 0], ev[1, 1], ev[2, 2] = 0, T, np.where(np.arange(T) == 2 * 4096, T, 0)  # none, all, the last one
    r = rng.standard_normal((len(n), H, T)).astype(np.float32)
    lg = np.array([-1e-3, -0.1, 0.0], dtype=np.float32) if decay else np.zeros(H, dtype=np.float32)
    pos, prio, held = kv.kvpop_retain_prompt(torch.from_numpy(ev).cuda(), torch.from_numpy(r).cuda(), S, lens=i32(n),
                                             log_gamma=torch.from_numpy(lg).cuda() if decay else None)
    pos, prio, held = pos.cpu().numpy(), prio.cpu().numpy(), held.cpu().numpy()
    for b in range(len(n)):
        m = min(max(int(n[b]), 0), T)
        for h in range(H):
            want = np.flatnonzero(ev[b, h, :m] >= m)[:S]
            assert held[b, h] == len(want), (b, h)
            np.testing.assert_array_equal(pos[b, h, :len(want)], want)
            np.testing.assert_array_equal(prio[b, h, :len(want)], oracle.static_priority_f32(r[b, h], lg[h])[want])
            assert (pos[b, h, len(want):] == -1).all() and np.isneginf(prio[b, h, len(want):]).all()


@pytest.mark.parametrize("s,w,k", [(2, 3, 4), (4, 16, 300), (0, 300, 5), (0, 0, 3), (5, 2, 1)])
def test_lists_are_the_running_mask_with_nan_too(s, w, k):
    """Ranks by the priorities' bits, as the library orders them; every list is compared, after every 25 tokens."""
    B, H, T, S = 2, 2, s + w + k + 75, s + w + k
    rng = np.random.default_rng(s + w + k)
    r = np.round(rng.standard_normal((B, H, T)), 1).astype(np.float32)
    flat = r.reshape(-1)
    for x in (-0.0, 0.0, -np.inf, np.inf, np.nan, -np.float32(np.nan)):
        flat[rng.integers(0, flat.size, max(1, flat.size // 40))] = x
    lg = np.array([-0.01, -0.2], dtype=np.float32)
    order = [[np.array([cc._order(x) for x in oracle.static_priority_f32(r[b, h], lg[h])]) for h in range(H)] for b in range(B)]
    pos = torch.full((B, H, S), -7, dtype=torch.int32, device="cuda")
    prio, held = torch.zeros(B, H, S, device="cuda"), torch.zeros(B, H, dtype=torch.int32, device="cuda")
    dev_lg, compared = torch.from_numpy(lg).cuda(), 0
    for q in range(T):
        kv.kvpop_retain_step(torch.from_numpy(r[..., max(0, q - w)].copy()).cuda(), i32([q] * B), pos, prio, held, s, w, k,
                             log_gamma=dev_lg)
        if q % 25 != 24 and q != T - 1:
            continue
        gp, gh = pos.cpu().numpy(), held.cpu().numpy()
        for b in range(B):
            for h in range(H):
                rank = oracle.ranks_from_priority(order[b][h][:q + 1])
                tau = oracle.running_cutoff_fenwick(rank, s, w, k)
                mask = oracle.running_topk_mask_rows(rank, tau, s, w, [q])[0]
                assert sorted(gp[b, h, :gh[b, h]].tolist()) == np.flatnonzero(mask).tolist(), (q, b, h)
                compared += 1
    assert compared >= 4 * B * H and np.isnan(r).any()
