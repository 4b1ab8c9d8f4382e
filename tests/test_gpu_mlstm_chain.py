"""The recurrence with what ranks, keeps and reads by it: a served KVpop model from its prompt on, and a training step
of its scorer."""
import numpy as np
import pytest

from oracle import compact_cache as cc

torch = pytest.importorskip("torch")
import paper_2607_05061_amd as kv  # noqa: E402
from cache_cases import bf16, i32  # noqa: E402
from mlstm_cases import inputs, on_gpu  # noqa: E402

pytestmark = pytest.mark.gpu


def test_a_served_model_keeps_what_its_scores_say():
    """A prompt: read-outs, scores, running top-k, retention, pages. Then tokens: one step of the recurrence, the score
    of the token that leaves the window, its slot, its row, attention. The slots are the oracle's for the same scores, and
    the scores those of the whole sequence."""
    rng = np.random.default_rng(0)
    B, H, T, n, D, s, w, k = 2, 2, 120, 80, 64, 2, 6, 30
    S, scale = s + w + k, D ** -0.5
    x, _ = on_gpu(inputs(rng, B, H, T, D))
    a = [x[y] for y in ("q", "k", "v", "ig", "fg")]
    head = torch.from_numpy(rng.standard_normal((H, 1, D))).float().cuda()
    score = lambda o: (head[:, :, :] * torch.nn.functional.silu(o.float())).sum(-1) if o.dim() == 4 else (head[:, 0] * torch.nn.functional.silu(o.float())).sum(-1)  # noqa: E731
    whole, _ = kv.kvpop_mlstm_fwd(*a, delay=w)
    state = kv.kvpop_mlstm_empty(B, H, D)
    o, _ = kv.kvpop_mlstm_fwd(*(y[:, :, :n] for y in a), delay=w, state=state)
    r = score(o).contiguous()
    evict = kv.kvpop_running_topk(r, s, w, k, evict=True)["evict"]
    pos, prio, held = kv.kvpop_retain_prompt(evict, r, S)
    keys, vals = (bf16(rng.standard_normal((B, H, T, D)))[0] for _ in range(2))
    cache = kv.kvpop_cache_empty(B, H, S, D, 16)
    kv.kvpop_cache_append(cache, keys[:, :, :n], vals[:, :, :n], held, count=held, src=pos)
    states = [[{j: [int(pos[b, h, j]), np.float32(prio[b, h, j].item())] for j in range(int(held[b, h]))} for h in range(H)] for b in range(B)]
    ones = torch.ones_like(held)
    for t in range(n, T):
        ro = kv.kvpop_mlstm_step(x["q"][:, :, t - w], *(y[:, :, t] for y in a[1:]), state)
        # two roundings of o apart, and of its terms, which are no larger together than the largest |v|
        assert (ro.float() - whole[:, :, t - w].float()).abs().max() <= 4 * 2.0 ** -8 * x["v"].float().abs().max()
        rt = score(ro).contiguous()
        want = [[cc.retain_step(states[b][h], t, np.float32(rt[b, h].item()), 0.0, s, w, k) for h in range(H)] for b in range(B)]
        slot = kv.kvpop_retain_step(rt, i32([t] * B), pos, prio, held, s, w, k)
        assert slot.tolist() == want
        kv.kvpop_cache_append(cache, keys[:, :, t:t + 1], vals[:, :, t:t + 1], held, count=ones, start=slot)
        out, lse = kv.kvpop_cache_attn(bf16(rng.standard_normal((B, 2 * H, 1, D)))[0], cache, held, scale)
        assert out.isfinite().all() and lse.isfinite().all()


def test_a_training_step_of_the_scorer():
    """Scores from the differentiable recurrence, the target from attention, the boundary tokens of the running top-k, the
    pairwise loss: the gradients that reach q, k, v and the gates are the backward pass's for the loss's own do."""
    rng = np.random.default_rng(1)
    B, H, G, T, D, s, w, k = 1, 2, 2, 200, 64, 2, 8, 40
    x, _ = on_gpu(inputs(rng, B, H, T, D), tokens=True)
    a = [x[y].detach().requires_grad_() for y in ("q", "k", "v", "ig", "fg")]
    head = torch.from_numpy(rng.standard_normal((H, 1, D))).float().cuda()
    q, _ = bf16(rng.standard_normal((B, H * G, T, D)))
    key, _ = bf16(rng.standard_normal((B, H, T, D)))
    _, lse = kv.kvpop_future_attn_target(q, key, D ** -0.5, w)
    target, _ = kv.kvpop_future_attn_scores(q, key, lse, D ** -0.5, w)

    def loss(o):
        r = (head * torch.nn.functional.silu(o.float())).sum(-1)
        top = kv.kvpop_running_topk(target, s, w, k)
        u = torch.arange(T, device="cuda")
        new = (u - w).clamp(min=0)
        bnd = top["boundary"].long()
        use = (bnd >= 0) & (u >= s + w + k)
        y = torch.where(torch.gather(target, 2, new.expand(B, H, T)) > torch.gather(target, 2, bnd.clamp(min=0)), 1.0, -1.0)
        d = torch.gather(r, 2, new.expand(B, H, T)) - torch.gather(r, 2, bnd.clamp(min=0))
        return (torch.nn.functional.softplus(-y * d) * use).sum() / use.sum()

    o = kv.kvpop_mlstm(*a, delay=w)
    o.retain_grad()
    loss(o).backward()
    assert o.grad.abs().sum() > 0
    ro, rl = kv.kvpop_mlstm_fwd(*(y.detach() for y in a), delay=w)
    assert torch.equal(o, ro)
    want = kv.kvpop_mlstm_bwd(o.grad, *(y.detach() for y in a), ro, rl, delay=w)
    for y, g in zip(a, want):
        assert torch.equal(y.grad, g) and g.isfinite().all() and g.abs().sum() > 0


def test_what_the_binding_refuses():
    x, _ = on_gpu(inputs(np.random.default_rng(2), 1, 2, 400, 64))
    a = [x[y] for y in ("q", "k", "v", "ig", "fg")]
    o, lse = kv.kvpop_mlstm_fwd(*a)
    st = kv.kvpop_mlstm_empty(1, 2, 64)
    need = kv.kvpop_mlstm_fwd_workspace_size(1, 2, 400, 64)
    byte = torch.empty(1, dtype=torch.uint8, device="cuda")
    for bad in (byte.expand(need), torch.empty(need - 1, dtype=torch.uint8, device="cuda"), torch.empty(need, dtype=torch.uint8)):
        with pytest.raises(ValueError, match="workspace"):
            kv.kvpop_mlstm_fwd(*a, workspace=bad)
    with pytest.raises(ValueError, match="workspace"):
        kv.kvpop_mlstm_bwd(x["do"], *a, o, lse, workspace=byte.expand(1 << 30))
    for i, bad in ((0, a[0].float()), (3, a[3].float()), (4, a[4].half())):
        with pytest.raises(TypeError):
            kv.kvpop_mlstm_fwd(*(bad if j == i else y for j, y in enumerate(a)))
    for i, bad in ((1, a[1][:, :, :-1]), (2, a[2][..., ::2]), (3, a[3][:, :, :-1]), (1, a[1].transpose(2, 3).contiguous().transpose(2, 3)),
                   (4, a[4].cpu())):
        with pytest.raises(ValueError):
            kv.kvpop_mlstm_fwd(*(bad if j == i else y for j, y in enumerate(a)))
    with pytest.raises(ValueError):
        kv.kvpop_mlstm_fwd(*a, state=st._replace(z=st.z[:, :1]))
    with pytest.raises(ValueError):
        kv.kvpop_mlstm_fwd(*a, state=st._replace(m=None))
    with pytest.raises(kv.KvpopError):
        kv.kvpop_mlstm_fwd(*a, state=st._replace(m=st.z[0, 0, :2].view(1, 2)))  # the state over itself
    with pytest.raises(ValueError):
        kv.kvpop_mlstm_fwd(*a, lens=i32([1, 2]))
    with pytest.raises(ValueError):
        kv.kvpop_mlstm_bwd(x["do"], *a, o, None)
    with pytest.raises(TypeError):
        kv.kvpop_mlstm_step(*(y[:, :, 0].float() for y in a), st)
    with pytest.raises(ValueError):
        kv.kvpop_mlstm_step(*(y[:, :, 0] for y in a[:4]), a[4][:, :1, 0], st)
    with pytest.raises(kv.KvpopError):
        kv.kvpop_mlstm_fwd(*a, o=a[0])
    with pytest.raises(kv.KvpopError):
        kv.kvpop_mlstm_fwd(*a, delay=-1)
