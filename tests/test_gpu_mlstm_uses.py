"""Uses of the mLSTM recurrence beside plain calls: a differentiable pass in a graph, inputs shared by heads, states
that idle and masked tokens pass, sequences behind large gates."""
import numpy as np
import pytest

from oracle import mlstm as om

torch = pytest.importorskip("torch")
import paper_2607_05061_amd as kv  # noqa: E402
from cache_cases import i32  # noqa: E402
from mlstm_cases import inputs, on_gpu  # noqa: E402

pytestmark = pytest.mark.gpu
ARGS = ("q", "k", "v", "ig", "fg")


def test_a_captured_differentiable_pass():
    """torch.autograd.grad inside a capture, replayed with other inputs, eager work between."""
    rng = np.random.default_rng(30)
    B, H, T, D = 1, 3, 500, 64
    x, _ = on_gpu(inputs(rng, B, H, T, D), tokens=True)
    a = [x[n].detach().requires_grad_() for n in ARGS]

    def step():
        o = kv.kvpop_mlstm(*a, scale=0.3, delay=7)
        return (o.detach(), *torch.autograd.grad(o, a, x["do"]))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        y, _ = on_gpu(inputs(rng, B, H, T, D), tokens=True)
        with torch.no_grad():
            for n, t in zip(ARGS, a):
                t.copy_(y[n])
            x["do"].copy_(y["do"])
        graph.replay()
        torch.cuda.synchronize()
        got = [z.clone() for z in out]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(p, r) for p, r in zip(got, want))


def test_two_graphs_replayed_in_turn():
    """Each graph has memory of its own: neither sees the other's."""
    rng = np.random.default_rng(31)
    x, _ = on_gpu(inputs(rng, 1, 2, 700, 64))
    y, _ = on_gpu(inputs(rng, 1, 2, 900, 64))
    cases = [[z[n] for n in ARGS] for z in (x, y)]
    want = [kv.kvpop_mlstm_fwd(*a) for a in cases]
    torch.cuda.synchronize()
    graphs, out = [], []
    for a in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out.append(kv.kvpop_mlstm_fwd(*a))
        graphs.append(g)
    for i in (0, 1, 1, 0, 1):
        for t in out[i]:
            t.fill_(7)
        graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, r) for p, r in zip(out[i], want[i]))


def test_keys_and_gates_shared_by_heads():
    """Expanded inputs (stride 0) are read as they are; a leaf gets the sum of its heads' gradients. Each head's is
    rounded to bf16, torch's sum by 2^-8 of each partial sum at most."""
    rng = np.random.default_rng(32)
    B, H, T, D = 2, 4, 333, 64
    x, _ = on_gpu(inputs(rng, B, H, T, D), tokens=True)
    k, ig = (x[n][:, :1].contiguous().requires_grad_() for n in ("k", "ig"))
    q, v, fg = (x[n] for n in ("q", "v", "fg"))
    o = kv.kvpop_mlstm(q, k.expand(B, H, T, D), v, ig.expand(B, H, T), fg, delay=3)
    full = [q, k.detach().expand(B, H, T, D).contiguous(), v, ig.detach().expand(B, H, T).contiguous(), fg]
    ro, lse = kv.kvpop_mlstm_fwd(*full, delay=3)
    assert torch.equal(o, ro)
    _, dk, _, dig, _ = kv.kvpop_mlstm_bwd(x["do"], *full, ro, lse, delay=3)
    o.backward(x["do"])
    for got, parts in ((k.grad, dk), (ig.grad, dig)):
        want = parts.double().sum(1, keepdim=True)
        bound = 2.0 ** -8 * H * parts.double().abs().sum(1, keepdim=True)  # a rounding per addend, whatever the order
        assert ((got.double() - want).abs() <= bound + 1e-30).all()


@pytest.mark.parametrize("T", [1, 70, 700])
def test_an_empty_sequence_keeps_its_state_bit_for_bit(T):
    rng = np.random.default_rng(33 + T)
    B, H, D = 3, 2, 64
    x, _ = on_gpu(inputs(rng, B, H, T, D))
    a = [x[n] for n in ARGS]
    st = kv.kvpop_mlstm_empty(B, H, D)
    kv.kvpop_mlstm_fwd(*a, state=st)
    before = [t.clone() for t in st]
    kv.kvpop_mlstm_fwd(*a, state=st, lens=i32([0, T, 0]))
    for t, w in zip(st, before):
        assert torch.equal(t[0], w[0]) and torch.equal(t[2], w[2])
    whole = [t.clone() for t in before]  # the other one is what it is where all sequences have tokens
    kv.kvpop_mlstm_fwd(*a, state=kv.KvpopMlstmState(*whole))
    assert all(torch.equal(t[1], w[1]) for t, w in zip(st, whole))
    kv.kvpop_mlstm_step(*(y[:, :, 0] for y in a), st, active=i32([0, 1, 0]))
    for t, w in zip(st, before):
        assert torch.equal(t[0], w[0]) and torch.equal(t[2], w[2])


@pytest.mark.parametrize("T", [64, 600])
def test_a_state_outlives_masked_tokens(T):
    """ig = -inf and fg = -40 over T tokens: what is held keeps its elements' ratios, m falls by T log f; the next read-out
    is that of before (the factor cancels): a rounding of o on each side, of a read state's elements (2^-8 each)
    and fp32 sums."""
    rng = np.random.default_rng(34)
    B, H, D = 1, 2, 64
    x, _ = on_gpu(inputs(rng, B, H, 100, D))
    a = [x[n] for n in ARGS]
    st = kv.kvpop_mlstm_empty(B, H, D)
    kv.kvpop_mlstm_fwd(*a, state=st)
    C, z, m = (t.clone() for t in st)
    y, _ = on_gpu(inputs(rng, B, H, T, D))
    y["ig"].fill_(float("-inf"))
    y["fg"].fill_(-40.0)
    y["k"].fill_(float("nan"))
    o, _ = kv.kvpop_mlstm_fwd(*(y[n] for n in ARGS), state=st)
    fall = T * 40.0
    assert ((st.m - (m - fall)).abs() <= 2.0 ** -22 * (fall + m.abs())).all()
    for now, was in ((st.C, C), (st.z, z)):
        assert ((now - was).abs() <= 2.0 ** -20 * was.abs()).all()
    q = y["q"].double()
    want = torch.matmul(q, C.double()) / torch.matmul(q, z.double().unsqueeze(-1))
    spread = torch.matmul(q.abs(), C.double().abs()) / torch.matmul(q, z.double().unsqueeze(-1)).abs()
    assert ((o.double() - want).abs() <= 3 * 2.0 ** -8 * spread).all()


@pytest.mark.parametrize("T,D,delay", [(1, 64, 0), (2, 128, 0), (5, 64, 0), (17, 128, 1), (42, 64, 0), (300, 64, 7),
                                       (512, 128, 0)])
def test_queries_that_see_few_tokens(T, D, delay):
    """A normalised read-out of one token is v itself, bit for bit, and has no gradient but v's. With few tokens do . (v - o)
    is a small difference; dq and dk still have the error of independent roundings of their own terms: o rounded
    (its part in do . o taken out by x . dx = 0, to a rounding of each term), the weights of a row, the result: 3 of at most
    2^-8 / sqrt(3) in the 2-norm."""
    rng = np.random.default_rng(40 + T)
    B, H = 3, 4
    x, ref = on_gpu(inputs(rng, B, H, T, D))
    a = [x[n] for n in ARGS]
    o, lse = kv.kvpop_mlstm_fwd(*a, delay=delay)
    grads = kv.kvpop_mlstm_bwd(x["do"], *a, o, lse, delay=delay)
    if delay == 0:
        assert torch.equal(o[:, :, 0], x["v"][:, :, 0])
    want = [np.zeros((B, H, T, D)), np.zeros((B, H, T, D))]
    for b in range(B):
        for h in range(H):
            y = [ref[n][b, h] for n in ARGS]
            exact, lse64, *_ = om.read(*y, 1.0, delay, True)
            g = om.grads(ref["do"][b, h], *y, exact, lse64, 1.0, delay, True)[0]
            want[0][b, h], want[1][b, h] = g[0], g[1]
    for name, got, w, unit in (("dq", grads[0], want[0], ref["do"]), ("dk", grads[1], want[1], ref["do"])):
        err = np.linalg.norm(got.double().cpu().numpy() - w)
        if T == 1:  # nothing but what fp32 leaves of do . v - do . o
            assert err <= 2.0 ** -20 * np.linalg.norm(unit) * np.linalg.norm(ref["v"]), name
        else:
            assert err <= 3 * 2.0 ** -8 / 3 ** 0.5 * np.linalg.norm(w), name
