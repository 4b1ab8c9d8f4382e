"""Normalised read-outs of signed features: x . z cancels, and o is the quotient of what it and the normaliser are, not
of rounded weights' sums."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2607_05061_amd as kv  # noqa: E402
from mlstm_cases import check_grads, check_read, inputs, norm_error, on_gpu  # noqa: E402
from oracle import mlstm as om  # noqa: E402

pytestmark = pytest.mark.gpu

ARGS = ("q", "k", "v", "ig", "fg")


@pytest.mark.parametrize("T,D,delay", [(3, 64, 0), (64, 64, 0), (300, 64, 3), (300, 128, 0), (700, 64, 20)])
@pytest.mark.parametrize("state", [False, True])
def test_read_outs(T, D, delay, state):
    rng = np.random.default_rng(60 + T)
    x, ref = on_gpu(inputs(rng, 2, 2, T, D, signed=True))
    a = [x[n] for n in ARGS]
    st, before = None, None
    if state:
        st = [rng.standard_normal((2, 2, D, D)) * 0.2, rng.standard_normal((2, 2, D)) * 0.1, rng.standard_normal((2, 2))]
        st = kv.KvpopMlstmState(*(torch.as_tensor(y, dtype=torch.float32).cuda() for y in st))
        before = [y.double().cpu().numpy() for y in st]
    o, lse = kv.kvpop_mlstm_fwd(*a, 0.3, delay, True, state=st)
    check_read(ref, None, 0.3, delay, True, o, lse, before, st)


@pytest.mark.parametrize("D", [64, 128])
def test_keys_that_oppose_what_is_held(D):
    """Positive weights beside a held part of the other sign: their sum cancels as well. Per row the numerator's terms and o
    are rounded once each, and nothing else by more than 2^-14 of the terms."""
    rng = np.random.default_rng(61)
    B, H, T = 2, 2, 40
    x = inputs(rng, B, H, T, D, ig=(0.0, 0.1))
    g, ref = on_gpu(x)
    C = rng.standard_normal((B, H, D, D)) * 0.2
    z = -0.9 * ref["k"].mean(2) * 8 * rng.random((B, H, 1))
    st = kv.KvpopMlstmState(*(torch.as_tensor(y, dtype=torch.float32).cuda() for y in (C, z, np.zeros((B, H)))))
    before = [y.double().cpu().numpy() for y in st]
    o, lse = kv.kvpop_mlstm_fwd(*(g[n] for n in ARGS), state=st)
    check_read(ref, None, 1.0, 0, True, o, lse, before, st)


def test_the_divisor_is_the_sum_and_not_the_sum_of_rounded_weights():
    """Over all rows whose normaliser is at least 2^-10 of its terms' absolute sum, the 2-norm error of o is that of independent
    roundings: of the terms, each at most 2^-8 / sqrt(3) of itself in the mean square, and of o. The terms' root of the sum of
    squares, over x's and k's elements together, stands in for them."""
    rng = np.random.default_rng(62)
    T = D = 64
    for _ in range(8):
        x, ref = on_gpu(inputs(rng, 2, 4, T, D, signed=True))
        o, lse = kv.kvpop_mlstm_fwd(*(x[n] for n in ARGS))
        for b in range(2):
            for h in range(4):
                q, k, v, ig, fg = (ref[n][b, h] for n in ARGS)
                ro, rl, W, _, dens = om.read(q, k, v, ig, fg, 1.0, 0, True)
                use = ~np.isneginf(rl) & (dens < 1024)
                # per row: sqrt(sum over tokens and columns (w s v)^2), W is already divided by the normaliser
                rss = np.sqrt((((W * (q @ k.T)) ** 2) @ (v ** 2)))
                bound = 2.0 ** -8 / 3 ** 0.5 * (np.linalg.norm(rss[use]) + np.linalg.norm(ro[use]))
                got = o[b, h].double().cpu().numpy()[use]
                assert np.linalg.norm(got - ro[use]) <= bound, (norm_error(got, ro[use]), bound / np.linalg.norm(ro[use]))


@pytest.mark.parametrize("T,D,delay", [(3, 64, 0), (64, 64, 0), (64, 128, 1), (300, 64, 3), (300, 128, 0), (512, 64, 0), (700, 64, 20)])
def test_gradients(T, D, delay):
    x, ref = on_gpu(inputs(np.random.default_rng(60 + T), 2, 2, T, D, signed=True))
    a = [x[n] for n in ARGS]
    o, lse = kv.kvpop_mlstm_fwd(*a, 0.3, delay, True)
    check_grads(ref, None, 0.3, delay, True, o, lse, kv.kvpop_mlstm_bwd(x["do"], *a, o, lse, 0.3, delay, True))


@pytest.mark.parametrize("where", ["first key", "a late key", "a masked key", "a query", "all queries"])
def test_gradients_of_features_that_are_mostly_positive(where):
    """Negative elements here and there, large enough that some rows cancel."""
    rng = np.random.default_rng(63)
    x = inputs(rng, 2, 2, 400, 64)
    if where == "all queries":
        x["q"][..., ::2] *= -0.7
    elif where == "a query":
        x["q"][:, :, 200, :40] *= -0.7
    else:
        t = {"first key": 0, "a late key": 301, "a masked key": 7}[where]
        x["k"][:, :, t] *= -6.0
        if where == "a masked key":
            x["ig"][:, :, t] = -np.inf
    g, ref = on_gpu(x)
    a = [g[n] for n in ARGS]
    o, lse = kv.kvpop_mlstm_fwd(*a)
    check_read(ref, None, 1.0, 0, True, o, lse)
    grads = kv.kvpop_mlstm_bwd(g["do"], *a, o, lse)
    check_grads(ref, None, 1.0, 0, True, o, lse, grads)
    if where == "a masked key":  # what it holds does not matter
        a[1][:, :, 7] = float("nan")
        for p, r in zip(grads, kv.kvpop_mlstm_bwd(g["do"], *a, o, lse)):
            assert torch.equal(p, r)
