"""Normalised read-outs of signed features: x . z cancels, and o is the quotient of what it and the normaliser are, not
of rounded weights' sums."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2607_05061_amd as kv  # noqa: E402
from mlstm_cases import check, check_read, inputs, norm_error, on_gpu  # noqa: E402
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


def check_exact_grads(ref, scale, delay, lse, grads):
    """Gradients of the exact read-out (o's rounding is taken out of do . o) for this lse. As in check_grads, a term is rounded once
    (u = 2^-8), the result too, and 2^-13 of the terms for the rest. Beside that what x . dx, which corrects do . o, is off by:
    2^-15 of A, the absolute sum of its terms over tokens and both products' elements (what is held keeps 16 bits when it is made
    and 16 when it is read, fp32 sums of D and 64 terms: 2^-17 each). It adds as much times a row's sum of W |k| to dq, and its
    share to dk and dig. Where features cancel, A is far larger than what it is the sum of."""
    lse = lse.double().cpu().numpy()
    grads = [y.double().cpu().numpy() for y in grads]
    B, H, T, D = ref["q"].shape
    for b in range(B):
        for h in range(H):
            q, k, v, ig, fg, do = (ref[n][b, h] for n in (*ARGS, "do"))
            o = om.read(q, k, v, ig, fg, scale, delay, True)[0]
            want, terms = om.grads(do, q, k, v, ig, fg, o, lse[b, h], scale, delay, True)
            live, k = np.isfinite(ig), om.clean(k, np.isneginf(ig))
            got = np.flatnonzero(~np.isneginf(lse[b, h, :max(0, T - delay)]))
            W = np.where(live, np.exp(om.log_weights(ig, fg)[got + delay] - lse[b, h, got][:, None]), 0.0)
            X, G = np.abs(scale * q[got]), np.abs(do[got])
            off = 2.0 ** -15 * (W * (X @ np.abs(k).T) * (G @ np.abs(om.clean(v, ~live)).T)).sum(1)
            more = [np.zeros((T, D)) for _ in range(2)]
            more[0][got] = scale * off[:, None] * (W @ np.abs(k))
            more[1] = W.T @ (off[:, None] * X)
            more += [0.0, (np.abs(k) * more[1]).sum(1)]
            for i, name in enumerate(("dq", "dk", "dv", "dig")):
                extra = more[i]
                check("%s b%d h%d" % (name, b, h), grads[i][b, h], want[i],
                      1.01 * (2.0 ** -8 * np.abs(want[i]) + (2.0 ** -8 + 2.0 ** -13) * terms[i] + extra) + 1e-30)


@pytest.mark.parametrize("T,D,delay", [(1, 64, 0), (2, 64, 0), (3, 64, 0), (64, 64, 0), (64, 128, 1), (300, 64, 3), (300, 128, 0),
                                       (512, 64, 0), (700, 64, 20)])
def test_gradients(T, D, delay):
    x, ref = on_gpu(inputs(np.random.default_rng(60 + T), 2, 2, T, D, signed=True))
    a = [x[n] for n in ARGS]
    o, lse = kv.kvpop_mlstm_fwd(*a, 0.3, delay, True)
    check_exact_grads(ref, 0.3, delay, lse, kv.kvpop_mlstm_bwd(x["do"], *a, o, lse, 0.3, delay, True))


@pytest.mark.parametrize("n", [2, 4, 8, 64, 300])
@pytest.mark.parametrize("fg", [4.0, -3.0])
def test_gradients_of_rows_that_do_not_cancel(n, fg):
    """Over the rows whose normaliser is at least 2^-4 of its terms' absolute sum (do is 0 in the others): 2-norm errors
    as with positive features, 3 independent roundings of at most 2^-8 / sqrt(3) (weights, result, what x . dx leaves)."""
    rng = np.random.default_rng(64 + n)
    x = inputs(rng, 1, 8, n, 64, signed=True, fg=(fg, 1.0))
    for h in range(8):
        y = [torch.as_tensor(x[m][0, h]).to(torch.bfloat16).double().numpy() for m in ARGS]
        _, lse, _, _, dens = om.read(*y, 1.0, 0, True)
        x["do"][0, h][np.isneginf(lse) | (dens > 16)] = 0
    g, ref = on_gpu(x)
    a = [g[m] for m in ARGS]
    o, lse = kv.kvpop_mlstm_fwd(*a)
    grads = kv.kvpop_mlstm_bwd(g["do"], *a, o, lse)
    want = []
    for h in range(8):
        y = [ref[m][0, h] for m in ARGS]
        ro, rl, *_ = om.read(*y, 1.0, 0, True)
        want.append(om.grads(ref["do"][0, h], *y, ro, rl, 1.0, 0, True)[0])
    for i, name in enumerate(("dq", "dk", "dv", "dig")):
        assert norm_error(grads[i][0], np.stack([w[i] for w in want])) <= 3 * 2.0 ** -8 / 3 ** 0.5, name


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
    check_exact_grads(ref, 1.0, 0, lse, grads)
    if where == "a masked key":  # what it holds does not matter
        a[1][:, :, 7] = float("nan")
        for p, r in zip(grads, kv.kvpop_mlstm_bwd(g["do"], *a, o, lse)):
            assert torch.equal(p, r)
