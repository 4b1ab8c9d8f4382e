"""The forget gates' gradients of the mLSTM recurrence, which are running sums: against the sums over pairs in 64 bits, in a
norm that a wrong edge, token or reset does not pass (the first test shows that, without a GPU)."""
import numpy as np
import pytest

from oracle import mlstm as om

torch = pytest.importorskip("torch")
import paper_2607_05061_amd as kv  # noqa: E402
from cache_cases import i32  # noqa: E402
from mlstm_cases import check_forget, inputs, on_gpu, partial_sums  # noqa: E402

ARGS = ("q", "k", "v", "ig", "fg")


def head(seed, T, D, normalize, delay=0, resets=()):
    x = {n: y[0, 0] for n, y in inputs(np.random.default_rng(seed), 1, 1, T, D).items()}
    x["fg"][list(resets)] = -np.inf
    o, lse, *_ = om.read(*(x[n] for n in ARGS), D ** -0.5, delay, normalize)
    return x, o, lse


@pytest.mark.parametrize("normalize", [True, False])
@pytest.mark.parametrize("T,delay,resets", [(65, 0, ()), (300, 0, (70, 200)), (300, 100, ()), (450, 9, (64, 66, 300))])
def test_the_check_sees_what_is_wrong(T, delay, resets, normalize):
    x, o, lse = head(T, T, 64, normalize, delay, resets)
    G, *rest = partial_sums(x, o, lse, 0.125, delay, normalize)
    want = om.grads(x["do"], *(x[n] for n in ARGS), o, lse, 0.125, delay, normalize)[0][4]
    sig = np.exp(om.log_sigmoid(-x["fg"]))
    np.testing.assert_allclose(sig * G, want, atol=1e-9 * np.abs(want).max())
    rounded = torch.as_tensor(want).to(torch.bfloat16).double().numpy()
    check_forget("rounded", rounded, x["fg"], G, *rest, 64)

    def refused(got):
        with pytest.raises(AssertionError):
            check_forget("wrong", got, x["fg"], G, *rest, 64)

    refused(np.zeros(T))
    refused(np.concatenate([[0], rounded[:-1]]))
    refused(np.concatenate([rounded[1:], [0]]))
    refused(-rounded)
    if T > 128 and not any(64 <= r < 128 for r in resets):  # a segment from its edge on, without what is held there
        edge = rounded.copy()
        edge[64:128] -= sig[64:128] * G[64]
        refused(edge)
    if resets:  # a sum that goes on over a reset
        r = max(resets, key=lambda r: abs(G[r - 1]))
        refused(rounded + np.where(np.arange(T) > r, sig, 0) * G[r - 1])


def run(seed, B, H, T, D, delay=0, normalize=True, lens=None, heads=None, edit=None, tokens=False, **kw):
    x = inputs(np.random.default_rng(seed), B, H, T, D, **kw)
    if edit:
        edit(x)
    g, ref = on_gpu(x, tokens)
    a, dev, scale = [g[n] for n in ARGS], None if lens is None else i32(lens), D ** -0.5
    o, lse = kv.kvpop_mlstm_fwd(*a, scale, delay, normalize, dev)
    dfg = kv.kvpop_mlstm_bwd(g["do"], *a, o, lse, scale, delay, normalize, dev)[4].double().cpu().numpy()
    o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    for b, h in heads or [(b, h) for b in range(B) for h in range(H)]:
        n = T if lens is None else min(max(int(lens[b]), 0), T)
        y = {m: ref[m][b, h, :n] for m in ref}
        sums = partial_sums(y, o[b, h, :n], lse[b, h, :n], scale, delay, normalize)
        check_forget("b%d h%d" % (b, h), dfg[b, h, :n], y["fg"], *sums, D)
        assert (dfg[b, h, n:] == 0).all() and (dfg[b, h, :n][np.isneginf(y["fg"])] == 0).all()


both = pytest.mark.parametrize("normalize", [True, False])


@pytest.mark.gpu
@both
@pytest.mark.parametrize("T", [2, 3, 17, 63, 64, 65, 130, 300, 700])
@pytest.mark.parametrize("D", [64, 128])
def test_lengths(T, D, normalize):
    run(T + D, 2, 2, T, D, normalize=normalize)


@pytest.mark.gpu
@both
@pytest.mark.parametrize("delay,lens", [(1, [500, 499]), (64, [500, 321]), (100, [450, 130]), (300, [500, 301]), (7, [257, 65])])
def test_delays_and_ragged_ends(delay, lens, normalize):
    run(delay, 2, 2, 500, 64, delay=delay, lens=lens, normalize=normalize, tokens=True)


@pytest.mark.gpu
@both
@pytest.mark.parametrize("delay", [0, 20])
@pytest.mark.parametrize("at", [[0, 5, 64, 66, 67, 127, 130, 400], [10, 37, 300], [255, 256, 257], [192], list(range(3, 440, 9)), [449]])
def test_resets(at, delay, normalize):
    """Within waves, blocks and segments (64 tokens each here), at their ends, and everywhere."""
    def edit(x):
        x["fg"][0, :, at] = -np.inf
        x["fg"][1, :, [min(t + 13, 449) for t in at]] = -np.inf
    run(len(at), 2, 2, 450, 64, delay=delay, normalize=normalize, lens=[450, 433], edit=edit)


@pytest.mark.gpu
@both
@pytest.mark.parametrize("T,delay,fg", [(2000, 0, (4.0, 1.5)), (2000, 300, (7.0, 1.0)), (1337, 20, (1.0, 1.0))])
def test_long_segments(T, delay, fg, normalize):
    """128 heads: segments of 512 tokens (of 384 for 1337), two blocks of the forget kernel each; some heads with resets within
    them and at their edges."""
    def edit(x):
        x["fg"][0, 1, [100, 511, 512, 600, 767, 768, 1300]] = -np.inf
        x["fg"][1, 63, 1100] = -np.inf
    lens = [T, T - 250]
    run(T + delay, 2, 64, T, 64, delay=delay, normalize=normalize, lens=lens, edit=edit, fg=fg,
        heads=[(0, 0), (0, 1), (1, 62), (1, 63)])


@pytest.mark.gpu
@pytest.mark.parametrize("T", [2500, 4097])
def test_one_head_in_many_segments(T):
    run(T, 1, 1, T, 64, delay=100, fg=(9.0, 0.5))


@pytest.mark.gpu
@both
@pytest.mark.parametrize("ig,fg", [((0, 5), (0, 5)), ((20, 1), (10, 1)), ((-30, 1), (-20, 3)), ((0, 0.1), (-3, 1))])
def test_gates(ig, fg, normalize):
    run(3, 1, 3, 300, 64, ig=ig if normalize else (min(ig[0], 5), ig[1]), fg=fg, normalize=normalize)
