"""Forget gates of any finite size: the tokens behind a very negative one keep the weights that their own gates give
them, in the read-outs, what is held, the gradients and single tokens."""
import numpy as np
import pytest

from oracle import mlstm as om

torch = pytest.importorskip("torch")
import paper_2607_05061_amd as kv  # noqa: E402
from cache_cases import i32  # noqa: E402
from mlstm_cases import check_grads, check_read, inputs, on_gpu  # noqa: E402

pytestmark = pytest.mark.gpu

ARGS = ("q", "k", "v", "ig", "fg")
LEAST = torch.finfo(torch.bfloat16).min
SIZES = [-1e4, -1e6, -2.0 ** 24, -2e7, -1e9, -1e13, -1e16, -1e20, LEAST]
PLACES = ([3], [0, 1, 2], [63, 64], [5, 40, 64, 65, 127, 130, 200, 258, 300])


def falls(size, at):
    def edit(x):
        x["fg"][0, 0, at] = size
        x["fg"][0, 1, [y + 7 for y in at]] = size
    return edit


def data(size, at, seed, T=320, D=64):
    x = inputs(np.random.default_rng(seed), 1, 2, T, D)
    falls(size, at)(x)
    return on_gpu(x)


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("at", PLACES)
@pytest.mark.parametrize("normalize", [True, False])
def test_read_outs_and_gradients(size, at, normalize):
    g, ref = data(size, at, 50)
    a = [g[n] for n in ARGS]
    o, lse = kv.kvpop_mlstm_fwd(*a, 0.3, 5, normalize)
    check_read(ref, None, 0.3, 5, normalize, o, lse)
    grads = kv.kvpop_mlstm_bwd(g["do"], *a, o, lse, 0.3, 5, normalize)
    check_grads(ref, None, 0.3, 5, normalize, o, lse, grads)


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("D", [64, 128])
def test_what_is_held(size, D):
    rng = np.random.default_rng(51)
    st = [rng.standard_normal((1, 2, D, D)) * 0.2, rng.random((1, 2, D)) + 0.1, rng.standard_normal((1, 2))]
    st = kv.KvpopMlstmState(*(torch.as_tensor(x, dtype=torch.float32).cuda() for x in st))
    before = [y.double().cpu().numpy() for y in st]
    g, ref = data(size, [5, 40, 64, 130, 258, 310], 52, D=D)
    o, lse = kv.kvpop_mlstm_fwd(*(g[n] for n in ARGS), state=st)
    check_read(ref, None, 1.0, 0, True, o, lse, before, st)


@pytest.mark.parametrize("size", [-2e7, -1e13, LEAST])
def test_beyond_two_to_the_24_a_gate_forgets_exactly(size):
    """Where an fp32 logarithm has no bits left for another token's gate, everything before is forgotten as by -inf: bit for
    bit, with masked tokens behind the gate too."""
    def results(gate):
        x = inputs(np.random.default_rng(53), 2, 2, 330, 64)
        falls(gate, [0, 5, 40, 64, 130, 258])(x)
        x["ig"][:, :, 38:50] = -np.inf
        x["ig"][1, :, 250:320] = -np.inf
        g, _ = on_gpu(x)
        a = [g[n] for n in ARGS]
        st = kv.kvpop_mlstm_empty(2, 2, 64)
        got = kv.kvpop_mlstm_fwd(*(y[:, :, 100:] for y in a), state=st) + tuple(st)
        o, lse = kv.kvpop_mlstm_fwd(*a, delay=3)
        got += (o, lse) + kv.kvpop_mlstm_bwd(g["do"], *a, o, lse, delay=3)
        return got + (kv.kvpop_mlstm_step(*(y[:, :, 5].contiguous() for y in a), st),) + tuple(st)
    for x, y in zip(results(size), results(-np.inf)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("size", [-1e6, -1e13, LEAST])
def test_a_prompt_and_its_tokens_agree(size):
    g, ref = data(size, [5, 40, 60], 54, T=90)
    a = [g[n] for n in ARGS]
    o, _ = kv.kvpop_mlstm_fwd(*a)
    st = kv.kvpop_mlstm_empty(1, 2, 64)
    for t in range(90):
        o1 = kv.kvpop_mlstm_step(*(y[:, :, t] for y in a), st)
        # two roundings of o apart, and of its terms, which are no larger together than the largest |v|
        assert (o1.float() - o[:, :, t].float()).abs().max() <= 4 * 2.0 ** -8 * g["v"].float().abs().max()
    for h in range(2):
        want = om.held(*(ref[n][0, h] for n in ARGS[1:]))
        assert abs(float(st.m[0, h]) - want[2]) <= 2.0 ** -18 * (abs(want[2]) + 1)


def test_a_very_negative_input_gate_hides_a_token():
    """The usual finite mask in ig: its token has no weight beside any other."""
    x = inputs(np.random.default_rng(55), 1, 2, 200, 64)
    x["ig"][:, :, 20:70] = LEAST
    x["ig"][:, :, 199] = LEAST
    g, ref = on_gpu(x)
    a = [g[n] for n in ARGS]
    o, lse = kv.kvpop_mlstm_fwd(*a, lens=i32([200]))
    check_read(ref, None, 1.0, 0, True, o, lse)
    check_grads(ref, None, 1.0, 0, True, o, lse, kv.kvpop_mlstm_bwd(g["do"], *a, o, lse))
