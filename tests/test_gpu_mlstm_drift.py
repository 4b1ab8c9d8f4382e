"""A served state over thousands of tokens: what m loses by its rounding, C and z have."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2607_05061_amd as kv  # noqa: E402
from mlstm_cases import b16  # noqa: E402
from oracle import mlstm as om  # noqa: E402

pytestmark = pytest.mark.gpu


def start(rng, B, H, D, m):
    C, z = rng.standard_normal((B, H, D, D)), rng.random((B, H, D)) + 0.5
    st = kv.KvpopMlstmState(*(torch.as_tensor(x, dtype=torch.float32).cuda() for x in (C, z, np.array([m]))))
    return st, [y.double().cpu().numpy() for y in st]


def check(st, before, fall, steps):
    """Per step an element is multiplied by 2^x of an exponent near 0 (one step of fp32 below 1: 2^-24, twice for the
    function's own error) and rounded (2^-24): 2^-22 in all."""
    for h in range(2):
        shift = np.exp(float(st.m[0, h]) - before[2][0, h] + fall)
        for now, was in ((st.C, before[0]), (st.z, before[1])):
            got = now[0, h].double().cpu().numpy() * shift
            assert np.abs(got / was[0, h] - 1).max() <= steps * 2.0 ** -22


def test_slow_decays_beside_a_large_m_are_kept():
    """log f = -2.3e-6 is below half of the last place of m = 100: in 3000 tokens 6.8e-3 would be lost."""
    rng = np.random.default_rng(70)
    B, H, D, steps = 1, 2, 64, 3000
    st, before = start(rng, B, H, D, [100.0, -70.0])
    x = [b16(y)[0] for y in (rng.random((B, H, D)), rng.random((B, H, D)), rng.random((B, H, D)), np.full((B, H), -np.inf))]
    fg, f64 = b16(np.full((B, H), 13.0))
    for _ in range(steps):
        kv.kvpop_mlstm_step(*x, fg, st)
    check(st, before, -steps * float(om.log_sigmoid(f64[0, 0])), steps)


@pytest.mark.parametrize("least", [-3e38, -1e30])
def test_a_state_near_the_end_of_the_range_of_m(least):
    """m = -3e38 and a gate of -1.6e7: m stays where fp32 has it, and what is held with it; nothing becomes NaN."""
    st = kv.KvpopMlstmState(torch.ones(1, 1, 64, 64, device="cuda"), torch.ones(1, 1, 64, device="cuda"), torch.full((1, 1), least, device="cuda"))
    x = [b16(y)[0] for y in (np.ones((1, 1, 64)), np.ones((1, 1, 64)), np.ones((1, 1, 64)), np.full((1, 1), -np.inf), np.full((1, 1), -1.6e7))]
    o = kv.kvpop_mlstm_step(*x, st)
    assert (o == 1).all() and (st.C == 1).all() and (st.z == 1).all() and float(st.m) == float(np.float32(least))
