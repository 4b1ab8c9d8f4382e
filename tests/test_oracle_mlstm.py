"""The oracle of the mLSTM recurrence: against the recurrence token by token, by hand, and its gradients against
differences (no GPU)."""
import numpy as np
import pytest

from oracle import mlstm as om


def _inputs(T, D, seed):
    rng = np.random.default_rng(seed)
    return [rng.random((T, D)), rng.random((T, D)), rng.standard_normal((T, D)), rng.standard_normal(T), 1 + rng.standard_normal(T)]


@pytest.mark.parametrize("normalize", [True, False])
def test_read_is_the_recurrence(normalize):
    x = _inputs(30, 5, 0)
    o, C, z = om.recur(*x, 0.7, normalize)
    np.testing.assert_allclose(om.read(*x, 0.7, 0, normalize)[0], o, rtol=1e-11)
    hC, hz, m = om.held(*x[1:])
    np.testing.assert_allclose(hC * np.exp(m), C, rtol=1e-11)
    np.testing.assert_allclose(hz * np.exp(m), z, rtol=1e-11)


def test_a_state_carries_on_and_a_delay_reads_later():
    x = _inputs(30, 4, 1)
    o = om.read(*x, 1.0, 0, True)[0]
    first = om.held(*(y[:13] for y in x[1:]))
    np.testing.assert_allclose(om.read(*(y[13:] for y in x), 1.0, 0, True, first)[0], o[13:], rtol=1e-10)
    late = om.read(*x, 1.0, 3, True)
    moved = [np.concatenate([np.zeros((3, 4)), x[0][:-3]])] + x[1:]
    np.testing.assert_allclose(late[0][:27], om.read(*moved, 1.0, 0, True)[0][3:], rtol=1e-12)
    assert (late[0][27:] == 0).all() and np.isneginf(late[1][27:]).all()


def test_by_hand():
    k = np.array([[1.0, 0.0], [0.0, 2.0]])
    v = np.array([[3.0, 0.0], [0.0, 5.0]])
    o, lse, *_ = om.read(np.ones((2, 2)), k, v, np.log([1.0, 2.0]), np.array([0.0, 0.0]), 1.0, 0, False)
    np.testing.assert_allclose(o, [[3, 0], [1.5, 20]])       # f = 1/2: C = k v / 2 + 2 k v
    o, lse, *_ = om.read(np.ones((2, 2)), k, v, np.log([1.0, 2.0]), np.array([0.0, 0.0]), 1.0, 0, True)
    np.testing.assert_allclose(o, [[3, 0], [1.5 / 4.5, 20 / 4.5]])
    np.testing.assert_allclose(np.exp(lse), [1, 4.5])
    o, *_ = om.read(np.ones((2, 2)), k, v, np.log([1.0, 2.0]), np.array([0.0, -np.inf]), 1.0, 0, True)
    np.testing.assert_allclose(o[1], [0, 5])                 # forgotten


@pytest.mark.parametrize("normalize", [True, False])
@pytest.mark.parametrize("delay", [0, 2])
def test_gradients_are_differences(normalize, delay):
    T, D = 7, 3
    x = _inputs(T, D, 2)
    do = np.random.default_rng(3).standard_normal((T, D))
    f = lambda y: (om.read(*y, 0.6, delay, normalize)[0] * do).sum()  # noqa: E731
    o, lse, *_ = om.read(*x, 0.6, delay, normalize)
    got, _ = om.grads(do, *x, o, lse, 0.6, delay, normalize)
    for i, g in enumerate(got):
        flat = g.reshape(-1)
        for j in range(flat.size):
            up, down = ([y.copy() for y in x] for _ in range(2))
            up[i].reshape(-1)[j] += 1e-5
            down[i].reshape(-1)[j] -= 1e-5
            assert abs((f(up) - f(down)) / 2e-5 - flat[j]) < 1e-7 * (1 + abs(flat[j])), (i, j)
