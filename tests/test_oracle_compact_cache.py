"""Pins of the compact cache's oracle (no GPU): codes against numbers worked out by hand
and torch's own casts, exponents against their definition, the append against a page's
exact content, retention against the running top-k mask of the whole sequence."""
import math

import numpy as np
import pytest

import oracle
from oracle import compact_cache as cc

torch = pytest.importorskip("torch")


def test_e4m3_values_are_torchs():
    mine = cc.code_values("e4m3")
    theirs = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(mine, theirs)


def test_codes_round_to_nearest_even():
    assert [int(c) for c in cc.code_of([0.5, 1.5, 2.5, -0.5, -1.5, 200, -200, math.nan, math.inf], "int8")] == \
        [0, 2, 2, 0, 254, 127, 129, 0, 127]
    x = torch.cat([torch.randn(20000, dtype=torch.float64) * 2.0 ** e for e in range(-11, 9, 3)])
    f = x.float()  # 24 bits: torch's cast of these is the one rounding
    want = f.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(cc.code_of(f.double().numpy(), "e4m3"), want)
    assert [int(c) for c in cc.code_of([2.0 ** -10, 3 * 2.0 ** -10, 17.0, 19.0, -1e9, math.nan, 1.0625], "e4m3")] == \
        [0, 2, 0x58, 0x5A, 0xFE, 0, 0x38]


@pytest.mark.parametrize("fmt,qmax", [("int8", 127.0), ("e4m3", 448.0)])
def test_exponent_is_the_least_that_holds(fmt, qmax):
    for e in (-32, -31, -7, 0, 5, 31, 32):
        assert cc.needed_exponent([qmax * 2.0 ** e, 0.0], fmt) == e
        assert cc.needed_exponent([np.nextafter(qmax * 2.0 ** e, math.inf)], fmt) == min(e + 1, 32)
    assert cc.needed_exponent([], fmt) == -32
    assert cc.needed_exponent([math.inf, math.nan, qmax], fmt) == 0


def test_rotation_is_that_of_complex_numbers():
    rng = np.random.default_rng(0)
    x, a = rng.standard_normal((5, 24)), rng.standard_normal((5, 8))
    for adjacent in (False, True):
        y = cc.rotate(x, np.cos(a), np.sin(a), adjacent)
        i, j = (np.arange(0, 16, 2), np.arange(1, 16, 2)) if adjacent else (np.arange(8), np.arange(8, 16))
        z = (x[:, i] + 1j * x[:, j]) * np.exp(1j * a)
        np.testing.assert_allclose(y[:, i], z.real, atol=1e-15, rtol=0)
        np.testing.assert_allclose(y[:, j], z.imag, atol=1e-15, rtol=0)
        np.testing.assert_array_equal(y[:, 16:], x[:, 16:])


def test_append_grows_a_page_and_starts_one_afresh():
    pages = np.zeros((3, 16, 2), dtype=np.uint8)
    exps = np.array([5, 5, 5], dtype=np.int8)
    table = [2, 0]
    cc.append(pages, exps, table, "int8", np.array([[100.0, -3.0]]), held=1, start=0)
    assert exps.tolist() == [5, 5, 0] and pages[2, 0].view(np.int8).tolist() == [100, -3]
    cc.append(pages, exps, table, "int8", np.full((16, 2), 254.0), held=17, start=1)  # to the next page's first slot
    assert exps.tolist() == [1, 5, 1]
    assert pages[2, 0].view(np.int8).tolist() == [50, -2]  # -1.5 to even
    assert (pages[2, 1:] == 127).all() and (pages[0, 0] == 127).all() and (pages[0, 1:] == 0).all()
    cc.append(pages, exps, table, "int8", np.array([[1.0, 1.0]]), held=17, start=16)  # alone in its page
    assert exps.tolist() == [-6, 5, 1] and (pages[0, 0] == 64).all()
    cc.append(pages, exps, table, "int8", np.array([[1.0, 1.0]]), held=17, start=3)   # among others
    assert exps.tolist() == [-6, 5, 1] and (pages[2, 3] == 0).all()                   # 0.5 to even


@pytest.mark.parametrize("s,w,k", [(2, 3, 4), (0, 1, 2), (0, 0, 3), (2, 0, 1), (5, 2, 1)])
@pytest.mark.parametrize("lg", [0.0, -0.05])
def test_retention_step_by_step_is_the_running_mask(s, w, k, lg):
    T = 60
    rng = np.random.default_rng(s + 10 * w + 100 * k)
    r = np.round(rng.standard_normal(T), 1).astype(np.float32)  # with ties
    r[7], r[20], r[33] = -0.0, 0.0, -np.inf
    rank = oracle.ranks_from_priority(oracle.static_priority_f32(r, lg))
    tau = oracle.running_cutoff_bruteforce(rank, s, w, k)
    mask = oracle.running_topk_mask_rows(rank, tau, s, w, np.arange(T))
    state = {}
    for q in range(T):
        cc.retain_step(state, q, r[q - w] if q >= w else 0.0, lg, s, w, k)
        assert sorted(x[0] for x in state.values()) == np.flatnonzero(mask[q]).tolist(), q


def test_attend_matches_a_direct_sum():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((2, 4)), rng.standard_normal((3, 4)), rng.standard_normal((3, 4))
    seen = np.array([[True, True, False], [False, False, False]])
    o, lse, p = cc.attend(q, k, v, seen, 0.5)
    e = [math.exp(0.5 * q[0] @ k[j]) for j in range(2)]
    np.testing.assert_allclose(o[0], (e[0] * v[0] + e[1] * v[1]) / sum(e), rtol=1e-14)
    assert abs(lse[0] - math.log(sum(e))) < 1e-14 and lse[1] == -math.inf and (o[1] == 0).all() and (p[1] == 0).all()
