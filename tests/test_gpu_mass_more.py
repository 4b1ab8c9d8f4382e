"""Eviction by accumulated attention weight (include/kvpop_mass.h), more of its paths against the oracle: lists that fill up,
chunks whose rows see all of a workgroup's keys in each format and width, long prompts."""
import numpy as np
import pytest

from oracle import mass as om

torch = pytest.importorskip("torch")
import paper_2607_05061_amd as kv  # noqa: E402
from cache_cases import HostCache, bf16, i32  # noqa: E402
from test_gpu_mass import check_mass  # noqa: E402

pytestmark = pytest.mark.gpu


def test_many_lists_fill_up_at_once():
    """The last free slot of each, then the least mass: every workgroup sees one held."""
    B, H, s, w, k = 512, 8, 2, 3, 60
    S = s + w + k
    rng = np.random.default_rng(0)
    pos = i32(np.tile(np.arange(S), (B, H, 1)))
    m = rng.permuted(np.tile(np.arange(S, dtype=np.float32), (B, H, 1)), axis=2)
    mass = torch.from_numpy(m).cuda()
    held = i32(np.full((B, H), S - 1))
    assert (kv.kvpop_mass_step(i32([S - 1] * B), pos, mass, held, s, w, k) == S - 1).all()
    assert (held == S).all() and (pos[..., S - 1] == S - 1).all() and (mass[..., S - 1] == 0).all()
    m[..., S - 1] = 0
    can = np.where((np.arange(S) >= s) & (np.arange(S) <= S - w), m, np.inf)
    np.testing.assert_array_equal(kv.kvpop_mass_step(i32([S] * B), pos, mass, held, s, w, k).cpu().numpy(), can.argmin(-1))
    assert (held == S).all()
