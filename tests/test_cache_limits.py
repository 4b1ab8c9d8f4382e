"""The compact cache's largest calls: one launch takes 2^32 - 1 threads, and what needs more is refused
before it is launched (no GPU: calls that pass the checks end in a forced HIP error)."""
import ctypes
import os

import pytest

import paper_2607_05061_amd as kv

pytestmark = pytest.mark.skipif(not os.path.exists(kv.lib_path()),
                                reason="libkvpop.so not built (python -m paper_2607_05061_amd.build)")
TB = 1 << 40


@pytest.fixture(autouse=True)
def _nothing_is_launched(monkeypatch):
    monkeypatch.setenv("KVPOP_TEST_FORCE_EHIP", "719")


def _cache(B, H, per=1, D=64, P=16):
    return kv.KvpopCacheC(B, H, D, kv.KVPOP_CACHE_INT8, P, 1, per, *((20 + i) * TB for i in range(5)))


def _append(B, H, N, M=None, Hq=0):
    a = kv.KvpopAppendC(N, M or N, *(kv.KvpopRowsC(i * TB, 0, 0, 0) for i in (1, 2)))
    a.held = 3 * TB
    if M:
        a.src = 4 * TB
    if Hq:
        a.q, a.n_q_heads, a.q_out = kv.KvpopRowsC(13 * TB, 0, 0, 0), Hq, 14 * TB
    return kv.lib().kvpop_cache_append(ctypes.byref(_cache(B, H)), ctypes.byref(a), None)


def _attn(B, H, Hq, N, D=64, per=1):
    q = kv.KvpopRowsC(1 * TB, 0, 0, 0)
    c = _cache(B, H, per, D)
    size = kv.lib().kvpop_cache_attn_workspace_size(ctypes.byref(c), Hq, N)
    return kv.lib().kvpop_cache_attn(ctypes.byref(c), Hq, N, 0.1, ctypes.byref(q), 3 * TB, None, 4 * TB, 14 * TB, 16 * TB,
                                     size, None)


def _retained(B, H):
    return kv.KvpopRetainC(B, H, 1, 1 * TB, 2 * TB, 3 * TB)


def _prompt(B, H, T):
    return kv.lib().kvpop_retain_prompt(ctypes.byref(_retained(B, H)), T, 4 * TB, 18 * TB, None, None, None)


def _step(B, H):
    return kv.lib().kvpop_retain_step(ctypes.byref(_retained(B, H)), 4 * TB, None, 5 * TB, 0, 0, 1, 6 * TB, None)


@pytest.mark.parametrize("call,most", [
    (lambda n: _append(n, 1, 1), 2 ** 25 - 1),              # 64 threads per list and side
    (lambda n: _append(1, n, 1, M=33), (2 ** 32 - 1) // 384),  # ... and page: 33 slots reach into 3, from any first one
    (lambda n: _append(n, 1, 1, Hq=4), 32537630),           # and 4 per token and 4 query heads: 64 (2 n + n / 16)
    (lambda n: _attn(n, 1, 1, 1), 2 ** 24 - 1),             # 256 per list and 16 rows
    (lambda n: _attn(1, n, n, 300), 2 ** 22 - 1),           # 512 per list and 256 rows
    (lambda n: _prompt(n, 1, 1), 2 ** 22 - 1),              # 1024 per list and 4096 positions
    (lambda n: _prompt(1, n, 4097), 2 ** 21 - 1),
    (lambda n: _step(n, 1), 2 ** 24 - 1),                   # 256 per list
])
def test_more_threads_than_a_launch_takes(call, most):
    assert call(most) == kv.KVPOP_EHIP  # passed every check
    assert call(most + 1) == kv.KVPOP_EUNSUPPORTED
