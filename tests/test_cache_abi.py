"""The compact cache's entry points: what the header declares is exported, and bad arguments
are rejected with the documented status before anything is launched (no GPU needed; the
device addresses are fake)."""
import ctypes
import math
import os
import re

import pytest

import paper_2607_05061_amd as kv

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "kvpop_cache.h")
pytestmark = pytest.mark.skipif(not os.path.exists(kv.lib_path()),
                                reason="libkvpop.so not built (python -m paper_2607_05061_amd.build)")
EINVAL, EUNS = kv.KVPOP_EINVAL, kv.KVPOP_EUNSUPPORTED
GB = 1 << 30


def test_declared_functions_are_exported():
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"^\s*(?:int|size_t)\s+(kvpop_\w+)\s*\(", src, flags=re.M))
    assert names == {"kvpop_cache_append", "kvpop_cache_attn", "kvpop_cache_attn_workspace_size",
                     "kvpop_retain_prompt", "kvpop_retain_step"}
    for n in names:
        assert ctypes.cast(getattr(kv.lib(), n), ctypes.c_void_p).value
        assert n in kv.__all__


def cache(B=2, H=2, D=128, fmt=0, P=64, n=40, per=4, k=1 * GB, v=2 * GB, ke=3 * GB, ve=4 * GB, table=5 * GB):
    return kv.KvpopCacheC(B, H, D, fmt, P, n, per, k, v, ke, ve, table)


def rows(ptr, sb=10240, sh=1280, st=128):
    return kv.KvpopRowsC(ptr, sb, sh, st)


def append(c=None, N=10, M=None, **kw):
    a = kv.KvpopAppendC(N, N if M is None else M, rows(6 * GB), rows(7 * GB))
    a.held = 8 * GB
    for n, x in kw.items():
        setattr(a, n, x)
    return kv.lib().kvpop_cache_append(ctypes.byref(c or cache()), ctypes.byref(a), None)


def attn(c=None, Hq=4, N=3, scale=0.1, q=None, held=8 * GB, lens=None, o=9 * GB, lse=10 * GB, ws=11 * GB, size=None):
    c = c or cache()
    size = kv.lib().kvpop_cache_attn_workspace_size(ctypes.byref(c), Hq, N) if size is None else size
    q = rows(6 * GB) if q is None else q
    return kv.lib().kvpop_cache_attn(ctypes.byref(c), Hq, N, scale, ctypes.byref(q), held, lens, o, lse, ws, size, None)


def retained(B=2, H=2, S=20, pos=1 * GB, prio=2 * GB, held=3 * GB):
    return kv.KvpopRetainC(B, H, S, pos, prio, held)


def prompt(s=None, T=50, evict=4 * GB, scores=5 * GB, lg=None, lens=None):
    return kv.lib().kvpop_retain_prompt(ctypes.byref(s or retained()), T, evict, scores, lg, lens, None)


def step(s=None, scores=4 * GB, lg=None, q=5 * GB, sinks=2, w=3, k=15, slot=6 * GB):
    return kv.lib().kvpop_retain_step(ctypes.byref(s or retained()), scores, lg, q, sinks, w, k, slot, None)


@pytest.mark.parametrize("call", [append, attn])
def test_cache_checks(call):
    for kw in (dict(B=0), dict(H=0), dict(D=0), dict(P=0), dict(n=0), dict(per=0), dict(B=-1), dict(k=None), dict(v=None),
               dict(ke=None), dict(ve=None), dict(table=None)):
        assert call(cache(**kw)) == EINVAL, kw
    for kw in (dict(D=96), dict(P=8), dict(P=48), dict(P=256), dict(fmt=2), dict(fmt=-1), dict(per=(1 << 24) // 64 + 1),
               dict(k=GB + 8), dict(v=2 * GB + 4), dict(table=5 * GB + 2)):
        assert call(cache(**kw)) == EUNS, kw
    if call is append:
        assert call(cache(v=1 * GB + 64 * 128 * 16)) == EINVAL        # values over keys
        assert call(cache(ke=2 * GB + 16)) == EINVAL                  # exponents over values
        assert call(cache(table=3 * GB + 4)) == EINVAL                # the table over exponents


def test_append_checks():
    assert kv.lib().kvpop_cache_append(None, None, None) == EINVAL
    assert kv.lib().kvpop_cache_append(ctypes.byref(cache()), None, None) == EINVAL
    for kw in (dict(N=0), dict(M=0, src=12 * GB), dict(M=9), dict(held=None), dict(k=rows(None)), dict(v=rows(None)),
               dict(k=rows(6 * GB, st=-8)), dict(v=rows(7 * GB, sb=-8)), dict(k=rows(6 * GB, st=1 << 62)), dict(rot_dim=-16),
               dict(rot_dim=144), dict(rot_dim=64), dict(rot_dim=64, cos=12 * GB, n_positions=5),
               dict(rot_dim=64, cos=12 * GB, sin=13 * GB), dict(adjacent=2), dict(n_q_heads=-1),
               dict(q=rows(12 * GB), q_out=13 * GB), dict(q=rows(12 * GB), n_q_heads=4),
               dict(q=rows(12 * GB), n_q_heads=4, q_out=12 * GB + 64),  # the rotated queries over the queries
               dict(q=rows(12 * GB), n_q_heads=4, q_out=1 * GB),        # over the keys' pages
               dict(k=rows(1 * GB + 4096)),                             # new keys inside the pages
               dict(v=rows(2 * GB - 64)),                               # pages that begin inside the new values
               dict(held=3 * GB)):                                      # the lengths over exponents
        assert append(**kw) == EINVAL, kw
    table = dict(cos=12 * GB, sin=13 * GB, n_positions=5)
    for kw in (dict(k=rows(6 * GB + 8)), dict(v=rows(7 * GB, st=132)), dict(v=rows(7 * GB, sh=4)), dict(rot_dim=24, **table),
               dict(held=8 * GB + 2), dict(count=12 * GB + 1), dict(start=12 * GB + 2), dict(pos0=12 * GB + 3),
               dict(src=12 * GB + 2), dict(rot_dim=64, cos=12 * GB + 4, sin=13 * GB, n_positions=5),
               dict(q=rows(12 * GB), n_q_heads=4, q_out=13 * GB + 8), dict(N=(1 << 24) + 1)):
        assert append(**kw) == EUNS, kw
    assert append(cache(B=30000, H=30000, table=100 * GB, per=1), M=1 << 20, src=30000 * GB, held=20000 * GB) == EUNS  # too many workgroups


def test_attn_checks():
    c = cache()
    for kw in (dict(Hq=0), dict(Hq=3), dict(N=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf),
               dict(scale=math.nan), dict(q=rows(None)), dict(held=None), dict(o=None), dict(lse=None),
               dict(q=rows(6 * GB, sb=-8)), dict(o=6 * GB + 64), dict(o=2 * GB), dict(lse=9 * GB + 16),
               dict(lse=8 * GB), dict(o=3 * GB), dict(lse=5 * GB)):
        assert attn(c, **kw) == EINVAL, kw
    for kw in (dict(q=rows(6 * GB + 2)), dict(q=rows(6 * GB, st=12)), dict(o=9 * GB + 8), dict(lse=10 * GB + 2),
               dict(held=8 * GB + 1), dict(lens=12 * GB + 2), dict(Hq=2 * 1025), dict(N=(1 << 24) + 1)):
        assert attn(c, **kw) == EUNS, kw
    long = cache(per=1000, n=5000)
    need = kv.lib().kvpop_cache_attn_workspace_size(ctypes.byref(long), 4, 1)
    assert need > 0
    assert attn(long, N=1, size=need - 1) == EINVAL
    assert attn(long, N=1, ws=None) == EINVAL
    assert attn(long, N=1, ws=11 * GB + 8) == EUNS
    assert attn(long, N=1, ws=9 * GB + 64) == EINVAL     # the workspace over o
    assert attn(long, N=1, ws=1 * GB) == EINVAL          # the workspace over the pages
    assert kv.lib().kvpop_cache_attn_workspace_size(ctypes.byref(cache(P=48)), 4, 1) == 0
    assert kv.lib().kvpop_cache_attn_workspace_size(None, 4, 1) == 0


def test_retain_checks():
    for call in (prompt, step):
        for kw in (dict(B=0), dict(H=0), dict(S=0), dict(pos=None), dict(prio=None), dict(held=None)):
            assert call(retained(**kw)) == EINVAL, kw
        for kw in (dict(pos=GB + 2), dict(prio=2 * GB + 1), dict(held=3 * GB + 2), dict(S=(1 << 24) + 1)):
            assert call(retained(**kw)) == EUNS, kw
        assert call(retained(prio=1 * GB + 64)) == EINVAL
        assert call(retained(held=2 * GB + 64)) == EINVAL
    for kw in (dict(T=0), dict(evict=None), dict(scores=None), dict(evict=1 * GB + 16), dict(scores=2 * GB)):
        assert prompt(**kw) == EINVAL, kw
    for kw in (dict(T=(1 << 24) + 1), dict(evict=4 * GB + 2), dict(lens=8 * GB + 1), dict(lg=8 * GB + 2)):
        assert prompt(**kw) == EUNS, kw
    for kw in (dict(scores=None), dict(q=None), dict(slot=None), dict(sinks=-1), dict(w=-1), dict(k=0), dict(k=16),
               dict(sinks=2 ** 31 - 1, w=2 ** 31 - 1, k=2 ** 31 - 1), dict(slot=4 * GB), dict(slot=3 * GB), dict(q=1 * GB)):
        assert step(**kw) == EINVAL, kw
    for kw in (dict(scores=4 * GB + 1), dict(q=5 * GB + 2), dict(slot=6 * GB + 2), dict(lg=7 * GB + 1)):
        assert step(**kw) == EUNS, kw


def test_forced_hip_error(monkeypatch):
    monkeypatch.setenv("KVPOP_TEST_FORCE_EHIP", "719")
    for call in (append, attn, prompt, step):
        assert call() == kv.KVPOP_EHIP
        assert kv.kvpop_strerror(kv.KVPOP_EHIP).startswith("HIP error: ")
    assert append(N=0) == EINVAL


def test_binding_refuses_what_the_library_cannot_see():
    torch = pytest.importorskip("torch")
    with pytest.raises((TypeError, ValueError)):
        kv.kvpop_cache_append(kv.KvpopCache(*[None] * 5), None, None, None)
    c = kv.kvpop_cache_empty(1, 2, 100, 64, 32, device="cpu")
    assert c.page_table.shape == (1, 2, 4) and c.k_pages.shape == (8, 32, 64) and c.k_pages.dtype == torch.int8
    assert kv.kvpop_cache_empty(1, 1, 1, 64, dtype=torch.float8_e4m3fn, device="cpu").v_pages.dtype == torch.float8_e4m3fn
    for bad, err in ((dict(page_size=48), ValueError), (dict(page_size=0), ValueError), (dict(head_dim=96), ValueError),
                     (dict(batch=0), ValueError), (dict(tokens=0), ValueError), (dict(n_kv_heads=-1), ValueError),
                     (dict(dtype=torch.float32), TypeError)):
        with pytest.raises(err):
            kv.kvpop_cache_empty(**{**dict(batch=1, n_kv_heads=1, tokens=5, head_dim=64, device="cpu"), **bad})
    with pytest.raises(ValueError, match="GPU"):
        kv.kvpop_cache_attn(torch.zeros(1, 2, 1, 64, dtype=torch.bfloat16), c, torch.zeros(1, 2, dtype=torch.int32), 0.1)
    with pytest.raises(ValueError, match="GPU"):
        kv.kvpop_retain_step(torch.zeros(1, 1), torch.zeros(1, dtype=torch.int32), torch.zeros(1, 1, 4, dtype=torch.int32),
                             torch.zeros(1, 1, 4), torch.zeros(1, 1, dtype=torch.int32), 1, 1, 1)
    with pytest.raises(ValueError, match="GPU"):
        kv.kvpop_retain_prompt(torch.zeros(1, 1, 4, dtype=torch.int32), torch.zeros(1, 1, 4), 4)


def test_packed_structures_are_the_mirrors():
    """The binding packs the structures' fields at once: sizes and offsets are ctypes' own."""
    for pack, mirror in ((kv._CACHE_PACK, kv.KvpopCacheC), (kv._ROWS_PACK, kv.KvpopRowsC),
                         (kv._APPEND_PACK, kv.KvpopAppendC), (kv._RETAIN_PACK, kv.KvpopRetainC)):
        assert pack.size == ctypes.sizeof(mirror), mirror
        n = len(pack.unpack(bytes(pack.size)))
        x = mirror.from_buffer_copy(pack.pack(*range(1, n + 1)))
        flat = []
        for name, t in mirror._fields_:
            v = getattr(x, name)
            flat += [getattr(v, f) for f, _ in t._fields_] if t is kv.KvpopRowsC else [v]
        assert flat == list(range(1, n + 1)), mirror
