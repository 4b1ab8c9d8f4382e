"""The mLSTM recurrence's entry points: what the header declares is exported, bad arguments are rejected with
the documented status before anything is launched (no GPU; the device addresses are fake), and the binding packs what the
library reads."""
import ctypes
import math
import os
import re

import pytest

import paper_2607_05061_amd as kv

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "kvpop_mlstm.h")
pytestmark = pytest.mark.skipif(not os.path.exists(kv.lib_path()),
                                reason="libkvpop.so not built (python -m paper_2607_05061_amd.build)")
EINVAL, EUNS = kv.KVPOP_EINVAL, kv.KVPOP_EUNSUPPORTED
GB = 1 << 30


def rows(ptr, sb=8 * 300 * 128, sh=300 * 128, st=128):
    return kv.KvpopRowsC(ptr, sb, sh, st)


def gate(ptr, sb=2400, sh=300, st=1):
    return kv.KvpopRowsC(ptr, sb, sh, st)


def call(B=2, H=8, T=300, D=128, delay=0, norm=1, scale=1.0, q=None, k=None, v=None, ig=None, fg=None, lens=None):
    return kv.KvpopMlstmC(B, H, T, D, delay, norm, scale, q or rows(1 * GB), k or rows(2 * GB), v or rows(3 * GB),
                          ig or gate(4 * GB), fg or gate(5 * GB), lens)


def state(C=6 * GB, z=7 * GB, m=8 * GB):
    return kv.KvpopMlstmStateC(C, z, m)


def fwd(a=None, s=None, o=9 * GB, lse=10 * GB, ws=11 * GB, size=None):
    a = a or call()
    size = kv.lib().kvpop_mlstm_fwd_workspace_size(ctypes.byref(a)) if size is None else size
    return kv.lib().kvpop_mlstm_fwd(ctypes.byref(a), ctypes.byref(s) if s else None, o, lse, ws, size, None)


def bwd(a=None, do=None, o=9 * GB, lse=10 * GB, ws=11 * GB, size=None, **g):
    a = a or call()
    size = kv.lib().kvpop_mlstm_bwd_workspace_size(ctypes.byref(a)) if size is None else size
    grads = kv.KvpopMlstmGradsC(*(g.get(n, (20 + i) * GB) for i, n in enumerate(("dq", "dk", "dv", "dig", "dfg"))))
    do = rows(12 * GB) if do is None else do
    return kv.lib().kvpop_mlstm_bwd(ctypes.byref(a), ctypes.byref(do), o, lse, ctypes.byref(grads), ws, size, None)


def step(a=None, s=None, o=9 * GB):
    return kv.lib().kvpop_mlstm_step(ctypes.byref(a or call(T=1)), ctypes.byref(s or state()), o, None)


def test_declared_functions_are_exported():
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"^\s*(?:int|size_t)\s+(kvpop_\w+)\s*\(", src, flags=re.M))
    assert names == {"kvpop_mlstm_fwd", "kvpop_mlstm_fwd_workspace_size", "kvpop_mlstm_bwd", "kvpop_mlstm_bwd_workspace_size",
                     "kvpop_mlstm_step"}
    for n in names:
        assert ctypes.cast(getattr(kv.lib(), n), ctypes.c_void_p).value
        assert n in kv.__all__


@pytest.mark.parametrize("f,T", [(fwd, 300), (bwd, 300), (step, 1)])
def test_call_checks(f, T):
    for kw in (dict(B=0), dict(H=0), dict(D=0), dict(T=0), dict(delay=-1), dict(norm=2), dict(norm=-1), dict(scale=0.0),
               dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan), dict(q=rows(None)), dict(k=rows(None)),
               dict(v=rows(None)), dict(ig=gate(None)), dict(fg=gate(None)), dict(q=rows(GB, st=-8)), dict(k=rows(GB, sb=-8)),
               dict(ig=gate(4 * GB, st=-1)), dict(fg=gate(5 * GB, sb=1 << 62))):
        assert f(call(**{"T": T, **kw})) == EINVAL, kw
    for kw in (dict(D=96), dict(T=(1 << 24) + 1), dict(q=rows(GB + 8)), dict(k=rows(2 * GB, st=132)), dict(v=rows(3 * GB, sh=4)),
               dict(ig=gate(4 * GB + 1)), dict(fg=gate(5 * GB + 1)), dict(lens=13 * GB + 2), dict(B=1 << 15, H=1 << 15),
               dict(B=1 << 20, H=64)):
        assert f(call(**{"T": T, **kw})) == EUNS, kw


def test_fwd_checks():
    assert kv.lib().kvpop_mlstm_fwd(None, None, None, None, None, 0, None) == EINVAL
    for kw in (dict(o=None), dict(o=1 * GB), dict(o=3 * GB + 64), dict(lse=9 * GB + 64), dict(lse=4 * GB), dict(ws=None),
               dict(size=0), dict(ws=9 * GB), dict(ws=2 * GB), dict(s=state(C=None)), dict(s=state(z=None)), dict(s=state(m=None)),
               dict(s=state(C=2 * GB)), dict(s=state(z=6 * GB + 64)), dict(s=state(m=9 * GB))):
        assert fwd(**kw) == EINVAL, kw
    for kw in (dict(o=9 * GB + 8), dict(lse=10 * GB + 2), dict(ws=11 * GB + 8), dict(s=state(C=6 * GB + 8)),
               dict(s=state(z=7 * GB + 4)), dict(s=state(m=8 * GB + 2))):
        assert fwd(**kw) == EUNS, kw
    need = kv.kvpop_mlstm_fwd_workspace_size(2, 8, 300, 128)
    assert need > 0 and fwd(size=need - 1) == EINVAL
    assert kv.kvpop_mlstm_fwd_workspace_size(2, 8, 64, 128) == 0 == kv.kvpop_mlstm_fwd_workspace_size(2, 8, 300, 96)
    assert kv.lib().kvpop_mlstm_fwd_workspace_size(None) == kv.lib().kvpop_mlstm_bwd_workspace_size(None) == 0
    assert kv.kvpop_mlstm_bwd_workspace_size(2, 8, 300, 128) > 2 * need


def test_bwd_checks():
    assert kv.lib().kvpop_mlstm_bwd(ctypes.byref(call()), None, None, None, None, None, 0, None) == EINVAL
    for kw in (dict(o=None), dict(lse=None), dict(do=rows(None)), dict(do=rows(12 * GB, st=-8)), dict(ws=None), dict(size=64),
               dict(dq=None), dict(dk=None), dict(dv=None), dict(dig=None), dict(dfg=None), dict(dq=12 * GB), dict(dk=20 * GB),
               dict(dv=9 * GB), dict(dig=23 * GB + 2, dfg=23 * GB), dict(ws=22 * GB), dict(ws=10 * GB)):
        assert bwd(**kw) == EINVAL, kw
    for kw in (dict(o=9 * GB + 8), dict(lse=10 * GB + 1), dict(do=rows(12 * GB + 8)), dict(dq=20 * GB + 8), dict(dv=22 * GB + 2),
               dict(dig=23 * GB + 1), dict(dfg=24 * GB + 1), dict(ws=11 * GB + 4)):
        assert bwd(**kw) == EUNS, kw


def test_step_checks():
    one = lambda **kw: call(T=1, **kw)  # noqa: E731
    assert step(call(T=2)) == EINVAL and step(one(delay=1)) == EINVAL
    assert kv.lib().kvpop_mlstm_step(ctypes.byref(one()), None, 9 * GB, None) == EINVAL
    for kw in (dict(o=None), dict(o=6 * GB), dict(s=state(C=None)), dict(s=state(z=None)), dict(s=state(m=None)),
               dict(s=state(z=1 * GB))):
        assert step(**kw) == EINVAL, kw
    for kw in (dict(o=9 * GB + 8), dict(s=state(C=6 * GB + 4)), dict(s=state(m=8 * GB + 1))):
        assert step(**kw) == EUNS, kw


def test_forced_hip_error(monkeypatch):
    monkeypatch.setenv("KVPOP_TEST_FORCE_EHIP", "719")
    for f in (fwd, bwd, step):
        assert f() == kv.KVPOP_EHIP
    assert fwd(call(T=0)) == EINVAL


def test_packed_structures_are_the_mirrors():
    for pack, mirror in ((kv._MLSTM_PACK, kv.KvpopMlstmC), (kv._THREE_PACK, kv.KvpopMlstmStateC), (kv._FIVE_PACK, kv.KvpopMlstmGradsC)):
        assert pack.size == ctypes.sizeof(mirror), mirror
        n = len(pack.unpack(bytes(pack.size)))
        x = mirror.from_buffer_copy(pack.pack(*range(1, n + 1)))
        flat = []
        for name, t in mirror._fields_:
            v = getattr(x, name)
            flat += [getattr(v, f) for f, _ in t._fields_] if t is kv.KvpopRowsC else [v]
        assert flat == list(range(1, n + 1)), mirror


def test_binding_refuses_what_the_library_cannot_see():
    torch = pytest.importorskip("torch")
    st = kv.kvpop_mlstm_empty(1, 2, 64, device="cpu")
    assert st.C.shape == (1, 2, 64, 64) and st.z.shape == (1, 2, 64) and torch.isneginf(st.m).all()
    for bad in (dict(batch=0), dict(n_heads=0), dict(head_dim=96)):
        with pytest.raises(ValueError):
            kv.kvpop_mlstm_empty(**{**dict(batch=1, n_heads=1, head_dim=64, device="cpu"), **bad})
    x, g = torch.zeros(1, 2, 5, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 5, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        kv.kvpop_mlstm_fwd(x, x, x, g, g)
    with pytest.raises(ValueError, match="GPU"):
        kv.kvpop_mlstm_bwd(x, x, x, x, g, g, x, g.float())
    with pytest.raises(ValueError, match="GPU"):
        kv.kvpop_mlstm_step(x[:, :, 0], x[:, :, 0], x[:, :, 0], g[:, :, 0], g[:, :, 0], st)
    with pytest.raises(ValueError):
        kv.kvpop_mlstm_step(x, x, x, g, g, st)
