"""A library that is not the binding's: of another version, or of an older build that has the version but fewer
entry points, is refused with a message that says what to do (no GPU)."""
import os
import shutil
import subprocess

import pytest

import paper_2607_05061_amd as kv

CC = shutil.which("cc") or shutil.which("gcc")


@pytest.mark.skipif(CC is None, reason="no C compiler")
@pytest.mark.parametrize("version,text", [(kv.ABI_VERSION - 1, "ABI version %d" % (kv.ABI_VERSION - 1)),
                                          (kv.ABI_VERSION, "rebuild it")])
def test_another_library_is_refused(tmp_path, monkeypatch, version, text):
    src, out = str(tmp_path / "old.c"), str(tmp_path / "old.so")
    with open(src, "w") as f:
        f.write("int kvpop_abi_version(void) { return %d; }\n" % version)
        f.write("int kvpop_row_lse(void) { return 0; }\n")
    subprocess.run([CC, "-shared", "-fPIC", src, "-o", out], check=True, timeout=60)
    monkeypatch.setenv("KVPOP_LIB", out)
    monkeypatch.setattr(kv, "_LIB", None)
    with pytest.raises(RuntimeError, match=text):
        kv.lib()
    assert kv._LIB is None
    monkeypatch.undo()
    if os.path.exists(kv.lib_path()):
        assert kv.kvpop_abi_version() == kv.ABI_VERSION
