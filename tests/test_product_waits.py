"""Matrix products' results are read only after the wait states that they need (gfx950 has no interlock there). The
compiler puts them in; where such a result was first read behind a branch it once left them out, and rows of
gradients were wrong. This follows every path behind every product of the recurrence's and the masses' kernels in the
assembly that the compiler makes of them here (no GPU)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2607_05061_amd import build

NEED = 7  # wait states of the 16x16x32 products, which take 8 passes (4 cycles each hide one wait state)


def _registers(token):
    token = token.strip().lstrip("-|").rstrip("|,")
    m = re.match(r"^([va])\[(\d+):(\d+)\]$", token)
    if m:
        return {(m.group(1), i) for i in range(int(m.group(2)), int(m.group(3)) + 1)}
    m = re.match(r"^([va])(\d+)$", token)
    return {(m.group(1), int(m.group(2)))} if m else set()


def early_reads(asm):
    """(products, [(kernel, product, reader, wait states between)])."""
    total, bad = 0, []
    for f in re.finditer(r"^(_Z\w+):.*?^\.Lfunc_end\d+", asm, re.S | re.M):
        code, labels = [], {}
        for line in f.group(0).split("\n"):
            line = line.split(";")[0].rstrip()
            m = re.match(r"^(\.L\w+):", line)
            if m:
                labels[m.group(1)] = len(code)
            elif line.strip() and not line.strip().startswith(".") and not line.endswith(":"):
                op, *rest = line.strip().split(None, 1)
                code.append((op, [x.strip() for x in rest[0].split(",")] if rest else []))
        for at, (op, args) in enumerate(code):
            if not op.startswith("v_mfma"):
                continue
            total += 1
            result, todo, seen = _registers(args[0]), [(at + 1, 0)], set()
            while todo:
                i, waits = todo.pop()
                if i >= len(code) or waits >= NEED or (i, waits) in seen:
                    continue
                seen.add((i, waits))
                o, b = code[i]
                if o == "s_nop":
                    todo.append((i + 1, waits + int(b[0]) + 1))
                elif o == "s_branch":
                    todo.append((labels[b[0]], waits + 1))
                elif o.startswith("v_mfma"):  # the accumulator goes on by itself
                    if any(_registers(x) & result for x in b[1:3]):
                        bad.append((f.group(1), args, code[i], waits))
                    else:
                        todo.append((i + 1, waits + 4))
                elif o.startswith(("v_", "ds_", "global_", "flat_", "buffer_", "scratch_")) and any(_registers(x) & result for x in b):
                    bad.append((f.group(1), args, code[i], waits))
                elif o != "s_endpgm":
                    if o.startswith("s_cbranch"):
                        todo.append((labels[b[0]], waits + 1))
                    todo.append((i + 1, waits + 1))
    return total, bad


def test_the_check_sees_a_read_behind_a_branch():
    text = "_Zk:\n\tv_mfma_f32_16x16x32_bf16 v[0:3], v[4:7], v[8:11], v[0:3]\n\ts_cbranch_vccnz .LBB0_1\n\ts_nop 7\n.LBB0_1:\n%s" \
           "\tv_mul_f32_e32 v12, s0, v2\n\ts_endpgm\n.Lfunc_end0:\n"
    assert [x[3] for x in early_reads(text % "")[1]] == [1]
    assert early_reads(text % "\ts_nop 5\n") == (1, [])


@pytest.mark.skipif(shutil.which(build.hipcc()) is None, reason="no hipcc")
@pytest.mark.parametrize("source", ["kvpop_mlstm.hip", "kvpop_mass.hip"])
def test_products_are_read_after_their_waits(source, tmp_path):
    out = str(tmp_path / "k.s")
    subprocess.run([build.hipcc(), *build.HIP_FLAGS, "--cuda-device-only", "-S", "-I", build.INCLUDE, "-I", build.CSRC,
                    os.path.join(build.CSRC, source), "-o", out], check=True, capture_output=True, timeout=300)
    total, bad = early_reads(open(out).read())
    assert total > 100 and not bad, bad[:3]
