"""The check of tests/test_product_waits.py, closer: all 8 wait states that the compiler puts between a 16x16x32 product and a
use of its result, operands with modifiers behind them (offsets, lane swaps), another product counted as one state, and
the compact cache's attention too (no GPU)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2607_05061_amd import build

NEED = 8  # what the compiler leaves before vector and memory instructions that read or overwrite such a result
MEMORY = ("ds_", "global_", "flat_", "buffer_", "scratch_")


def _registers(token):
    """Of an operand's first word: `v[2:3] offset:16`, `-v7`, `|v7|`, `v0 quad_perm:[1,0,3,2]`."""
    word = (token.strip().split() or [""])[0].lstrip("-|").rstrip("|")
    m = re.match(r"^([va])\[(\d+):(\d+)\]$", word)
    if m:
        return {(m.group(1), i) for i in range(int(m.group(2)), int(m.group(3)) + 1)}
    m = re.match(r"^([va])(\d+)$", word)
    return {(m.group(1), int(m.group(2)))} if m else set()


def early_uses(asm):
    """(products, [(kernel, product, user, wait states between)])."""
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
                args = [x.strip() for x in rest[0].split(",")] if rest else []
                code.append((op, args, [_registers(x) for x in args]))
        for at, (op, args, regs) in enumerate(code):
            if not op.startswith("v_mfma_f32_16x16x32"):
                continue
            total += 1
            result, todo, seen = regs[0], [(at + 1, 0)], set()
            while todo:
                i, waits = todo.pop()
                if i >= len(code) or waits >= NEED or (i, waits) in seen:
                    continue
                seen.add((i, waits))
                o, b, r = code[i]
                if o == "s_nop":
                    todo.append((i + 1, waits + int(b[0]) + 1))
                elif o == "s_branch":
                    todo.append((labels[b[0]], waits + 1))
                elif o == "s_endpgm":
                    continue
                elif o.startswith("v_mfma"):  # an accumulator goes on by itself, another product's operands do not
                    if any(x & result for x in r[1:3]):
                        bad.append((f.group(1), args, (o, b), waits))
                    else:
                        todo.append((i + 1, waits + 1))
                elif o.startswith(("v_",) + MEMORY) and any(x & result for x in r):
                    bad.append((f.group(1), args, (o, b), waits))
                else:
                    if o.startswith("s_cbranch"):
                        todo.append((labels[b[0]], waits + 1))
                    todo.append((i + 1, waits + 1))
    return total, bad


@pytest.mark.parametrize("between,user,found", [
    ("\ts_nop 6\n", "v_mul_f32_e32 v12, s0, v2", 7),
    ("\ts_nop 7\n", "v_mul_f32_e32 v12, s0, v2", None),
    ("", "ds_write_b64 v9, v[2:3] offset:16", 0),
    ("", "v_mov_b32_dpp v5, v0 quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf", 0),
    ("", "v_fma_f32 v5, -v0, |v1|, v6", 0),
    ("", "global_store_dwordx2 v[20:21], v[0:1], off offset:32", 0),
    ("", "v_mul_f32_e32 v2, s0, v12", 0),
    ("\tv_mfma_f32_16x16x32_bf16 v[20:23], v[4:7], v[8:11], v[20:23]\n", "v_add_f32_e32 v12, v3, v13", 1),
    ("", "v_mfma_f32_16x16x32_bf16 v[20:23], v[0:3], v[8:11], v[20:23]", 0),
    ("", "v_mfma_f32_16x16x32_bf16 v[0:3], v[4:7], v[8:11], v[0:3]", None),
    ("\ts_cbranch_vccnz .LBB0_1\n\ts_nop 7\n.LBB0_1:\n", "v_mul_f32_e32 v12, s0, v2", 1),
])
def test_what_the_check_sees(between, user, found):
    text = "_Zk:\n\tv_mfma_f32_16x16x32_bf16 v[0:3], v[4:7], v[8:11], v[0:3]\n%s\t%s\n\ts_nop 7\n\ts_endpgm\n.Lfunc_end0:\n"
    assert [x[3] for x in early_uses(text % (between, user))[1]] == ([] if found is None else [found])


@pytest.mark.skipif(shutil.which(build.hipcc()) is None, reason="no hipcc")
@pytest.mark.parametrize("source", ["kvpop_mlstm.hip", "kvpop_mass.hip", "kvpop_cache_attn.hip"])
def test_products_are_used_after_their_waits(source, tmp_path):
    out = str(tmp_path / "k.s")
    subprocess.run([build.hipcc(), *build.HIP_FLAGS, "--cuda-device-only", "-S", "-I", build.INCLUDE, "-I", build.CSRC,
                    os.path.join(build.CSRC, source), "-o", out], check=True, capture_output=True, timeout=300)
    total, bad = early_uses(open(out).read())
    assert total > 50 and not bad, bad[:3]
