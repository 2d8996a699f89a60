"""The linear product's tile kernel and the attention kernels write MFMAs as inline assembly, which the compiler's
hazard recogniser does not look into.  What the sources rely on is checked in the assembly this compiler makes of them:
accumulators are left alone until the fence, operands were written last by loads, the result of an attention score's
first MFMA is first used by an MFMA with another one in between, and nothing in the hot kernels spills to memory, whose
reloads would wait for the loads in flight."""
import os
import re
import subprocess

import pytest

from paper_2406_09425_amd import build

from test_ksplit_assembly_cpu import instructions, registers
from test_wtile_assembly_cpu import check


def kernels(tmp_path, source, pattern):
    out = str(tmp_path / (source + ".s"))
    subprocess.run([build.hipcc()] + build.COMMON + build.DEVICE + ["--cuda-device-only", "-S", os.path.join(build.CSRC, source), "-o", out],
                   check=True, capture_output=True)
    with open(out) as f:
        return {m.group(1): m.group(0) for m in re.finditer(rf"^(_ZN5sgprs\d+(?:{pattern})\w+):.*?^\.Lfunc_end", f.read(), re.S | re.M)}


def test_linear_tiles(tmp_path):
    found = kernels(tmp_path, "linear.hip", "linear_tile_kernel|linear_staged_kernel")
    tiles = {n: t for n, t in found.items() if "linear_tile_kernel" in n}
    assert len(tiles) == 8                                     # four activations, two tiles
    for name, text in found.items():
        assert "scratch_" not in text, name
    for name, text in tiles.items():
        assert check(text) == (2 * 64 if "ELi256ELi256E" in name else 2 * 16), name


def first_scores(text):
    """Number of inline MFMAs that start a score from zero; raises where their result is used too early."""
    code, count = list(instructions(text)), 0
    for at, (inline, t) in enumerate(code):
        if not (inline and t.startswith("v_mfma_f32_32x32x16_bf16")):
            continue
        operands = t.split(" ", 1)[1].split(", ")
        assert operands[3] == "0", t
        count += 1
        mine, between = registers(operands[0]), 0
        for _, later in code[at + 1:]:
            name, _, rest = later.partition(" ")
            if registers(rest) & mine:
                assert name.startswith("v_mfma") and between >= 1, (t, later)
                break
            between += name.startswith("v_mfma")
    return count


def test_attention_scores(tmp_path):
    found = kernels(tmp_path, "attention.hip", "attention_prompt_kernel")
    assert len(found) == 8                                     # two types, four widths of a head
    for name, text in found.items():
        assert "scratch_" not in text, name
        assert first_scores(text) == (2 if "ILi1E" in name else 0), name


def test_the_checks_see_what_they_look_for():
    asm = ";;#ASMSTART\nv_mfma_f32_32x32x16_bf16 v[0:15], v[32:35], v[36:39], 0\n;;#ASMEND"
    other = ";;#ASMSTART\nv_mfma_f32_32x32x16_bf16 v[16:31], v[32:35], v[36:39], 0\n;;#ASMEND"
    more = "v_mfma_f32_32x32x16_bf16 v[0:15], v[32:35], v[36:39], v[0:15]\nv_mfma_f32_32x32x16_bf16 v[16:31], v[32:35], v[36:39], v[16:31]"
    assert first_scores("\n".join([asm, "ds_read_b128 v[32:35], v40", other, more])) == 2
    for bad in ([asm, more, other], [asm, other, "v_max_f32_e32 v50, v3, v4", more], [asm, other, "v_mov_b32_e32 v16, 0", more]):
        with pytest.raises(AssertionError):
            first_scores("\n".join(bad))
