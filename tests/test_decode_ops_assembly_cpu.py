"""What the source of the decoding step's operators relies on, checked in the assembly this compiler makes of it: MFMAs and
transposing reads that are written as inline assembly, which the compiler's hazard recogniser and its counting of waits do
not look into, and kernels whose loads run ahead and that must not spill."""
import os
import re
import subprocess

import pytest

from paper_2406_09425_amd import build

from test_block_ops_edges_cpu import settled_operands
from test_ksplit_assembly_cpu import registers
from test_wtile_assembly_cpu import check

KERNEL = re.compile(r"^(_ZN5sgprs\d+(\w+)):.*?^\.Lfunc_end", re.S | re.M)


def kernels(tmp_path, source):
    out = str(tmp_path / source) + ".s"
    subprocess.run([build.hipcc()] + build.COMMON + build.DEVICE + ["--cuda-device-only", "-S", os.path.join(build.CSRC, source), "-o", out], check=True, capture_output=True)
    with open(out) as f:
        return {m.group(1): m.group(0) for m in KERNEL.finditer(f.read())}


def reads(text):
    """Numbers of transposing reads in the blocks of inline assembly; a block waits for its reads, and none of them writes a
    register that a later one takes its address from."""
    counts = []
    for block in re.findall(r"^\s*;;#ASMSTART(.*?)^\s*;;#ASMEND", text, re.S | re.M):
        code = [t.strip() for t in block.split("\n") if t.strip()]
        if not any(t.startswith("ds_read") for t in code):
            continue
        assert re.fullmatch(r"s_waitcnt lgkmcnt\(0\)", code[-1]) and all(t.startswith("ds_read_b64_tr_b16") for t in code[:-1]), block
        written = set()
        for t in code[:-1]:
            to, address = (registers(part) for part in t.partition(" ")[2].split(" offset")[0].split(","))
            assert not address & written, block
            written |= to
        counts.append(len(code) - 1)
    return counts


def test_products_of_integers(tmp_path):
    found = kernels(tmp_path, "linear_i8.hip")
    tiles = 0
    for name, text in found.items():
        assert "scratch_" not in text, name
        if "linear_i8_tile_kernel" not in name:
            continue
        text, tiles = text.replace("v_mfma_i32_16x16x64_i8", "v_mfma_f32_16x16x32_bf16"), tiles + 1
        b = int(re.search(r"ELi(\d+)ELi\1E", name)[1])
        assert settled_operands(text) == check(text) == 2 * (b // 32) ** 2, name  # two halves of a k-tile, 2 x 2 wavefronts
    assert tiles == 5 * 4 * 2  # sizes and depths, activations, types


def test_paged_attention(tmp_path):
    found = kernels(tmp_path, "paged.hip")
    assert sum("paged_attention_kernel" in name for name in found) == 4 + 3 * 4  # bf16, fp32 by heads of a key head
    for name, text in found.items():
        assert "scratch_" not in text, name
        counts = reads(text)
        assert bool(counts) == ("paged_attention_kernelILi1E" in name), name


def test_norm(tmp_path):
    for name, text in kernels(tmp_path, "rms_norm.hip").items():
        assert "scratch_" not in text, name


def test_the_check_of_reads_sees_what_it_looks_for():
    read, wait = "ds_read_b64_tr_b16 v[0:1], v%d offset:16", "s_waitcnt lgkmcnt(0)"
    block = lambda *lines: "\n".join((";;#ASMSTART",) + lines + (";;#ASMEND",))  # noqa: E731
    assert reads(block(read % 2, read % 3, wait)) == [2] and reads(block("s_nop 15")) == []
    for bad in (block(read % 2), block(wait, read % 2), block(read % 2, read % 1, wait), block(read % 2, "s_waitcnt lgkmcnt(1)")):
        with pytest.raises(AssertionError):
            reads(bad)
