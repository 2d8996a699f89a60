"""Host logic of the attention-block operators at the ends of what their descriptors may say, and what their sources
rely on in the assembly this compiler makes of them."""
import pytest

import paper_2406_09425_amd as S

from test_block_ops_assembly_cpu import kernels
from test_ksplit_assembly_cpu import registers

INT_MAX = 2 ** 31 - 1


def test_group_norm_of_the_largest_number_of_positions():
    """A mean and a sum of squares for each of a million chunks of 2048 positions: no wrapped numbers of chunks."""
    need = S.sgprs_group_norm_workspace(S.GroupNormDesc(n=1, hw=INT_MAX, c=1, groups=1, dtype=S.SGPRS_BF16, eps=1e-5), 256)
    assert INT_MAX // 65536 * 8 <= need <= INT_MAX // 256 * 8


@pytest.mark.parametrize("scale,fine", [(2e38, True), (-2e38, True), (2.4e38, False), (-2.9e38, False)])
def test_attention_scales_stay_finite_in_base_2(scale, fine):
    d = S.AttentionDesc(n_seqs=1, total_q=1, total_kv=1, max_q=1, max_kv=1, heads=1, kv_heads=1, head_dim=8, dtype=S.SGPRS_F32, scale=scale)
    if fine:
        assert S.sgprs_attention_workspace(d, 256) == 0
    else:
        with pytest.raises(S.SgprsError) as e:
            S.sgprs_attention_workspace(d, 256)
        assert e.value.status == -5


def test_lanes_of_a_join_meet_before_they_read_each_others_weights(tmp_path):
    """A wavefront per row: nothing but the fences holds its LDS writes and reads in their order."""
    found = {n: t for n, t in kernels(tmp_path, "attention.hip", "attention_join_kernel").items() if "ELi4E" in n}
    assert len(found) == 2                                     # two types
    for name, text in found.items():
        assert text.count("wave barrier") == 2, name


WAIT_STATES = 2  # that the matrix cores need between a vector instruction's result and its use as an operand


def settled_operands(text):
    """Number of inline MFMAs; raises where a vector instruction wrote an operand within the wait states before one, or
    where another way into the code joins there."""
    code, count = [], 0
    inline = False
    for line in (t.strip() for t in text.split("\n")):
        if line.startswith(";;#ASM"):
            inline = line.startswith(";;#ASMSTART")
        elif line.startswith(".LBB"):
            code.append((False, "label"))
        elif line and not line.startswith((";", ".")):
            code.append((inline, line.split(";")[0].strip()))
    for at, (written, t) in enumerate(code):
        if not (written and t.startswith("v_mfma")):
            continue
        count += 1
        operands, states, back = registers(",".join(t.split(",")[1:3])), 0, at - 1
        while states < WAIT_STATES:
            assert back >= 0 and code[back][1] != "label", t
            name, _, rest = code[back][1].partition(" ")
            if name.startswith("v_") and not name.startswith("v_cmp"):
                assert not registers(rest.split(",")[0]) & operands, (code[back][1], t)
            states += int(rest) + 1 if name == "s_nop" else 1
            back -= 1
    return count


def test_operands_of_inline_mfmas_keep_their_distance(tmp_path):
    found = kernels(tmp_path, "attention.hip", "attention_prompt_kernel|attention_decode_kernel")
    for name, text in found.items():
        assert "scratch_" not in text, name
        assert settled_operands(text) == (2 if "prompt" in name and "ILi1E" in name else 0), name
    found = kernels(tmp_path, "linear.hip", "linear_tile_kernel")
    for name, text in found.items():
        assert settled_operands(text) == (2 * 64 if "ELi256ELi256E" in name else 2 * 16), name


def test_the_check_of_operands_sees_what_it_looks_for():
    mfma = ";;#ASMSTART\nv_mfma_f32_32x32x16_bf16 v[0:15], v[32:35], v[36:39], 0\n;;#ASMEND"
    far, nop, other = "v_xor_b32_e32 v36, v50, v36", "s_nop 1", "v_mov_b32_e32 v60, v61"
    assert settled_operands("\n".join([far, nop, mfma])) == 1
    assert settled_operands("\n".join([far, other, "s_add_i32 s0, s0, 1", mfma])) == 1
    assert settled_operands("\n".join(["ds_read_b128 v[32:35], v40", "s_waitcnt lgkmcnt(0)", mfma])) == 1
    for bad in ([other, far, mfma], [other, far, "s_nop 0", mfma], [far, nop, ".LBB0_1:", other, mfma], [nop, "v_pk_mov_b32 v[34:35], v[0:1], v[2:3]", mfma]):
        with pytest.raises(AssertionError):
            settled_operands("\n".join(bad))
