"""Host logic of the attention-block operators at the ends of what their descriptors may say."""
import paper_2406_09425_amd as S

from test_block_ops_assembly_cpu import kernels

INT_MAX = 2 ** 31 - 1


def test_group_norm_of_the_largest_number_of_positions():
    """A mean and a sum of squares for each of a million chunks of 2048 positions: no wrapped numbers of chunks."""
    need = S.sgprs_group_norm_workspace(S.GroupNormDesc(n=1, hw=INT_MAX, c=1, groups=1, dtype=S.SGPRS_BF16, eps=1e-5), 256)
    assert INT_MAX // 65536 * 8 <= need <= INT_MAX // 256 * 8


def test_lanes_of_a_join_meet_before_they_read_each_others_weights(tmp_path):
    """A wavefront per row: nothing but the fences holds its LDS writes and reads in their order."""
    found = {n: t for n, t in kernels(tmp_path, "attention.hip", "attention_join_kernel").items() if "ELi4E" in n}
    assert len(found) == 2                                     # two types
    for name, text in found.items():
        assert text.count("wave barrier") == 2, name
