"""Host logic of the attention-block operators at the ends of what their descriptors may say."""
import paper_2406_09425_amd as S

INT_MAX = 2 ** 31 - 1


def test_group_norm_of_the_largest_number_of_positions():
    """A mean and a sum of squares for each of a million chunks of 2048 positions: no wrapped numbers of chunks."""
    need = S.sgprs_group_norm_workspace(S.GroupNormDesc(n=1, hw=INT_MAX, c=1, groups=1, dtype=S.SGPRS_BF16, eps=1e-5), 256)
    assert INT_MAX // 65536 * 8 <= need <= INT_MAX // 256 * 8
