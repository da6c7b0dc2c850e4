"""Index arithmetic of the attention at the ends of its range, without a device."""
import pytest


@pytest.mark.parametrize("group", [1, 2, 3, 77, 128])
def test_rows_that_see_a_key_far_away(group):
    """Tokens times heads of a group pass 32 bits in long sequences: a key far before a tile's queries is seen by all of them."""
    from paper_2108_03645_b200 import train
    first_row = train.lib().ones_attention_first_row
    far = [-(1 << 30) + 1, -(1 << 31) // group - 40, -(1 << 24) - 3, -(1 << 20)]
    for behind in [*(b for b in far if b > -(1 << 30)), *range(-300, 260)]:
        for lane in (0, 1, 31):  # keys of a warp, one behind the other
            got, exact = first_row(behind, group) + lane * group, (behind + lane) * group
            for row in (0, 1, 31, 32, 63, 64, 96, 127):
                assert (row >= got) == (row >= exact), (behind, lane, row)
