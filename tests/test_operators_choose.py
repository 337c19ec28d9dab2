"""The operators' rules on sizes: what a launch reads of its tables, which cut the sizes of the GPU tests reach."""
import pytest

from tests import native_operators as rules


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("apart", [False, True])
def test_rotary_units_read_angles_of_their_table(dtype, layout, apart):
    """A unit reads the angles of `unit_pairs` pairs from its first one on, also where fewer are its own: within its row of cosines, and for the last row's sines
    within the table."""
    for rot in range(2, 514, 2):
        for width, rows, heads in ((rot, 1, 1), (rot + 5, 70000, 4)):
            c = rules.rotary(dtype, layout, rot, width, rows, [heads], [apart])
            pairs = rot // 2
            last = (c.groups[0].pair_units - 1) * c.unit_pairs
            if apart and pairs >= c.unit_pairs:
                last = min(last, pairs - c.unit_pairs)     # (the last unit starts earlier)
            assert last < pairs and last + c.unit_pairs <= c.pitch, (rot, width)
            assert c.table >= 2 * c.groups[0].rows * c.pitch, (rot, width)


def test_rotary_groups_share_a_table_as_large_as_the_largest_needs():
    c = rules.rotary("bf16", "half", 64, 64, 20000, [32, 8, 1], [True, False, True])
    assert c.table == 2 * max(g.rows for g in c.groups) * c.pitch and len({g.rows for g in c.groups}) > 1
    assert c.blocks == sum(g.head_blocks * g.row_blocks for g in c.groups)
