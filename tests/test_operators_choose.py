"""The operators' rules on sizes: what a launch reads of its tables, which cut the sizes of the GPU tests reach."""
import pytest

from tests import native_operators as rules, operator_cases


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


# ---- the sizes of test_gpu_operators_long.py ----

@pytest.mark.parametrize("c", operator_cases.BLOCK, ids=lambda c: "%dx%dx%d" % (c["P"], c["rows"], c["d"]))
def test_block_norm_cases_have_several_rows_a_team(c):
    cut = rules.block(c["P"], c["rows"], c["d"], c["post"], c["pre"], c["gate"], c["dtype"], c["res"], len(operator_cases.block_params(c)))
    for slab in (cut.forward, cut.backward):
        assert slab >= 3 * cut.team_rows and c["rows"] > slab and c["rows"] % slab


def test_block_norm_cases_reach_every_kind_of_team():
    cuts = [rules.block(c["P"], c["rows"], c["d"], c["post"], c["pre"], c["gate"], c["dtype"], c["res"], 0) for c in operator_cases.BLOCK]
    assert {(t.T, t.alone) for t in cuts} == {(8, 0), (8, 1), (16, 0), (32, 0), (64, 0), (0, 0), (0, 1)}
    wide = [t.threads for t in cuts if t.T == 0 and not t.alone]
    assert min(wide) <= 512 and any(512 < n <= 768 for n in wide) and max(wide) > 768


def test_rotary_cases_have_several_rows_a_workgroup():
    several, several_units, short_heads, unlike = 0, 0, 0, 0
    for c in operator_cases.ROTARY:
        for dtype in ("fp32", "bf16"):
            for layout in ("half", "interleaved"):
                cut = rules.rotary(dtype, layout, c["rot"], c["width"], c["rows"], c["heads"], [c["apart"]] * len(c["heads"]))
                several += all(g.rows > 1 for g in cut.groups)
                several_units += any(g.rows > 2 and g.units > 1 and g.heads > 1 for g in cut.groups)
                short_heads += any(g.head_blocks > 1 and h % g.heads for g, h in zip(cut.groups, c["heads"]))
                unlike += len({g.rows for g in cut.groups}) > 1
                assert all(c["rows"] % g.rows or g.rows == 1 for g in cut.groups) or c["rows"] % cut.groups[0].rows
    assert several >= 20 and several_units >= 20 and short_heads >= 4 and unlike >= 8


def test_rotary_loop_over_blocks_of_rows():
    """The sizes of the test that goes round it."""
    c = rules.rotary("bf16", "half", 2, 2, 500_000_003, [1], [False]).groups[0]
    assert c.row_blocks == 1 << 21 and c.row_blocks * c.rows < 500_000_003 - c.rows


def test_clip_cases_reach_every_kernel():
    cuts = [rules.clip(P, sizes, operator_cases.clip_dtypes(sizes, kind)) for P, sizes, kind in operator_cases.CLIP]
    assert [c.held for c in cuts] == [8, 8, 8, 4, 0, 0, 0, 0, 0, 0]
    assert [bool(c.past_caches) for c in cuts] == [False] * 7 + [True] * 3
    assert [c.tables for c in cuts] == [1] * 6 + [3, 2, 2, 2]
