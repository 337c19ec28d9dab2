"""Memory that meets: the host's check against a plain one, byte by byte."""
import random

import pytest

from tests.native_apart import meeting


def _bytes(r):
    at, n, stride, count, _ = r
    return {at + k * stride + b for k in range(count) for b in range(n)}


def _meet(a, b):
    return bool((a[4] or b[4]) and _bytes(a) & _bytes(b))


@pytest.mark.parametrize("seed", range(8))
def test_meeting_regions_against_bytes(seed):
    rng = random.Random(seed)
    found = 0
    for _ in range(400):
        strides = rng.choice([[16], [24], [16, 24], [10, 16, 7]])
        regions = []
        for _ in range(rng.choice([2, 2, 3, 5, 12])):
            p = rng.choice(strides)
            regions.append((1000 + rng.randrange(160), rng.randrange(0, min(5, p) + 1), p, rng.choice([1, 2, 3, 6]), rng.random() < 0.5))
        got = meeting(regions)
        want = any(_meet(a, b) for i, a in enumerate(regions) for b in regions[:i])
        assert (got is not None) == want, regions
        if got:
            assert _meet(regions[got[0]], regions[got[1]]), regions
            found += 1
    assert 40 < found < 360      # (both answers are common)


def test_columns_of_flat_rows_are_apart():
    """A hundred columns of rows of 4096 bytes, written, the gaps between them read; one of them a byte too long is found."""
    cols = [(1 << 20) + 40 * k for k in range(100)]
    regions = [(c, 32, 4096, 64, True) for c in cols] + [(c + 32, 8, 4096, 64, False) for c in cols]
    assert meeting(regions) is None
    regions[17] = (cols[17], 33, 4096, 64, True)
    assert set(meeting(regions)) == {17, 117}
    # the last column's rows run into the next row's first column
    regions[17] = (cols[17], 32, 4096, 64, True)
    regions.append((cols[0] + 4090, 7, 4096, 64, False))
    assert set(meeting(regions)) == {0, 200}


def test_far_apart_and_large_regions():
    big = 1 << 40
    assert meeting([(0x1000, 1 << 30, big, 1024, True), (0x1000 + (1 << 30), 1 << 30, big, 1024, True)]) is None
    assert meeting([(0x1000, 1 << 30, big, 1024, True), (0x1000 + 1023 * big + (1 << 30) - 1, 1, 0, 1, False)]) == (0, 1)
    assert meeting([(0x1000, 1 << 30, big, 1024, True), (0x1000 + 1022 * big + (1 << 30), 8, 0, 1, False)]) is None
