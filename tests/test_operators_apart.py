"""Memory that meets: the host's check against a plain one, byte by byte."""
import random

import pytest

from tests.native_apart import heads_apart, meeting


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


def _head_bytes(v):
    at, row, head, rows, heads, width = v
    return {at + i * row + j * head + b for i in range(rows) for j in range(heads) for b in range(width)}


@pytest.mark.parametrize("seed", range(6))
def test_heads_against_bytes(seed):
    """Views that are said to be apart are; those of the same strides that are apart, both wholly beside one another in rows (or heads), are said to be."""
    rng = random.Random(seed)
    said = 0
    for _ in range(1500):
        rows, w = rng.choice([1, 2, 3, 5]), rng.choice([1, 2, 4])
        head, heads = rng.randrange(w, 14), [rng.choice([1, 2, 3]) for _ in range(2)]
        if rng.random() < 0.5:
            row = (max(heads) - 1) * head + w + rng.randrange(0, 30)
        else:
            row, head = head, (rows - 1) * head + w + rng.randrange(0, 30)
        views = [(1000 + rng.randrange(60), row + (rng.random() < 0.1), head + (rng.random() < 0.1), rows, n, w) for n in heads]
        meet = bool(_head_bytes(views[0]) & _head_bytes(views[1]))
        if heads_apart(*views):
            assert not meet, views
            said += 1
        assert heads_apart(*views) == heads_apart(*views[::-1]), views
    assert 200 < said


def test_heads_interleaved_in_a_joint_projection_are_apart():
    """[rows][heads][3][64]: queries, keys and values of a head side by side; [rows][3][heads][64]; [heads][rows][3][64]; a padded row."""
    w = 128
    for rows, heads in ((1, 1), (1, 8), (4096, 1), (4096, 8)):
        for pad in (0, 2, 50):
            p = 3 * heads * w + pad
            for part in (1, 2):
                assert heads_apart((4096, p, 3 * w, rows, heads, w), (4096 + part * w, p, 3 * w, rows, heads, w))
                assert heads_apart((4096, p, w, rows, heads, w), (4096 + part * heads * w, p, w, rows, heads, w))
                q, k = (4096, 3 * w, rows * 3 * w + pad, rows, heads, w), (4096 + part * w, 3 * w, rows * 3 * w + pad, rows, heads, w)
                assert heads_apart(q, k)
            assert rows * heads == 1 or not heads_apart((4096, p, 3 * w, rows, heads, w), (4096 + w - 1, p, 3 * w, rows, heads, w))
    # fewer key heads, every second of the places
    assert heads_apart((0, 1000, 20, 50, 8, 10), (10, 1000, 40, 50, 4, 10)) and not heads_apart((0, 1000, 20, 50, 8, 10), (20, 1000, 40, 50, 4, 10))
