"""The byte and product counts that bench.py's target workloads divide by (CPU)."""

import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import bench  # noqa: E402


def test_append_bytes():
    # one token: q in and out (2 x 32 heads), k and v in and out (4 x 8 heads), 256 bytes a head
    assert bench.append_bytes(1, 32, 8) == 256 * (64 + 32)


def test_causal_work():
    # one token over 10 keys: 2 x 8 heads of 10 keys and 2 x 32 rows; 4 x 128 products a pair
    assert bench.causal_work([1], [10], 32, 8) == (256 * (2 * 8 * 10 + 2 * 32), 4 * 128 * 32 * 10)
    # 3 new tokens over 5: 3 + 4 + 5 pairs; a sequence without new tokens is not read
    assert bench.causal_work([3, 0], [5, 900], 4, 2) == (256 * (2 * 2 * 5 + 2 * 4 * 3), 4 * 128 * 4 * 12)
