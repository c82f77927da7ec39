"""Drafted trees over the 4-bit cache and kept rows: launch shapes beside those of the other
tests."""
import pytest

import test_gpu_q4_tree as tree

pytestmark = pytest.mark.gpu

TREES = [
    # d, B, H, G, T, n_max, at, count
    # several tiles for every compute unit, four waves each
    (32, 16, 16, 2, 9, 100, [91, 0, 5, -3, *range(20, 68, 4)], [9] * 15 + [2]),
    (64, 16, 16, 2, 9, 100, [91, 0, 5, 100, *range(20, 68, 4)], None),
    (128, 16, 16, 2, 9, 100, [91, 0, 5, 99, *range(20, 68, 4)], [9] * 14 + [0, 1]),
    # many query rows: a workgroup per tile, and one tree whose keys are shared out
    (32, 16, 8, 2, 130, 300, list(range(0, 160, 10)), [130] * 15 + [77]),
    (32, 1, 8, 4, 129, 5000, [4870], None),
    (64, 1, 8, 4, 129, 5000, [4870], [100]),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,B,H,G,T,n_max,at,count", TREES)
def test_tree_attention(dtype, d, B, H, G, T, n_max, at, count):
    tree.test_tree_attention(dtype, d, B, H, G, T, n_max, at, count)


KEEPS = [
    # d, B, H, n_max, at, paths: over 512 and over 64 rows, backwards and forwards
    (128, 2, 2, 1500, [447, 20], [list(range(1023, -1, -1)), list(range(1024))]),
    (32, 2, 2, 1500, [64, 401], [list(range(0, 1026, 2)), list(range(1024, 511, -1))]),
    (64, 1, 3, 700, [129], [list(range(2, 412, 2))]),
    (32, 1, 2, 700, [63], [list(range(130, -1, -2))]),
]


@pytest.mark.parametrize("d,B,H,n_max,at,paths", KEEPS)
def test_keep(d, B, H, n_max, at, paths):
    tree.test_keep(d, B, H, n_max, at, paths)
