"""What the library says of how it would cut a batch of decode requests with shared prefixes; refusals of that query
and of the prefixes' lists."""
import ctypes

import numpy as np
import pytest

from paper_2511_04791_amd import _native as N
from test_cache_ops_abi import DECODES, SHAPE, B, _batch, _prefixes


def _plan(native, shape, rows, length, of, eight):
    (arr, b), p, cut, block = _batch(rows), _prefixes(length, of), N.SharedCut(), (ctypes.c_int32 * max(1, len(length)))(*[-1] * len(length))
    assert native.duet_shared_plan(B(shape), B(b), B(p), eight, B(cut), block) == 0
    return cut, list(block)


def test_plan_of_shared_prefixes(native):
    """Which kernel a prefix goes to, whether results are joined, and how the batch reaches the launches."""
    def decodes(n, tokens):
        return [(1, r, 1, tokens - 1) for r in range(n)]
    cut, block = _plan(native, SHAPE, decodes(3, 20), [], [-1] * 3, 0)
    assert (cut.many_rows, cut.teams, cut.lone, cut.direct, cut.tables) == (0, 0, 6, 1, 32)
    cut, block = _plan(native, SHAPE, decodes(33, 200), [], [-1] * 33, 1)
    assert (cut.many_rows, cut.teams, cut.lone, cut.direct, cut.tables) == (0, 66, 0, 1, 256)
    cut, block = _plan(native, SHAPE, decodes(257, 200), [], [-1] * 257, 0)
    assert (cut.many_rows, cut.teams, cut.direct, cut.tables) == (0, 2 * 257, 1, 0)
    # prefixes of nobody, of one request, of no token, of two
    cut, block = _plan(native, SHAPE, decodes(5, 200), [16, 32, 0, 64], [1, 2, 2, 3, 3], 0)
    assert block == [0, 0, 0, 16] and cut.tables == 32 and not cut.direct and cut.many_rows == 0
    shape = N.Shape(32, 8, 128, 16, N.BF16, 1)
    for n, rows, tables in ((32, 128, 32), (64, 256, 256), (65, 160, 256), (300, 256, 0)):
        cut, block = _plan(native, shape, decodes(n, 32769), [32768], [0] * n, 0)
        assert block == [rows] and cut.many_rows % (8 * -(-4 * n // 256)) == 0 and cut.many_rows > 0 and cut.lone == 8 * n
        assert cut.tables == tables and not cut.direct
    # nine prefixes are more than the small tables hold
    cut, block = _plan(native, shape, decodes(18, 100), [16] * 9, [i // 2 for i in range(18)], 1)
    assert block == [16] * 9 and cut.tables == 256


def test_plan_refusals(native):
    cut = N.SharedCut()
    arr, b = _batch(DECODES)
    p = _prefixes([32], [0, 0, -1])
    assert native.duet_shared_plan(B(SHAPE), B(b), B(p), 0, B(cut), None) == 0
    assert native.duet_shared_plan(B(SHAPE), B(b), None, 1, B(cut), None) == 0
    assert native.duet_shared_plan(B(SHAPE), B(b), B(p), 2, B(cut), None) == -1
    assert native.duet_shared_plan(B(SHAPE), B(b), B(p), 0, None, None) == -1
    assert native.duet_shared_plan(B(SHAPE), None, B(p), 0, B(cut), None) == -1
    assert native.duet_shared_plan(B(SHAPE), B(b), B(_prefixes([20], [0, 0, -1])), 0, B(cut), None) == -1


@pytest.mark.parametrize("x", [np.array([2 ** 32]), np.array([-2 ** 31 - 1]), [0.5], np.array([np.nan]), [2 ** 31], np.array([2 ** 32 - 1], np.uint32)])
def test_lists_of_prefixes_are_not_cut_to_32_bits(x):
    """2^32 would be taken as prefix 0, whose pages the request does not have."""
    import paper_2511_04791_amd as duet
    with pytest.raises(ValueError), np.errstate(invalid="ignore"):
        duet._int32s(x, "prefix_of")


@pytest.mark.parametrize("x", [[], [3, -1], np.array([5, 7], np.int64), np.array([1.0, 2.0]), np.arange(6, dtype=np.int32)[::2], range(4), np.array([], np.int32)])
def test_lists_of_prefixes(x):
    import paper_2511_04791_amd as duet
    y = duet._int32s(x, "prefix_of")
    assert y.dtype == np.int32 and y.flags.c_contiguous and y.tolist() == [int(i) for i in x]
