"""Calls of the 8-bit operators whose results would fall on one another. No GPU."""
import itertools

import pytest

import paper_2605_08696_b200 as P
from test_ops8_host import A, INVALID, _gemm, _norm, _quant

BAD_ADDRESS = A + 2               # refused for its alignment, which is looked at after the strides: nothing is launched


def _overlap(rows, blks, row, blk):
    places = [i * row + b * blk for i, b in itertools.product(range(rows), range(blks))]
    return len(set(places)) < len(places)


@pytest.mark.parametrize("rows,blks", [(1, 1), (1, 3), (2, 1), (2, 2), (2, 3), (3, 2), (4, 5), (7, 3)])
def test_written_scales_have_a_place_each(rows, blks):
    """Row and block strides that put two scales into one place are refused, all others are taken."""
    K = 128 * blks
    refused = 0
    for row, blk in itertools.product(range(1, 9), repeat=2):
        want = INVALID if _overlap(rows, blks, row, blk) else P.ERR_ALIGNMENT
        refused += want == INVALID
        assert _norm(R=rows, d=K, xs=K, qs=K, s=BAD_ADDRESS, sr=row, sb=blk) == want, (row, blk)
        assert _quant(R=rows, K=K, xs=K, qs=K, s=BAD_ADDRESS, sr=row, sb=blk) == want, (row, blk)
        assert _quant(R=128 * rows - 5, K=K, xs=K, qs=K, br=128, s=BAD_ADDRESS, sr=row, sb=blk) == want, (row, blk)
        # scales that are read may share places
        assert _gemm(M=rows, K=K, as_=K, ws=K, sa=BAD_ADDRESS, sar=row, sab=blk) == P.ERR_ALIGNMENT
    assert (refused > 0) == (rows > 1 and blks > 1)


def test_a_stored_sum_in_place_of_x_has_x_s_stride():
    kw = dict(x=A, xs=256, dl=A + (1 << 20), ds=128, s=BAD_ADDRESS)
    assert _norm(h=A, hs=256, **kw) == P.ERR_ALIGNMENT
    assert _norm(h=A, hs=128, **kw) == INVALID
    assert _norm(R=1, h=A, hs=128, **kw) == P.ERR_ALIGNMENT      # a single row has no stride


def test_a_product_of_more_tiles_than_are_counted_is_refused_before_anything_else():
    """2^30 tiles of 256 x 256 and more (2^46 elements of output)."""
    kw = dict(as_=128, ws=128, K=128, st=BAD_ADDRESS)
    M, N = 1 << 23, (1 << 23) - 256
    assert _gemm(M=M, N=N, os=N, **kw) == P.ERR_ALIGNMENT        # (2^15 x (2^15 - 1) tiles: the status word's address comes next)
    assert _gemm(M=M, N=N + 1, os=N + 1, **kw) == P.ERR_UNSUPPORTED
    assert _gemm(M=1 << 30, N=1 << 30, os=1 << 30, **kw) == P.ERR_UNSUPPORTED
