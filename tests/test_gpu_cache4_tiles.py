"""The 4-bit attention where a split has more tokens than the 8192 whose rows it looks up at a time."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def C():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from tests import cache4_common
    return cache4_common


def _check(C, c, lists):
    qb = c.query()
    for ids in lists:
        out, lse = c.attend(qb, ids)
        c.check(qb, ids, out, lse, [len(i) for i in ids[0]])


@pytest.mark.parametrize("splits", [1, 2])
@pytest.mark.parametrize("T", [8192, 8193, 16384, 16385])
def test_lists_that_fill_tiles_exactly(C, T, splits):
    T *= splits
    c = C.Cache(100, 1, 4, [T], [np.concatenate([np.arange(0, T, 64), [T]])], splits=splits)
    M = len(c.bounds[0]) - 1
    _check(C, c, [[[np.arange(M)]], [[np.arange(1, M)]]])


@pytest.mark.parametrize("splits", [1, 2, 3])
def test_chunks_that_cross_tiles(C, splits):
    """Few entries, held in registers, placed anew for each tile: chunks over the list's tokens 8192 and 16384, one inside a tile of its own, one of a token behind the border."""
    bounds = np.array([0, 7000, 9500, 9501, 17000, 17400, 41000, 41001])
    c = C.Cache(101, 1, 5, [41003], [bounds], splits=splits)
    _check(C, c, [[[np.arange(7)]], [[np.array([1, 3, 5])]], [[np.array([5])]], [[np.array([0, 2, 4, 5, 6])]]])


@pytest.mark.parametrize("splits", [1, 2])
def test_long_lists_over_several_tiles(C, splits):
    """More entries than a pass holds: each tile looks for its passes again."""
    c = C.Cache(102, 1, 3, [24007], [np.concatenate([np.arange(0, 6000), np.arange(6000, 24001, 5)])], splits=splits)
    M = len(c.bounds[0]) - 1
    _check(C, c, [[[np.arange(M)]], [[np.arange(0, M, 2)]], [[np.concatenate([np.arange(10), np.arange(M - 3000, M)])]]])


@pytest.mark.parametrize("splits", [1, 2])
def test_a_tail_longer_than_a_tile(C, splits):
    """Tiles that lie in the open tail alone, behind a short list, a long one, none."""
    c = C.Cache(103, 2, 8, [30000, 9000], [np.arange(0, 4001), np.array([0])], splits=splits)
    none = np.zeros(0, dtype=np.int64)
    for first in (np.arange(4000), np.arange(0, 4000, 3), none):
        _check(C, c, [[[first, none], [none, none]]])


def test_many_pairs_with_tiles_of_their_own(C):
    """520 pairs: one split each, of more than a tile."""
    import torch
    n = 8300
    c = C.Cache(104, 8, 1, [n] + [40] * 64, [np.concatenate([np.arange(0, 8200, 41), [8200]])] + [np.arange(0, 41, 8)] * 64)
    ids = [[np.arange(len(b) - 1)] * 8 for b in c.bounds]
    qb = c.query()
    out, lse = c.attend(qb, ids)
    from oracle import cache4_oracle as c4
    for b, h in ((0, 0), (0, 7), (1, 3), (64, 7)):
        C.check_attention(c.heads(qb, b, h), c.k4(b, h), c.v4(b, h), np.arange(c.lens[b]), out[b, h:h + 1], lse[b, h:h + 1], (b, h))
