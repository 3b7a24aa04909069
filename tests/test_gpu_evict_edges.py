"""Chunk weights where the list, the log-sum-exp or the keys are unusual, on the GPU against float64."""
import math

import numpy as np
import pytest

import lc_workloads as wl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def C():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from tests import cache4_common
    return cache4_common


def _weigh(C, c, qb, table, counts, lse, before, bits):
    import torch
    w = torch.from_numpy(before).cuda()
    call, K = (C.lc.lc_weigh_chunks4, c.K4) if bits == 4 else (C.lc.lc_weigh_chunks, c.K)
    call(c.idx, C.to_dev(qb), K, table, counts, torch.from_numpy(lse).cuda(), w)
    torch.cuda.synchronize()
    return w.cpu().numpy()


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("long", [False, True])
def test_heads_that_attended_to_nothing_with_keys_that_are_no_numbers(C, bits, long):
    """A head whose log-sum-exp is -inf adds nothing, also where its logits would be infinite or no numbers."""
    import torch
    bounds = np.array([0, 700, 1400, 1500]) if long else np.arange(0, 1501, 50)
    c = C.Cache(80, 1, 3, [1500], [bounds])
    M = len(bounds) - 1
    t, n = c.table([[np.arange(M)]])
    qb = c.query()
    c.K[0, 0, 10, 3] = math.nan
    c.K[0, 0, 1450] = math.inf
    C.lc.lc_cache4_store(c.K, c.V, c.K4, c.V4)
    bad = [int(np.searchsorted(bounds, r, side="right")) - 1 for r in (10, 1450)]
    before = np.full((1, 1, M), 2.0, dtype=np.float32)
    none = np.full((1, 3), -math.inf, dtype=np.float32)
    assert np.array_equal(_weigh(C, c, qb, t, n, none, before, bits), before)
    some = np.array([[-math.inf, 5.0, -math.inf]], dtype=np.float32)
    got = _weigh(C, c, qb, t, n, some, before, bits)
    fine = np.delete(np.arange(M), bad)
    assert np.isnan(got[0, 0, bad[0]]) and np.isfinite(got[0, 0, fine]).all() and (got[0, 0, fine] > 2).all()


@pytest.mark.parametrize("bits", [16, 4])
def test_entries_that_are_no_chunk_between_others(C, bits):
    """They hold no tokens, as in the attention; the chunk behind one is not measured against it."""
    import torch
    c = C.Cache(81, 1, 4, [400], [np.arange(0, 401, 10)])
    M = 40
    qb = c.query()
    good = [0, 4, 7, 9, 20, 39]
    lse = np.full((1, 4), 4.0, dtype=np.float32)
    before = np.ones((1, 1, M), dtype=np.float32)
    t, n = c.table([[np.array(good)]])
    want = _weigh(C, c, qb, t, n, lse, before, bits)
    holes = np.array([[[M + 5, 0, 0x7fffffff, 4, -1, 7, M, 9, -0x80000000, 20, 39, M]]], dtype=np.int32)
    got = _weigh(C, c, qb, torch.from_numpy(holes).cuda(), torch.tensor([[12]], dtype=torch.int32, device="cuda"), lse, before, bits)
    assert np.array_equal(got, want) and (want[0, 0, good] > 1).all() and (np.delete(want[0, 0], good) == 1).all()
