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


# A share of one token whose logit is one exact product, in EPS: the argument d scale - lse log2(e) is below 1 in size and rounded once (ln 2), the scale is off by .16 of its size
# (its constants' roundings, as float32 has them) times 32 powers of two at most (.16 * 32 ln 2), 2 of the exponential, 2 of the factor for what the offset's rounding
# has left, 1 of the product with it.
SHARE_EPS = 0.7 + 3.6 + 2 + 2 + 1


def _shares():
    """(log-sum-exp, logit d, share in float64, share with the rounded offset alone as float32 would have it)."""
    f = np.float32
    r = np.random.default_rng(6)
    d = np.round(r.uniform(16, 21.5, size=256) * math.sqrt(128) / 2) * 2
    lse = (d / math.sqrt(128) + r.uniform(-0.5, 0.5, size=256)).astype(f)
    off = f(-lse) * f(math.log2(math.e))
    rough = np.exp2(d * math.log2(math.e) / math.sqrt(128) + off.astype(np.float64))
    return lse, d, np.exp(d / math.sqrt(128) - lse.astype(np.float64)), rough


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("G", [1, 5])
def test_shares_to_a_few_roundings(C, bits, G):
    """Large log-sum-exps, whose product with log2(e) float32 holds to 2^-20."""
    lse, d, want, rough = _shares()
    assert (np.abs(rough - want) / want).max() > 1.2 * SHARE_EPS * C.EPS           # (so that the bound can tell)
    n = len(d)
    c = C.Cache(82, 1, G, [n], [np.arange(n + 1)])
    t, cnt = c.table([[np.arange(n)]])
    K = np.zeros((1, 1, c.Tc, 128))
    K[..., 5] = 4.0
    c.K.copy_(C.to_dev(wl.f32_to_bf16_bits(K.astype(np.float32))))
    C.lc.lc_cache4_store(c.K, c.K, c.K4, c.V4)
    worst = 0.0
    for i in range(n):
        # one head counts; another's logits and log-sum-exp stand beside it
        g = i % G
        q = np.zeros((1, G, 128))
        q[0, :, 5] = 1.0
        q[0, g, 5] = d[i] / 4.0
        qb = wl.f32_to_bf16_bits(q.astype(np.float32))
        assert np.array_equal(wl.bf16_bits_to_f64(qb), q)
        l = np.full((1, G), -math.inf, dtype=np.float32)
        l[0, g] = lse[i]
        got = _weigh(C, c, qb, t, cnt, l, np.zeros((1, 1, n), dtype=np.float32), bits)[0, 0]
        assert (got == got[0]).all()
        worst = max(worst, abs(float(got[0]) - want[i]) / want[i] / C.EPS)
    assert worst <= SHARE_EPS, worst


@pytest.mark.parametrize("bits", [16, 4])
def test_log_sum_exps_at_the_ends(C, bits):
    """Infinite or beyond every logit: a share of 0.  No number: none."""
    c = C.Cache(83, 1, 1, [100], [np.arange(0, 101, 10)])
    t, n = c.table([[np.arange(10)]])
    qb = c.query()
    before = np.ones((1, 1, 10), dtype=np.float32)
    for l in (math.inf, 3e38, 1e30, 1e10, 1e5):
        assert np.array_equal(_weigh(C, c, qb, t, n, np.full((1, 1), l, dtype=np.float32), before, bits), before), l
    assert np.isnan(_weigh(C, c, qb, t, n, np.full((1, 1), math.nan, dtype=np.float32), before, bits)).all()
