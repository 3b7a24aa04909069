"""The reference of the 4-bit cache and of the eviction, pinned to what their definitions say, and the host side of their entry points."""
import ctypes
import math

import numpy as np
import pytest
import torch

import lc_workloads as wl
from oracle import cache4_oracle as c4
from paper_2603_08453_amd import binding as lc


def rows(seed, n, spread=0):
    r = np.random.default_rng(seed)
    x = r.standard_normal((n, 128)) * 2.0 ** r.integers(-spread, spread + 1, size=(n, 1))
    return wl.bf16_bits_to_f64(wl.f32_to_bf16_bits(x.astype(np.float32)))


def test_a_value_is_off_by_half_a_step_at_most():
    x = rows(1, 64, 20)
    y = c4.unpack(c4.pack(x))
    unit = (2.0 ** (c4.pack(x)[:, 64:].astype(float) - 127)).repeat(32, axis=1)
    a = np.abs(x) / unit
    step = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0))
    assert np.all(np.abs(x - y) <= step / 2 * unit) and a.max() <= 7
    # and no smaller power would do: at half of it the largest value is off by more
    top = a.reshape(64, 4, 32).max(axis=2)
    assert np.all(2 * top > 7)
    # the nearest of all sixteen
    every = np.concatenate([c4.GRID, -c4.GRID])
    near = np.abs(x[:, :, None] / unit[:, :, None] - every).min(axis=2)
    assert np.array_equal(near, np.abs(x - y) / unit)


@pytest.mark.parametrize("x,code", [(0.25, 0), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6), (7.0, 7), (0.26, 1), (5.01, 7), (0.0, 0)])
def test_ties_go_to_the_even_code(x, code):
    assert c4.code_of(x) == c4.code_of(-x) == code


def test_blocks_at_the_ends_of_the_range():
    x = np.zeros((5, 128))
    x[0, 0] = 3.3895313892515355e38                         # the largest bfloat16: 1.99 2^127, four units of 2^126
    x[1, 40] = math.inf
    x[2, 127] = math.nan
    x[3, 0] = -2.0 ** -128                                  # below the smallest power: half of it
    p = c4.pack(x)
    assert p[0, 64] == 253 and c4.unpack(p[:1])[0, 0] == 3 * 2.0 ** 126
    assert p[1, 65] == 255 and p[2, 67] == 255 and not p[1, 16:32].any() and np.isnan(c4.unpack(p[1:2])[0, 32:64]).all()
    assert np.isfinite(c4.unpack(p[1:2])[0, :32]).all()
    assert p[3, 64] == 0 and c4.unpack(p[3:4])[0, 0] == -2.0 ** -128
    assert not p[4].any() and not c4.unpack(p[4:]).any()


def test_what_is_stored_is_exact_in_bfloat16_and_stored_again_the_same():
    y = c4.unpack(c4.pack(rows(2, 32, 30)))
    assert np.array_equal(wl.bf16_bits_to_f64(wl.f32_to_bf16_bits(y.astype(np.float32))), y)
    assert np.array_equal(c4.unpack(c4.pack(y)), y)


def test_kept_chunks_by_hand():
    bounds = np.array([0, 4, 10, 12, 20, 25])               # sizes 4 6 2 8 5
    w = np.array([[1.0, 5.0, 2.0, 4.0, 0.0], [1.0, 0.0, 2.0, 0.5, 0.0]])      # sums 2 5 4 4.5 0
    assert c4.keep(w, bounds, 25, 0, 0) == [0, 1, 2, 3, 4]
    assert c4.keep(w, bounds, 16, 0, 0) == [1, 2, 3]        # 6 + 8 + 2
    assert c4.keep(w, bounds, 15, 0, 0) == [1, 3]           # the third does not fit: the prefix ends
    assert c4.keep(w, bounds, 5, 0, 0) == []
    assert c4.keep(w, bounds, 15, 1, 3) == [0, 1, 4]        # 4 + 5 pinned, 6 left
    assert c4.keep(w, bounds, 3, 1, 3) == [0, 4]
    w[1, 1] = math.nan
    assert c4.keep(w, bounds, 16, 0, 0) == [0, 2, 3]        # no number: last
    assert c4.keep(np.zeros((2, 5)), bounds, 12, 0, 0) == [0, 1, 2]


def test_row_size():
    assert lc.LC_CACHE4_ROW == c4.ROW == 68
    lc.lib()


def test_stores_and_loads_are_refused_before_any_gpu_work():
    L = lc.lib()
    fake = ctypes.c_void_p(0x10000)                         # never dereferenced
    s = (ctypes.c_int64 * 3)(8 * 64 * 128, 64 * 128, 128)
    s4 = (ctypes.c_int64 * 3)(8 * 64 * 68, 64 * 68, 68)
    two = lambda a, b: (ctypes.c_int32 * 2)(a, b)

    def call(load=False, K=fake, K4=fake, s=s, s4=s4, first=None, counts=two(3, 4), B=2, H=8, d=128, cap=64):
        if load:
            return L.lc_cache4_load(K4, fake, s4, first, counts, B, H, d, K, fake, s, cap, None)
        return L.lc_cache4_store(K, fake, s, first, counts, B, H, d, K4, fake, s4, cap, None)

    i64 = lambda *a: (ctypes.c_int64 * 3)(*a)
    for load in (False, True):
        assert call(load, K=None) == call(load, K4=None) == call(load, counts=None) == lc.LC_ERR_INVALID_ARG
        assert call(load, B=0) == call(load, H=0) == call(load, cap=0) == lc.LC_ERR_INVALID_ARG
        assert call(load, d=64) == lc.LC_ERR_BAD_SHAPE
        assert call(load, s=i64(8192, 8192, 100)) == call(load, s=i64(8192, 8192, 120)) == lc.LC_ERR_BAD_SHAPE
        assert call(load, s4=i64(4352, 4352, 64)) == call(load, s4=i64(4352, 4352, 70)) == call(load, s4=i64(-68, 4352, 68)) == lc.LC_ERR_BAD_SHAPE
        assert call(load, K=ctypes.c_void_p(0x10008)) == call(load, K4=ctypes.c_void_p(0x10002)) == lc.LC_ERR_INVALID_ARG
        assert call(load, counts=two(3, -1)) == call(load, first=two(-1, 0)) == lc.LC_ERR_INVALID_ARG
        assert call(load, counts=two(3, 65)) == call(load, first=two(0, 61)) == lc.LC_ERR_CAPACITY
        assert call(load, counts=two(0x7fffffff, 0), first=two(0x7fffffff, 0)) == lc.LC_ERR_CAPACITY
        assert call(load, counts=two(0, 0)) == lc.LC_OK      # nothing to do, nothing launched


def test_calls_without_an_index_are_refused():
    L = lc.lib()
    fake, s4 = ctypes.c_void_p(0x10000), (ctypes.c_int64 * 3)(4352, 4352, 68)
    assert L.lc_sparse_decode4(None, fake, fake, fake, s4, fake, fake, 16, 32, fake, None, fake, 1 << 20, None) == lc.LC_ERR_INVALID_ARG
    assert L.lc_append4(None, fake, fake, s4, fake, fake, None, None) == lc.LC_ERR_INVALID_ARG
    assert L.lc_weigh_chunks(None, fake, fake, s4, fake, fake, 16, 32, fake, fake, None) == lc.LC_ERR_INVALID_ARG
    assert L.lc_weigh_chunks4(None, fake, fake, s4, fake, fake, 16, 32, fake, fake, None) == lc.LC_ERR_INVALID_ARG
    assert L.lc_evict_select(None, fake, 10, 0, fake, fake, fake, None, fake, 1 << 20, None) == lc.LC_ERR_INVALID_ARG
    assert L.lc_evict_rows(None, fake, fake, fake, fake, fake, s4, fake, fake, s4, None, None, None) == lc.LC_ERR_INVALID_ARG
    assert L.lc_evict_rows4(None, fake, fake, fake, fake, fake, s4, fake, fake, s4, None, None, None) == lc.LC_ERR_INVALID_ARG


def test_the_binding_checks_tensors():
    K = torch.zeros(2, 3, 8, 128, dtype=torch.bfloat16)
    K4 = torch.zeros(2, 3, 8, 68, dtype=torch.uint8)
    class Stream:
        cuda_stream = 0
    for bad in (dict(K4=torch.zeros(2, 3, 8, 64, dtype=torch.uint8)), dict(K4=torch.zeros(2, 4, 8, 68, dtype=torch.uint8)),
                dict(K=torch.zeros(2, 3, 8, 128)), dict(counts=[9, 0]), dict(counts=[1]), dict(first=[0, 0, 0])):
        a = dict(K=K, K4=K4, counts=None, first=None)
        a.update(bad)
        with pytest.raises(AssertionError):
            lc.lc_cache4_store(a["K"], a["K"], a["K4"], a["K4"], first=a["first"], counts=a["counts"], stream=Stream)
        with pytest.raises(AssertionError):
            lc.lc_cache4_load(a["K4"], a["K4"], a["K"], a["K"], first=a["first"], counts=a["counts"], stream=Stream)
