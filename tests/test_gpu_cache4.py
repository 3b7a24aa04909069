"""The 4-bit cache on the GPU against float64: rows stored and loaded, attention over it, the lazy update, captured calls."""
import math

import numpy as np
import pytest

import lc_workloads as wl
from oracle import cache4_oracle as c4

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def C():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from tests import cache4_common
    return cache4_common


def _all(c):
    return [[np.arange(len(c.bounds[b]) - 1) for _ in range(c.H)] for b in range(c.B)]


# ------------------------------------------------------------------ rows

@pytest.mark.parametrize("layout", ["bhtr", "bthr", "padded"])
@pytest.mark.parametrize("lens", [[1], [63, 64, 65], [0, 200, 1, 17]])
def test_stored_rows(C, lens, layout):
    import torch
    c = C.Cache(1, 3, 1, lens, [np.array([0]) for _ in lens], extra=5, layout=layout)
    lc = C.lc
    back = [torch.full_like(c.K, 7.0) for _ in range(2)]
    lc.lc_cache4_load(c.K4, c.V4, *back, counts=lens)
    torch.cuda.synchronize()
    for x4, bits, y in ((c.K4, c.kb, back[0]), (c.V4, c.vb, back[1])):
        got = x4.cpu().numpy()
        for b, n in enumerate(lens):
            for h in range(c.H):
                want = c4.pack(wl.bf16_bits_to_f64(bits[b][h]))
                assert np.array_equal(got[b, h, :n], want), (b, h)
                assert np.array_equal(y[b, h, :n].float().cpu().numpy(), c4.unpack(want).astype(np.float32))
            assert (got[b, :, n:] == 255).all() and (y[b, :, n:] == 7).all()        # rows behind are left as they were


def test_every_kind_of_value(C):
    """Zeros of both signs, the smallest and the largest, infinities and what is no number, values on the codes' edges."""
    import torch
    lc = C.lc
    r = np.random.default_rng(3)
    bits = r.integers(0, 65536, size=(1, 1, 512, 128)).astype(np.uint16)            # any bits: most blocks hold something not finite
    bits[0, 0, 256:] &= 0xbfff                                                      # (exponents up to 127: finite)
    bits[0, 0, 300:400] &= 0x81ff                                                   # small and subnormal
    bits[0, 0, 400, :64] = 0
    bits[0, 0, 400, 64:] = 0x8000
    bits[0, 0, 401] = 0x7f7f
    edges = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5, 7], dtype=np.float32)
    bits[0, 0, 402] = wl.f32_to_bf16_bits(np.tile(edges, 8))
    K = C.to_dev(bits)
    K4, V4 = (torch.zeros(1, 1, 512, 68, dtype=torch.uint8, device="cuda") for _ in range(2))
    lc.lc_cache4_store(K, K, K4, V4)
    torch.cuda.synchronize()
    want = c4.pack(wl.bf16_bits_to_f64(bits[0, 0]))
    assert np.array_equal(K4[0, 0].cpu().numpy(), want) and torch.equal(K4, V4)
    back = torch.zeros_like(K)
    lc.lc_cache4_load(K4, V4, back, torch.zeros_like(K))
    torch.cuda.synchronize()
    assert np.array_equal(back[0, 0].float().cpu().numpy(), c4.unpack(want).astype(np.float32), equal_nan=True)


def test_ranges_of_many_sequences(C):
    """More sequences than one launch takes, each with a range of its own."""
    import torch
    lc = C.lc
    B, H, T = 130, 2, 40
    r = np.random.default_rng(4)
    first, counts = r.integers(0, 20, size=B), r.integers(0, 21, size=B)
    bits = C.bf16_bits(r, B, H, 20, 128)
    K4, V4 = (torch.full((B, H, T, 68), 9, dtype=torch.uint8, device="cuda") for _ in range(2))
    K = C.to_dev(bits)
    lc.lc_cache4_store(K, K, K4, V4, first=first, counts=counts)
    torch.cuda.synchronize()
    got = K4.cpu().numpy()
    for b in list(range(0, B, 13)) + [63, 64, 127, 128, 129]:
        want = np.full((H, T, 68), 9, dtype=np.uint8)
        for h in range(H):
            want[h, first[b]:first[b] + counts[b]] = c4.pack(wl.bf16_bits_to_f64(bits[b, h, :counts[b]]))
        assert np.array_equal(got[b], want), b
    back = torch.full_like(K, 3.0)
    lc.lc_cache4_load(K4, V4, back, torch.zeros_like(K), first=first, counts=counts)
    torch.cuda.synchronize()
    for b in (0, 64, 129):
        assert np.array_equal(back[b, 1, :counts[b]].float().cpu().numpy(), c4.unpack(got[b, 1, first[b]:first[b] + counts[b]]).astype(np.float32))
        assert (back[b, :, counts[b]:] == 3).all()


@pytest.mark.parametrize("layout", ["bthd", "padded"])
def test_bfloat16_rows_in_other_layouts(C, layout):
    import torch
    lc = C.lc
    r = np.random.default_rng(14)
    B, H, T = 2, 3, 150
    bits = C.bf16_bits(r, B, H, T, 128)

    def like(fill):
        if layout == "bthd":
            return torch.full((B, T, H, 128), fill, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
        return torch.full((B, H, T, 144), fill, dtype=torch.bfloat16, device="cuda")[..., 8:136]
    K, V, Kb, Vb = like(0.0), like(0.0), like(9.0), like(9.0)
    K.copy_(C.to_dev(bits))
    V.copy_(C.to_dev(bits[::-1].copy()))
    K4, V4 = (torch.zeros(B, H, T, 68, dtype=torch.uint8, device="cuda") for _ in range(2))
    lc.lc_cache4_store(K, V, K4, V4, counts=[T, 70])
    lc.lc_cache4_load(K4, V4, Kb, Vb, counts=[T - 1, 70])
    torch.cuda.synchronize()
    for x4, y, src in ((K4, Kb, bits), (V4, Vb, bits[::-1])):
        for b, n, m in ((0, T, T - 1), (1, 70, 70)):
            want = c4.pack(wl.bf16_bits_to_f64(src[b, 1, :n]))
            assert np.array_equal(x4[b, 1, :n].cpu().numpy(), want) and not x4[b, 1, n:].any()
            assert np.array_equal(y[b, 1, :m].float().cpu().numpy(), c4.unpack(want)[:m].astype(np.float32)) and (y[b, 1, m:] == 9).all()


# ------------------------------------------------------------------ attention

@pytest.mark.parametrize("G", range(1, 9))
@pytest.mark.parametrize("lens,lo,hi,share", [([300, 77], 1, 40, 0.6), ([1], 1, 1, 1.0), ([2, 33], 3, 5, 0.5), ([2100, 900, 1], 20, 90, 0.5)])
def test_attention(C, G, lens, lo, hi, share):
    r = np.random.default_rng(G)
    c = C.Cache(10 + G, 2, G, lens, [C.cut(r, n, lo, hi) for n in lens], extra=3)
    qb = c.query()
    ids = c.lists(share)
    out, lse = c.attend(qb, ids)
    c.check(qb, ids, out, lse)


@pytest.mark.parametrize("layout,splits", [("bthr", 0), ("padded", 0), ("bhtr", 1), ("bhtr", 7), ("bthr", 256)])
def test_attention_in_other_layouts_and_splits(C, layout, splits):
    r = np.random.default_rng(5)
    lens = [3000, 1, 640]
    c = C.Cache(20, 2, 4, lens, [C.cut(r, n, 5, 60) for n in lens], layout=layout, splits=splits)
    qb, ids = c.query(), _all(c)
    out, lse = c.attend(qb, ids)
    c.check(qb, ids, out, lse)


def test_long_lists_and_long_chunks(C):
    """More entries than a workgroup's threads hold at once; a chunk that spans tiles and splits."""
    bounds = [np.arange(0, 5001), np.array([0, 4000, 4001, 4999])]
    c = C.Cache(21, 1, 3, [5003, 5000], bounds)
    qb = c.query()
    for ids in (_all(c), [[np.arange(0, 5000, 2)], [np.array([0, 2])]], [[np.arange(2040, 2060)], [np.array([1])]]):
        out, lse = c.attend(qb, ids)
        c.check(qb, ids, out, lse)


def test_more_pairs_than_workgroups(C):
    """528 (sequence, head) pairs: one split each, which nobody merges."""
    r = np.random.default_rng(15)
    lens = [int(x) for x in r.integers(1, 400, size=66)]
    c = C.Cache(34, 8, 2, lens, [C.cut(r, n, 3, 30) for n in lens])
    qb, ids = c.query(), c.lists(0.8)
    out, lse = c.attend(qb, ids)
    for b in (0, 17, 65):
        for h in range(8):
            C.check_attention(c.heads(qb, b, h), c.k4(b, h), c.v4(b, h), c4.active_rows(c.bounds[b], c.lens[b], ids[b][h]), out[b, 2 * h:2 * h + 2], lse[b, 2 * h:2 * h + 2], (b, h))


def test_a_list_of_more_passes_than_slots(C):
    """140000 chunks of one token: the list is read in 69 passes, two of them to a slot."""
    n = 140000
    c = C.Cache(33, 1, 2, [n + 3], [np.arange(n + 1)], levels=1)
    qb = c.query()
    for ids in ([[np.arange(n)]], [[np.concatenate([np.arange(100), np.arange(135000, n, 2)])]]):
        out, lse = c.attend(qb, ids)
        c.check(qb, ids, out, lse)


@pytest.mark.parametrize("G", [2, 7])
def test_rows_that_attend_to_nothing(C, G):
    r = np.random.default_rng(6)
    lens = [40, 41, 0]
    c = C.Cache(22, 2, G, lens, [np.array([0, 20, 40]), np.array([0, 20, 40]), np.array([0])], extra=1)
    none = np.zeros(0, dtype=np.int64)
    qb = c.query()
    ids = [[none, np.array([1])], [none, np.array([0])], [none, none]]       # no tail; a tail of one token; no tokens at all
    out, lse = c.attend(qb, ids)
    assert not out[0, :G].any() and (lse[0, :G] == -math.inf).all() and not out[2].any() and (lse[2] == -math.inf).all()
    c.check(qb, ids, out, lse)
    assert np.array_equal(c.attend(qb, ids, with_lse=False)[0], out)


def test_entries_that_are_no_chunk_hold_no_tokens(C):
    r = np.random.default_rng(7)
    c = C.Cache(23, 1, 4, [100], [C.cut(r, 97, 5, 9)])
    M = len(c.bounds[0]) - 1
    qb = c.query()
    good = [[np.array([0, 2, M - 1])]]
    bad = [[np.array([0, -1, 2, M, M - 1, 0x7fffffff, -0x80000000, M + 1])]]
    a, la = c.attend(qb, good)
    b, lb = c.attend(qb, bad)
    assert np.array_equal(a, b) and np.array_equal(la, lb)


def test_large_logits_and_values(C):
    """Logits over some thousand powers of two: most weights vanish, nothing overflows; values near the format's ends.  A weight, and each of its
    three terms, has no place below 2^-126: up to three times that of every value is lost, besides what check_attention counts."""
    r = np.random.default_rng(8)
    for k_scale, v_scale in ((30.0, 1.0), (1.0, 1e30), (1.0, 1e-30), (1e-20, 1.0)):
        c = C.Cache(24, 1, 4, [700], [C.cut(r, 690, 5, 60)], k_scale=k_scale, v_scale=v_scale)
        qb = c.query(scale=20.0 if k_scale == 30.0 else 1.0)
        ids = _all(c)
        out, lse = c.attend(qb, ids)
        assert np.isfinite(out).all()
        rows = c4.active_rows(c.bounds[0], 700, ids[0][0])
        ref, ref_lse, size, prod = c4.attend(c.heads(qb, 0, 0), c.k4(0, 0), c.v4(0, 0), rows)
        x = 130 * C.EPS * prod
        lost = 3 * 2.0 ** -126 * np.abs(c.v4(0, 0)).sum(axis=0)
        assert np.all(np.abs(out[0] - ref) <= (2 * math.expm1(x) + 2.0 ** -15) * size + lost), k_scale
        assert np.all(np.abs(lse[0] - ref_lse) <= x + 2.0 ** -22 * np.abs(ref_lse) + 2.0 ** -18)


def test_blocks_that_are_no_numbers(C):
    """A row with such a block reaches the outputs that attend to it and no others."""
    import torch
    c = C.Cache(25, 2, 3, [200], [np.arange(0, 201, 10)])
    qb = c.query()
    ids = [[np.array([0, 3, 7]), np.array([1, 3])]]
    before, lse_before = c.attend(qb, ids)
    c.K4[0, :, 25, 64:] = 255                               # in chunk 2, which nobody lists
    c.V4[0, :, 25, 64:] = 255
    c.V4[0, 0, 75, 65] = 255                                # in chunk 7, listed by head 0: columns 32 .. 63
    torch.cuda.synchronize()
    out, lse = c.attend(qb, ids)
    assert np.isnan(out[0, :3, 32:64]).all() and np.array_equal(np.delete(out[0, :3], np.s_[32:64], 1), np.delete(before[0, :3], np.s_[32:64], 1))
    assert np.array_equal(out[0, 3:], before[0, 3:]) and np.array_equal(lse, lse_before)
    c.K4[0, 1, 12, 64] = 255                                # a key of chunk 1: head 1's softmax is no number
    torch.cuda.synchronize()
    out, lse = c.attend(qb, ids)
    assert np.isnan(out[0, 3:]).all() and np.isnan(lse[0, 3:]).all() and np.isfinite(lse[0, :3]).all()


def test_a_query_that_is_no_number_stays_alone(C):
    r = np.random.default_rng(9)
    for G in (3, 8):
        c = C.Cache(26, 2, G, [500], [C.cut(r, 500, 5, 40)])
        qb, ids = c.query(), _all(c)
        before, lse_before = c.attend(qb, ids)
        qb[0, 1, 5] = 0x7fc0
        out, lse = c.attend(qb, ids)
        assert np.isnan(out[0, 1]).all() and np.isnan(lse[0, 1])
        keep = [i for i in range(2 * G) if i != 1]
        assert np.array_equal(out[0, keep], before[0, keep]) and np.array_equal(lse[0, keep], lse_before[0, keep])


def test_offsets_beyond_32_bits(C):
    """Sequences and heads further apart than 4 GiB."""
    import torch
    lc = C.lc
    c = C.Cache(27, 2, 4, [300, 200], [np.arange(0, 301, 10), np.arange(0, 201, 10)])
    qb, ids = c.query(), _all(c)
    out, lse = c.attend(qb, ids)
    far = 5 << 30
    big = torch.empty(far + (3 << 30), dtype=torch.uint8, device="cuda")
    K4, V4 = (big.as_strided((2, 2, 300, 68), (far, (2 << 30) + 68 * 300, 68, 1), o) for o in (0, 1 << 20))
    lc.lc_cache4_store(c.K, c.V, K4, V4, counts=c.lens)
    c.K4, c.V4 = K4, V4
    got, got_lse = c.attend(qb, ids)
    assert np.array_equal(got, out) and np.array_equal(got_lse, lse)
    c.idx.close()
    del big


def test_the_same_bits_every_time(C):
    r = np.random.default_rng(11)
    c = C.Cache(28, 4, 4, [4000, 3000], [C.cut(r, 4000, 5, 60), C.cut(r, 2990, 5, 60)])
    qb, ids = c.query(), _all(c)
    a = c.attend(qb, ids)
    for _ in range(5):
        b = c.attend(qb, ids)
        assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


def test_argument_errors(C):
    import ctypes
    import torch
    lc = C.lc
    c = C.Cache(29, 2, 4, [100], [np.arange(0, 101, 10)])
    t, n = c.table(_all(c))
    q, out = C.to_dev(c.query()), torch.full((1, 8, 128), 5.0, device="cuda")
    L = lc.lib()
    p = lambda x: ctypes.c_void_p(x.data_ptr())

    def call(q=p(q), K=p(c.K4), s=(2 * 100 * 68, 100 * 68, 68), ids=p(t), cap=t.shape[2], H_q=8, out=p(out), ws=p(c.ws), nws=c.ws.numel()):
        return L.lc_sparse_decode4(c.idx.handle, q, K, p(c.V4), (ctypes.c_int64 * 3)(*s), ids, p(n), cap, H_q, out, None, ws, nws, None)

    assert call(q=None) == call(K=None) == call(ids=None) == call(out=None) == call(ws=None) == call(cap=0) == lc.LC_ERR_INVALID_ARG
    assert call(H_q=7) == call(H_q=18) == call(H_q=1) == call(s=(0, 0, 64)) == call(s=(0, 0, 70)) == call(s=(0, 0, 1 << 25)) == lc.LC_ERR_BAD_SHAPE
    assert call(K=ctypes.c_void_p(c.K4.data_ptr() + 2)) == call(ws=ctypes.c_void_p(c.ws.data_ptr() + 16)) == lc.LC_ERR_INVALID_ARG
    assert call(nws=1024) == lc.LC_ERR_WORKSPACE_TOO_SMALL
    torch.cuda.synchronize()
    assert (out == 5).all()
    assert call() == lc.LC_OK
    assert call(nws=lc.lc_decode_workspace_bytes(c.cfg, 1, 8, 2)) == lc.LC_OK
    torch.cuda.synchronize()
    k = torch.zeros(1, 2, 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(lc.LycheeError) as e:                 # the cache is full
        lc.lc_append4(c.idx, c.K4, c.V4, k, k)
    assert e.value.code == lc.LC_ERR_CAPACITY and c.idx.info(0)[0] == 100


# ------------------------------------------------------------------ lazy update

@pytest.mark.parametrize("geometry", [0, 1])
def test_appended_tokens_and_chunks(C, geometry):
    """With keys that the format holds exactly, the index grows to the bits that it has over a bfloat16 cache; the rows are the rounded ones."""
    import torch
    lc = C.lc
    r = np.random.default_rng(12)
    lens = [150, 90]
    new = 60
    mk = lambda: C.Cache(30, 2, 2, lens, [np.arange(0, 151, 10), np.arange(0, 81, 10)], extra=new, extra_chunks=10, levels=3, geometry=geometry)
    a, b = mk(), mk()
    # the open tail's keys as the 4-bit cache holds them, on both sides
    lc.lc_cache4_load(a.K4, a.V4, a.K, a.V, counts=lens)
    lc.lc_cache4_load(b.K4, b.V4, b.K, b.V, counts=lens)
    exact = c4.unpack(c4.pack(wl.bf16_bits_to_f64(C.bf16_bits(r, new * 4, 128)))).reshape(new, 2, 2, 128)
    close = r.random((new, 2)) < 0.15
    for i in range(new):
        k = C.to_dev(wl.f32_to_bf16_bits(exact[i].astype(np.float32)))
        v = C.to_dev(C.bf16_bits(r, 2, 2, 128))
        lc.lc_append(a.idx, a.K, a.V, k, v, close[i], a.ws)
        lc.lc_append4(b.idx, b.K4, b.V4, k, v, close[i])
        if i == new - 1:
            torch.cuda.synchronize()
            for s in range(2):
                for h in range(2):
                    assert np.array_equal(b.V4[s, h, lens[s] + i].cpu().numpy(), c4.pack(v[s, h].float().cpu().numpy()[None])[0])
    assert lc.lc_index_export(a.idx) == lc.lc_index_export(b.idx)
    for s in range(2):
        n = b.idx.info(s)[0]
        assert n == lens[s] + new
        got = c4.unpack(b.K4[s, 1, :n].cpu().numpy())
        assert np.array_equal(got[lens[s]:], exact[:, s, 1])
        if n < b.Tc:
            assert (b.K4[s, :, n:] == 255).all()


# ------------------------------------------------------------------ captured

def test_captured_and_replayed(C):
    """A step of append and attention in a graph, another graph on the same workspace, eager calls between the replays."""
    import torch
    lc = C.lc
    r = np.random.default_rng(13)
    lens = [700, 500]
    c = C.Cache(31, 2, 4, lens, [np.arange(0, 701, 20), np.arange(0, 501, 20)], extra=64)
    t, n = c.table(_all(c))
    q = [C.to_dev(c.query()) for _ in range(2)]
    out = [torch.zeros(2, 8, 128, device="cuda") for _ in range(2)]
    lse = [torch.zeros(2, 8, device="cuda") for _ in range(2)]
    k, v = (torch.zeros(2, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    side = torch.cuda.Stream()
    graphs = []
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for i in range(2):
            lc.lc_sparse_decode4(c.idx, q[i], c.K4, c.V4, t, n, out[i], c.ws, lse=lse[i])
        for i in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                if i == 0:
                    lc.lc_append4(c.idx, c.K4, c.V4, k, v)
                lc.lc_sparse_decode4(c.idx, q[i], c.K4, c.V4, t, n, out[i], c.ws, lse=lse[i])
            graphs.append(g)
    torch.cuda.synchronize()
    rows = [[C.bf16_bits(r, 2, 2, 128) for _ in range(2)] for _ in range(4)]
    kk = [[c.k4(b, h) for h in range(2)] for b in range(2)]
    vv = [[c.v4(b, h) for h in range(2)] for b in range(2)]
    for step, (kb, vb) in enumerate(rows):
        k.copy_(C.to_dev(kb))
        v.copy_(C.to_dev(vb))
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        eager, eager_lse = torch.zeros_like(out[0]), torch.zeros_like(lse[0])
        for i in range(2):
            lc.lc_sparse_decode4(c.idx, q[i], c.K4, c.V4, t, n, eager, c.ws, lse=eager_lse)
            torch.cuda.synchronize()
            assert torch.equal(eager, out[i]) and torch.equal(eager_lse, lse[i]), (step, i)
        for b in range(2):
            for h in range(2):
                kk[b][h] = np.concatenate([kk[b][h], c4.unpack(c4.pack(wl.bf16_bits_to_f64(kb[b, h][None])))])
                vv[b][h] = np.concatenate([vv[b][h], c4.unpack(c4.pack(wl.bf16_bits_to_f64(vb[b, h][None])))])
                rows_ = np.arange(len(kk[b][h]))
                C.check_attention(wl.bf16_bits_to_f64(q[0][b, 4 * h:4 * h + 4].view(torch.int16).cpu().numpy().view(np.uint16)), kk[b][h], vv[b][h], rows_,
                                  out[0][b, 4 * h:4 * h + 4].cpu().numpy(), lse[0][b, 4 * h:4 * h + 4].cpu().numpy(), (step, b, h))


def test_on_another_stream(C):
    import torch
    lc = C.lc
    c = C.Cache(32, 2, 4, [900], [np.arange(0, 901, 20)])
    qb, ids = c.query(), _all(c)
    want, want_lse = c.attend(qb, ids)
    t, n = c.table(ids)
    q, out, lse = C.to_dev(qb), torch.zeros(1, 8, 128, device="cuda"), torch.zeros(1, 8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    lc.lc_sparse_decode4(c.idx, q, c.K4, c.V4, t, n, out, c.ws, lse=lse, stream=s)
    s.synchronize()
    assert np.array_equal(out.cpu().numpy(), want) and np.array_equal(lse.cpu().numpy(), want_lse)
