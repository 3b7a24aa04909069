"""Eviction by accumulated attention weight on the GPU against float64: weights, selection, rows, and the whole of it around a 4-bit cache."""
import ctypes
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


# ------------------------------------------------------------------ weights

def _lse(C, c, qb, ids, keys):
    """As the attention over the listed chunks and the tail gives it, float32."""
    lse = np.full((c.B, c.H * c.G), -math.inf, dtype=np.float32)
    for b in range(c.B):
        for h in range(c.H):
            rows = c4.active_rows(c.bounds[b], c.lens[b], ids[b][h])
            k = keys(b, h)
            lse[b, h * c.G:(h + 1) * c.G] = c4.attend(c.heads(qb, b, h), k, k, rows)[1]
    return lse


def _weigh(C, c, qb, ids, lse, weights, bits, table=None):
    import torch
    t, n = table or c.table(ids)
    w = torch.from_numpy(weights).cuda()
    call, K = (C.lc.lc_weigh_chunks4, c.K4) if bits == 4 else (C.lc.lc_weigh_chunks, c.K)
    call(c.idx, C.to_dev(qb), K, t, n, torch.from_numpy(lse).cuda(), w)
    torch.cuda.synchronize()
    return w.cpu().numpy()


def _check_weights(C, c, qb, ids, lse, before, got, keys):
    """A share is an exponential with the logit's error (130 EPS sum |q_i k_i| / sqrt(d)) and those of the difference to the log-sum-exp (3 EPS of both in powers of
    two), and shares are added up in float32 (a chunk's tokens and heads: at most 64 roundings of a lane's sum and 12 to join them, up to 512 tokens), then to the weight."""
    for b in range(c.B):
        for h in range(c.H):
            q, k = c.heads(qb, b, h), keys(b, h)
            want = before[b, h].astype(np.float64)
            tol = np.zeros_like(want)
            for j, s in c4.chunk_weights(q, k, lse[b, h * c.G:(h + 1) * c.G].astype(np.float64), c.bounds[b], ids[b][h]).items():
                want[j] += s
                x = 130 * C.EPS * float((np.abs(q) @ np.abs(k[c.bounds[b][j]:c.bounds[b][j + 1]]).T).max()) / math.sqrt(128)
                x += 3 * C.EPS * (2 * x / (130 * C.EPS) + float(np.abs(lse[b, h * c.G:(h + 1) * c.G]).max()))
                tol[j] = (math.expm1(x) + 80 * C.EPS) * s + 2 * C.EPS * abs(want[j]) + 1e-36
            off = np.abs(got[b, h] - want)
            assert np.all(off <= tol), (b, h, float((off - tol).max()))
            untouched = np.ones(len(want), dtype=bool)
            untouched[ids[b][h]] = False
            assert np.array_equal(got[b, h][untouched], before[b, h][untouched])


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("G", range(1, 9))
def test_weights(C, G, bits):
    r = np.random.default_rng(G)
    lens = [700, 1, 333]
    c = C.Cache(40 + G, 2, G, lens, [C.cut(r, n, 1, 40) for n in lens], extra=2, layout="padded" if G % 2 else "bthr")
    keys = c.k4 if bits == 4 else (lambda b, h: wl.bf16_bits_to_f64(c.kb[b][h]))
    qb, ids = c.query(), c.lists(0.7)
    lse = _lse(C, c, qb, ids, keys)
    before = np.abs(r.standard_normal((3, 2, c.cfg.max_chunks))).astype(np.float32) * 0.01
    got = _weigh(C, c, qb, ids, lse, before, bits)
    _check_weights(C, c, qb, ids, lse, before, got, keys)
    again = _weigh(C, c, qb, ids, lse, got, bits)            # and once more: added to what is there
    _check_weights(C, c, qb, ids, lse, got, again, keys)


@pytest.mark.parametrize("bits", [16, 4])
def test_weights_of_long_chunks_and_long_lists(C, bits):
    bounds = [np.concatenate([np.arange(0, 3001), [3255, 3511, 3768, 4280]]), np.array([0, 255, 511, 768, 1279, 1280])]
    c = C.Cache(50, 2, 4, [4283, 1300], bounds)
    keys = c.k4 if bits == 4 else (lambda b, h: wl.bf16_bits_to_f64(c.kb[b][h]))
    qb = c.query()
    ids = [[np.arange(3004), np.arange(1, 3004, 2)], [np.arange(5), np.array([2])]]
    lse = _lse(C, c, qb, ids, keys)
    before = np.zeros((2, 2, c.cfg.max_chunks), dtype=np.float32)
    got = _weigh(C, c, qb, ids, lse, before, bits)
    _check_weights(C, c, qb, ids, lse, before, got, keys)
    # a whole list's weights and the tail's are the softmax: they add up to the group's heads
    rows = np.arange(bounds[1][-1], 1300)
    tail = np.exp(c.heads(qb, 1, 0) @ keys(1, 0)[rows].T / math.sqrt(128) - lse[1, :4, None].astype(np.float64)).sum()
    assert abs(got[1, 0].astype(np.float64).sum() + tail - 4) < 1e-4
    assert np.array_equal(_weigh(C, c, qb, ids, lse, before, bits), got)


@pytest.mark.parametrize("bits", [16, 4])
def test_weights_of_lists_longer_than_the_workgroups(C, bits):
    """64 pairs share the workgroups: each has more entries than a wavefront has lanes; a table with room for more."""
    n = 3000
    c = C.Cache(52, 8, 1, [n + 7] * 8, [np.concatenate([np.arange(0, n - 600), np.arange(n - 600, n + 1, 3)])] * 8)
    M = len(c.bounds[0]) - 1
    ids = [[np.arange(h % 3, M, 1 + h % 2) for h in range(8)] for _ in range(8)]
    keys = c.k4 if bits == 4 else (lambda b, h: wl.bf16_bits_to_f64(c.kb[b][h]))
    qb = c.query()
    lse = np.full((8, 8), 5.0, dtype=np.float32)
    before = np.abs(c.r.standard_normal((8, 8, c.cfg.max_chunks))).astype(np.float32)
    got = _weigh(C, c, qb, ids, lse, before, bits, c.table(ids, cap=M + 1500))
    for b, h in ((0, 0), (3, 5), (7, 7)):
        q, k = c.heads(qb, b, h), keys(b, h)
        share = np.exp(k[:c.bounds[b][-1]] @ q[0] / math.sqrt(128) - 5.0)
        want = before[b, h].astype(np.float64)
        want[ids[b][h]] += np.add.reduceat(share, c.bounds[b][:-1])[ids[b][h]]
        # as in _check_weights, with one head and at most three tokens
        x = 130 * C.EPS * float((np.abs(k) @ np.abs(q[0])).max()) / math.sqrt(128)
        x += 3 * C.EPS * (2 * x / (130 * C.EPS) + 5.0)
        assert np.all(np.abs(got[b, h] - want) <= (math.expm1(x) + 16 * C.EPS) * (want - before[b, h]) + 2 * C.EPS * want), (b, h)


@pytest.mark.parametrize("bits", [16, 4])
def test_a_table_with_the_largest_room(C, bits):
    """cap = 2^31 - 1, the lists as short as any."""
    import torch
    c = C.Cache(54, 1, 2, [300], [C.cut(np.random.default_rng(54), 300, 2, 20)])
    keys = c.k4 if bits == 4 else (lambda b, h: wl.bf16_bits_to_f64(c.kb[b][h]))
    qb, ids = c.query(), c.lists(0.7)
    t, n = c.table(ids)
    large = torch.empty(1, 1, 2**31 - 1, dtype=torch.int32, device="cuda")
    large[:, :, :t.shape[2]] = t
    lse = _lse(C, c, qb, ids, keys)
    before = np.zeros((1, 1, c.cfg.max_chunks), dtype=np.float32)
    got = _weigh(C, c, qb, ids, lse, before, bits, table=(large, n))
    _check_weights(C, c, qb, ids, lse, before, got, keys)


def test_entries_and_heads_that_add_nothing(C):
    import torch
    c = C.Cache(51, 1, 3, [200], [np.arange(0, 201, 10)])
    keys = c.k4
    qb, ids = c.query(), [[np.array([1, 4, 19])]]
    lse = _lse(C, c, qb, ids, keys)
    before = np.ones((1, 1, 20), dtype=np.float32)
    want = _weigh(C, c, qb, ids, lse, before, 4)
    t = torch.tensor([[[1, 1, 4, 4, 2, 19, 20, 0x7fffffff, -1]]], dtype=torch.int32, device="cuda")      # twice the same, descending, none of the chunks
    n = torch.tensor([[9]], dtype=torch.int32, device="cuda")
    assert np.array_equal(_weigh(C, c, qb, ids, lse, before, 4, (t, n)), want)
    assert np.array_equal(_weigh(C, c, qb, ids, lse, before, 4, (t, n * 0)), before)
    assert np.array_equal(_weigh(C, c, qb, ids, lse, before, 4, (t, n - 100)), before)
    assert np.array_equal(_weigh(C, c, qb, ids, lse, before, 4, (t, n + 100)), want)                    # counts end with the table
    none = np.full_like(lse, -math.inf)
    assert np.array_equal(_weigh(C, c, qb, ids, none, before, 4), before)


# ------------------------------------------------------------------ selection

def _select(C, c, weights, keep, recent, with_lens=True):
    import torch
    B, M = c.B, c.cfg.max_chunks
    ids = torch.full((B, M), 77, dtype=torch.int32, device="cuda")
    bounds = torch.full((B, M + 1), 77, dtype=torch.int32, device="cuda")
    counts, lens = (torch.full((B,), 77, dtype=torch.int32, device="cuda") for _ in range(2))
    C.lc.lc_evict_select(c.idx, torch.from_numpy(weights).cuda(), keep, recent, ids, bounds, counts, c.ws, keep_lens=lens if with_lens else None)
    torch.cuda.synchronize()
    return ids, bounds, counts, lens


def _check_select(C, c, weights, keep, recent, sink):
    ids, bounds, counts, lens = (x.cpu().numpy() for x in _select(C, c, weights, keep, recent))
    for b in range(c.B):
        M = len(c.bounds[b]) - 1
        want = c4.keep(weights[b, :, :M], c.bounds[b], keep, recent, sink)
        n = counts[b]
        assert n == len(want) and ids[b, :n].tolist() == want, (b, keep, recent, n, len(want))
        assert (ids[b, n:] == -1).all()
        size = np.diff(c.bounds[b])[want]
        assert np.array_equal(bounds[b, :n + 1], np.concatenate([[0], np.cumsum(size)])) and (bounds[b, n:] == size.sum()).all()
        assert lens[b] == size.sum() + c.lens[b] - c.bounds[b][-1]


@pytest.mark.parametrize("H,sink", [(1, 0), (3, 9), (8, 64)])
def test_selection(C, H, sink):
    r = np.random.default_rng(H)
    lens = [900, 5000, 1, 40, 0]
    bounds = [C.cut(r, 890, 1, 9), C.cut(r, 5000, 1, 5), np.array([0]), C.cut(r, 37, 37, 37), np.array([0])]
    c = C.Cache(60 + H, H, 1, lens, bounds, extra=1, sink=sink)
    w = np.exp(3 * r.standard_normal((5, H, c.cfg.max_chunks))).astype(np.float32)
    for keep, recent in ((0, 0), (1, 0), (37, 0), (450, 0), (450, 100), (100, 450), (2500, 1), (5000, 0), (1 << 30, 7), (0, 1 << 30)):
        _check_select(C, c, w, keep, recent, sink)
    # weights that differ in their last bits, and in nothing
    close = (1 + r.integers(0, 4, size=w.shape) * 2.0 ** -23).astype(np.float32)
    for keep in (1, 450, 2500):
        _check_select(C, c, close, keep, 50, sink)
        _check_select(C, c, np.zeros_like(w), keep, 0, sink)
    few = np.where(r.random(w.shape) < 0.3, w, 0).astype(np.float32)            # most of them never attended to
    for keep in (300, 2000, 4000):
        _check_select(C, c, few, keep, 64, sink)


def test_selection_of_weights_that_are_no_numbers(C):
    r = np.random.default_rng(4)
    c = C.Cache(64, 2, 1, [3000], [C.cut(r, 3000, 1, 5)])
    w = np.exp(r.standard_normal((1, 2, c.cfg.max_chunks))).astype(np.float32)
    M = len(c.bounds[0]) - 1
    w[0, 0, 5:M:7] = np.nan
    w[0, 1, 3:M:50] = np.inf
    w[0, 1, 4:M:50] = -np.inf
    w[0, 0, 11:M:90] = -1.0
    w[0, :, 12:M:90] = -0.0
    for keep in (10, 700, 2000, 2600, 2999, 3000):
        _check_select(C, c, w, keep, 0, 0)
    _check_select(C, c, np.full_like(w, np.nan), 1000, 0, 0)
    _check_select(C, c, np.full_like(w, np.inf), 1000, 0, 0)


def test_selection_among_many(C):
    """More chunks than threads, in one sequence 40000 of a token or two."""
    r = np.random.default_rng(5)
    c = C.Cache(65, 1, 1, [60000], [C.cut(r, 60000, 1, 2)])
    for w in (np.exp(4 * r.standard_normal((1, 1, c.cfg.max_chunks))), r.integers(0, 3, size=(1, 1, c.cfg.max_chunks)), 1e-40 * r.integers(0, 9, size=(1, 1, c.cfg.max_chunks))):
        for keep, recent in ((100, 0), (30000, 2000), (59990, 0)):
            _check_select(C, c, w.astype(np.float32), keep, recent, 0)


@pytest.mark.parametrize("H,chunks", [(2, (30000, 5, 14000)), (1, (14337, 13000, 0))])
def test_selection_by_several_workgroups(C, H, chunks):
    """A sequence with more chunks than one workgroup takes, others of the batch with fewer or none."""
    r = np.random.default_rng(H)
    bounds = [np.concatenate([[0], np.cumsum(r.integers(1, 3, size=n))]) for n in chunks]
    c = C.Cache(66, H, 1, [int(x[-1]) + 3 for x in bounds], bounds, sink=21)
    shape, n = (3, H, c.cfg.max_chunks), int(bounds[0][-1])
    spread = np.exp(3 * r.standard_normal(shape))
    for w in (spread, np.where(r.random(shape) < 0.2, spread, 0), np.zeros(shape), np.where(r.random(shape) < 0.1, np.nan, spread),
              1 + r.integers(0, 3, size=shape) * 2.0 ** -23, np.where(r.random(shape) < 0.5, np.inf, -spread)):
        for keep, recent in ((0, 0), (1, 300), (n // 3, 64), (n - 1, 0), (n, 0)):
            _check_select(C, c, w.astype(np.float32), keep, recent, 21)


@pytest.mark.parametrize("room,per", [(14336, 8), (14337, 16)])
def test_workspace_of_the_selection(C, room, per):
    """Its size goes by the room for chunks; a larger one is used no further."""
    import torch
    lc = C.lc
    c = C.Cache(68, 1, 1, [300], [np.arange(301)], extra=room, extra_chunks=room - 300, sink=5)
    w = np.exp(c.r.standard_normal((1, 1, room))).astype(np.float32)
    ws = torch.full((per * room + 256,), 7, dtype=torch.uint8, device="cuda")
    out = [torch.zeros(1, n, dtype=torch.int32, device="cuda") for n in (room, room + 1, 1)]
    with pytest.raises(lc.LycheeError) as e:
        lc.lc_evict_select(c.idx, torch.from_numpy(w).cuda(), 100, 0, *out, ws[:per * room - 1])
    assert e.value.code == lc.LC_ERR_WORKSPACE_TOO_SMALL
    lc.lc_evict_select(c.idx, torch.from_numpy(w).cuda(), 100, 0, *out, ws[:per * room])
    torch.cuda.synchronize()
    want = c4.keep(w[0, :, :300], np.arange(301), 100, 0, 5)
    assert out[0][0, :int(out[2])].tolist() == want and (ws[per * room:] == 7).all()


@pytest.mark.parametrize("chunks", [4096, 12288, 14336, 14337])
def test_captured_selection_of_a_growing_index(C, chunks):
    """The launches are chosen when they are captured; later calls have other weights and more chunks."""
    import torch
    lc = C.lc
    c = C.Cache(67, 1, 1, [chunks], [np.arange(chunks + 1)], extra=6, extra_chunks=6)
    M = c.cfg.max_chunks
    w = torch.zeros(1, 1, M, device="cuda")
    got = [torch.zeros(1, n, dtype=torch.int32, device="cuda") for n in (M, M + 1)] + [torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2)]
    call = lambda: lc.lc_evict_select(c.idx, w, 3000, 9, got[0], got[1], got[2], c.ws, keep_lens=got[3])
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    row = torch.zeros(1, 1, 128, dtype=torch.bfloat16, device="cuda")
    for step in range(4):
        now = np.exp(c.r.standard_normal((1, 1, M))).astype(np.float32)
        w.copy_(torch.from_numpy(now))
        graph.replay()
        torch.cuda.synchronize()
        bounds = np.arange(chunks + step + 1)
        want = c4.keep(now[0, :, :chunks + step], bounds, 3000, 9, 0)
        assert int(got[2]) == len(want) == int(got[3]) and got[0][0, :len(want)].tolist() == want and (got[0][0, len(want):] == -1).all()
        eager = _select(C, c, now, 3000, 9)
        assert all(torch.equal(x, y) for x, y in zip(got, eager))
        lc.lc_append(c.idx, c.K, c.V, row, row, [1], c.ws)


# ------------------------------------------------------------------ rows

@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("layout", ["bhtr", "bthr", "padded"])
def test_rows_that_stay(C, bits, layout):
    import torch
    lc = C.lc
    r = np.random.default_rng(6)
    lens = [1500, 1, 300, 64, 0]
    bounds = [C.cut(r, 1490, 1, 7), np.array([0]), np.array([0, 299]), np.arange(65), np.array([0])]
    c = C.Cache(70, 2, 1, lens, bounds, extra=2, layout=layout, sink=3)
    w = np.exp(r.standard_normal((5, 2, c.cfg.max_chunks))).astype(np.float32)
    for keep, recent in ((700, 50), (0, 0), (1 << 20, 0), (63, 1)):
        ids, kb, counts, new = _select(C, c, w, keep, recent)
        if bits == 16:
            K, V, to = c.K, c.V, [torch.full_like(c.K, 5.0).transpose(0, 1).contiguous().transpose(0, 1) for _ in range(2)]
        else:
            K, V, to = c.K4, c.V4, [torch.full((5, 2, c.Tc, 100), 99, dtype=torch.uint8, device="cuda")[..., 8:76] for _ in range(2)]
        wt = torch.full((5, 2, c.cfg.max_chunks), -3.0, device="cuda")
        wd = torch.from_numpy(w).cuda()
        lc.lc_evict_rows(c.idx, ids, kb, counts, K, V, *to, weights=wd, weights_to=wt)
        torch.cuda.synchronize()
        for b in range(5):
            pick = ids[b, :counts[b]].cpu().numpy()
            rows = torch.from_numpy(c4.active_rows(c.bounds[b], lens[b], pick)).cuda()
            assert len(rows) == int(new[b])
            for x, y in ((K, to[0]), (V, to[1])):
                assert torch.equal(y[b, :, :len(rows)], x[b][:, rows]), (b, keep)
                assert (y[b, :, len(rows):] == (5 if bits == 16 else 99)).all()
            assert np.array_equal(wt[b, :, :len(pick)].cpu().numpy(), w[b][:, pick]) and not wt[b, :, len(pick):].any()
        before = [t.clone() for t in to]
        lc.lc_evict_rows(c.idx, ids, kb, counts, K, V, *to)                      # without weights: the same rows
        torch.cuda.synchronize()
        assert torch.equal(to[0], before[0]) and torch.equal(to[1], before[1])


def test_argument_errors(C):
    import torch
    lc = C.lc
    c = C.Cache(71, 2, 4, [100], [np.arange(0, 101, 10)])
    L, i64 = lc.lib(), lambda *a: (ctypes.c_int64 * 3)(*a)
    p = lambda x, o=0: ctypes.c_void_p(x.data_ptr() + o)
    t, n = c.table([[np.arange(10)] * 2])
    q, lse, w = C.to_dev(c.query()), torch.zeros(1, 8, device="cuda"), torch.full((1, 2, 10), 4.0, device="cuda")
    s, s4 = (2 * 100 * 128, 100 * 128, 128), (2 * 100 * 68, 100 * 68, 68)

    def weigh(q=p(q), K=p(c.K), s=s, ids=p(t), cap=10, H_q=8, lse=p(lse), w=p(w)):
        return L.lc_weigh_chunks(c.idx.handle, q, K, i64(*s), ids, p(n), cap, H_q, lse, w, None)

    def weigh4(K=p(c.K4), s=s4, H_q=8):
        return L.lc_weigh_chunks4(c.idx.handle, p(q), K, i64(*s), p(t), p(n), 10, H_q, p(lse), p(w), None)

    assert weigh(q=None) == weigh(K=None) == weigh(ids=None) == weigh(cap=0) == weigh(lse=None) == weigh(w=None) == lc.LC_ERR_INVALID_ARG
    assert weigh(K=p(c.K, 8)) == weigh(q=p(q, 8)) == weigh4(K=p(c.K4, 2)) == lc.LC_ERR_INVALID_ARG
    assert weigh(H_q=7) == weigh(H_q=18) == weigh(s=(0, 0, 120)) == weigh(s=(0, 0, 1 << 24)) == weigh4(s=(0, 0, 66)) == weigh4(s=(0, 0, 1 << 25)) == lc.LC_ERR_BAD_SHAPE
    ids, kb, counts = torch.zeros(1, 10, dtype=torch.int32, device="cuda"), torch.zeros(1, 11, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")

    def select(w=p(w), keep=10, recent=0, ids=p(ids), ws=p(c.ws), nws=c.ws.numel()):
        return L.lc_evict_select(c.idx.handle, w, keep, recent, ids, p(kb), p(counts), None, ws, nws, None)

    assert select(w=None) == select(ids=None) == select(ws=None) == select(keep=-1) == select(recent=-1) == select(ws=p(c.ws, 8)) == lc.LC_ERR_INVALID_ARG
    assert select(nws=79) == lc.LC_ERR_WORKSPACE_TOO_SMALL
    to = [torch.full_like(c.K, 5.0) for _ in range(2)]

    def rows(K=p(c.K), V=p(c.V), K_to=p(to[0]), V_to=p(to[1]), s=s, st=s, w=None, wt=None):
        return L.lc_evict_rows(c.idx.handle, p(ids), p(kb), p(counts), K, V, i64(*s), K_to, V_to, i64(*st), w, wt, None)

    assert rows(K=None) == rows(V_to=None) == rows(w=p(w)) == rows(wt=p(w)) == rows(w=p(w), wt=p(w)) == rows(K=p(c.K, 8)) == lc.LC_ERR_INVALID_ARG
    assert rows(K_to=p(c.K)) == rows(V_to=p(c.K)) == rows(V_to=p(to[0])) == lc.LC_ERR_INVALID_ARG
    assert rows(s=(0, 0, 100)) == rows(st=(0, 0, 100)) == lc.LC_ERR_BAD_SHAPE
    torch.cuda.synchronize()
    assert (w == 4).all() and not counts.any() and (to[0] == 5).all()
    assert select(nws=80) == rows() == weigh() == weigh4() == lc.LC_OK
    torch.cuda.synchronize()


# ------------------------------------------------------------------ together

def test_a_generation_with_evictions(C):
    """A prompt stored in 4 bits, tokens generated over it, two evictions on the way: every step's attention and the weights against float64 over what the cache should hold."""
    import torch
    lc = C.lc
    r = np.random.default_rng(7)
    H, G, B, T0, steps = 2, 4, 2, [900, 700], 90
    cap = 1000
    bounds = [C.cut(r, n, 8, 30) for n in T0]
    c = C.Cache(72, H, G, T0, bounds, extra=cap - 900, extra_chunks=120, levels=3, sink=8)
    spare = [c.narrow("bhtr") for _ in range(2)]
    K4, V4, idx = c.K4, c.V4, c.idx
    weights, weights_to = (torch.zeros(B, H, c.cfg.max_chunks, device="cuda") for _ in range(2))
    # what the cache should hold, on the host
    hold = [[(c.k4(b, h), c.v4(b, h)) for h in range(H)] for b in range(B)]
    cuts = [list(x) for x in bounds]
    ids = torch.zeros(B, H, c.cfg.max_chunks, dtype=torch.int32, device="cuda")
    counts = torch.zeros(B, H, dtype=torch.int32, device="cuda")
    out, lse = torch.zeros(B, H * G, 128, device="cuda"), torch.zeros(B, H * G, device="cuda")
    gathered = np.zeros((B, H, c.cfg.max_chunks))
    for step in range(steps):
        qb = c.query()
        q = C.to_dev(qb)
        lc.lc_retrieve(idx, q, 200, ids, counts, c.ws)
        lc.lc_sparse_decode4(idx, q, K4, V4, ids, counts, out, c.ws, lse=lse)
        lc.lc_weigh_chunks4(idx, q, K4, ids, counts, lse, weights)
        torch.cuda.synchronize()
        for b in range(B):
            for h in range(H):
                pick = ids[b, h, :counts[b, h]].cpu().numpy()
                k, v = hold[b][h]
                assert np.all(np.diff(pick) > 0) and np.diff(cuts[b])[pick[np.array(cuts[b])[pick] >= 8]].sum() <= 200     # (the pinned chunks are not charged)
                qh, l = c.heads(qb, b, h), lse[b, h * G:(h + 1) * G].cpu().numpy()
                C.check_attention(qh, k, v, c4.active_rows(np.array(cuts[b]), len(k), pick), out[b, h * G:(h + 1) * G].cpu().numpy(), l, (step, b, h))
                for j, s in c4.chunk_weights(qh, k, l.astype(np.float64), np.array(cuts[b]), pick).items():
                    gathered[b, h, j] += s
        # 60 steps of shares at most G each, every one off by 1e-4 of itself at most at these logits, and added up in float32
        assert np.allclose(weights.cpu().numpy(), gathered, rtol=1e-4, atol=1e-6)
        kb, vb, close = C.bf16_bits(r, B, H, 128), C.bf16_bits(r, B, H, 128), r.random(B) < 0.08
        lc.lc_append4(idx, K4, V4, C.to_dev(kb), C.to_dev(vb), close)
        for b in range(B):
            for h in range(H):
                k, v = hold[b][h]
                hold[b][h] = (np.concatenate([k, c4.unpack(c4.pack(wl.bf16_bits_to_f64(kb[b, h][None])))]), np.concatenate([v, c4.unpack(c4.pack(wl.bf16_bits_to_f64(vb[b, h][None])))]))
            if close[b]:
                cuts[b].append(len(hold[b][0][0]))
        if step in (30, 65):
            kept = [torch.zeros(B, c.cfg.max_chunks, dtype=torch.int32, device="cuda"), torch.zeros(B, c.cfg.max_chunks + 1, dtype=torch.int32, device="cuda"),
                    torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")]
            lc.lc_evict_select(idx, weights, 500, 60, *kept[:3], c.ws, keep_lens=kept[3])
            lc.lc_evict_rows(idx, *kept[:3], K4, V4, *spare, weights=weights, weights_to=weights_to)
            n, lens = kept[2].tolist(), kept[3].tolist()
            new_bounds = [kept[1][b, :n[b] + 1].tolist() for b in range(B)]
            w = weights.cpu().numpy()
            for b in range(B):
                old = np.array(cuts[b])
                pick = kept[0][b, :n[b]].cpu().numpy()
                assert pick.tolist() == c4.keep(w[b, :, :len(old) - 1], old, 500, 60, 8)
                rows = c4.active_rows(old, len(hold[b][0][0]), pick)
                hold[b] = [(k[rows], v[rows]) for k, v in hold[b]]
                assert new_bounds[b] == [0] + np.cumsum(np.diff(old)[pick]).tolist() and lens[b] == len(rows) and new_bounds[b][-1] <= 500
                cuts[b] = new_bounds[b]
                g = np.zeros_like(gathered[b])
                g[:, :len(pick)] = gathered[b][:, pick]
                gathered[b] = g
            (K4, V4), spare = spare, [K4, V4]
            weights, weights_to = weights_to, weights
            wide = [torch.zeros(B, H, cap, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
            lc.lc_cache4_load(K4, V4, *wide, counts=lens)
            idx = lc.lc_build_index(c.cfg, wide[0], lens, new_bounds, c.buf, c.ws)
    assert idx.info(0)[0] == len(hold[0][0][0]) < T0[0] + steps


def test_captured_weights_and_eviction(C):
    """A step's weights and a whole eviction in one graph; every replay against the eager calls."""
    import torch
    lc = C.lc
    r = np.random.default_rng(8)
    lens = [800, 600]
    c = C.Cache(73, 2, 4, lens, [C.cut(r, n, 3, 20) for n in lens], extra=1)
    t, n = c.table([[np.arange(len(b) - 1)] * 2 for b in c.bounds])
    M = c.cfg.max_chunks
    q, lse = C.to_dev(c.query()), torch.full((2, 8), 7.0, device="cuda")
    mk = lambda: dict(w=torch.zeros(2, 2, M, device="cuda"), wt=torch.zeros(2, 2, M, device="cuda"), K=torch.zeros_like(c.K4), V=torch.zeros_like(c.V4),
                      kept=[torch.zeros(2, M, dtype=torch.int32, device="cuda"), torch.zeros(2, M + 1, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")])
    a, e = mk(), mk()

    def step(s):
        lc.lc_weigh_chunks4(c.idx, q, c.K4, t, n, lse, s["w"])
        lc.lc_evict_select(c.idx, s["w"], 300, 40, *s["kept"], c.ws)
        lc.lc_evict_rows(c.idx, *s["kept"], c.K4, c.V4, s["K"], s["V"], weights=s["w"], weights_to=s["wt"])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(mk())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step(a)
    torch.cuda.synchronize()
    for i in range(4):
        q.copy_(C.to_dev(c.query()))
        g.replay()
        torch.cuda.synchronize()
        step(e)
        torch.cuda.synchronize()
        for x, y in zip([a[k] for k in ("w", "wt", "K", "V")] + a["kept"], [e[k] for k in ("w", "wt", "K", "V")] + e["kept"]):
            assert torch.equal(x, y), i
        assert int(a["kept"][2].min()) > 0
