"""The rows that stay, moved past the caches, by fewer workgroups than tiles, and with more weights than workgroups: exactly, and nothing behind them touched."""
import numpy as np
import pytest

from oracle import cache4_oracle as c4

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def C():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from tests import cache4_common
    return cache4_common


def _select(C, c, weights, keep, recent):
    import torch
    B, M = c.B, c.cfg.max_chunks
    kept = [torch.zeros(B, M, dtype=torch.int32, device="cuda"), torch.zeros(B, M + 1, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")]
    C.lc.lc_evict_select(c.idx, weights, keep, recent, *kept, c.ws)
    return kept


def _check_rows(c, kept, pairs, fill, sequences=None):
    """pairs: (source, destination)."""
    import torch
    torch.cuda.synchronize()
    for b in range(c.B) if sequences is None else sequences:
        pick = kept[0][b, :int(kept[2][b])].cpu().numpy()
        rows = torch.from_numpy(c4.active_rows(c.bounds[b], c.lens[b], pick)).cuda()
        for x, y in pairs:
            assert torch.equal(y[b, :, :len(rows)], x[b][:, rows]), b
            assert (y[b, :, len(rows):] == fill).all(), b


@pytest.mark.parametrize("layout", ["bhtd", "bthd", "padded"])
def test_bfloat16_rows_past_the_caches(C, layout):
    """Over 32 MB of keys and values: 70034 rows of two heads at 512 bytes are 36."""
    import torch
    r = np.random.default_rng(1)
    lens = [30011, 5003, 0, 1, 2]
    c = C.Cache(110, 2, 1, lens, [C.cut(r, 30000, 1, 30), C.cut(r, 5003, 200, 900), np.array([0]), np.array([0, 1]), np.array([0])], extra=3, sink=4)
    assert sum(lens) * 2 * 512 > 32 << 20
    T = c.Tc

    def like(fill):
        if layout == "bhtd":
            return torch.full((5, 2, T, 128), fill, dtype=torch.bfloat16, device="cuda")
        if layout == "bthd":
            return torch.full((5, T, 2, 128), fill, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
        return torch.full((5, 2, T, 144), fill, dtype=torch.bfloat16, device="cuda")[..., 8:136]
    K, V, K_to, V_to = like(0.0), like(0.0), like(9.0), like(9.0)
    K.copy_(c.K)
    V.copy_(c.V)
    w = torch.from_numpy(np.exp(r.standard_normal((5, 2, c.cfg.max_chunks))).astype(np.float32)).cuda()
    for keep, recent in ((16000, 100), (1 << 30, 0), (5, 0)):
        kept = _select(C, c, w, keep, recent)
        K_to.fill_(9.0)
        V_to.fill_(9.0)
        C.lc.lc_evict_rows(c.idx, *kept, K, V, K_to, V_to)
        _check_rows(c, kept, ((K, K_to), (V, V_to)), 9.0)


def test_narrow_rows_by_fewer_workgroups_than_tiles(C):
    """64 pairs have 64 workgroups each for up to 79 tiles."""
    import torch
    r = np.random.default_rng(2)
    lens = [5003, 4097, 4096, 5000, 1, 0, 640, 4999]
    c = C.Cache(111, 8, 1, lens, [C.cut(r, max(0, n - 3), 3, 40) for n in lens], extra=1)
    w = torch.from_numpy(np.exp(r.standard_normal((8, 8, c.cfg.max_chunks))).astype(np.float32)).cuda()
    to = [torch.full_like(c.K4, 99) for _ in range(2)]
    for keep in (1 << 30, 4500, 2000):
        kept = _select(C, c, w, keep, 50)
        for x in to:
            x.fill_(99)
        C.lc.lc_evict_rows(c.idx, *kept, c.K4, c.V4, *to)
        _check_rows(c, kept, ((c.K4, to[0]), (c.V4, to[1])), 99)


def test_bfloat16_rows_by_fewer_workgroups_than_tiles(C):
    """8192 pairs have 4 workgroups each for up to 5 tiles."""
    import torch
    lc, B, H, T = C.lc, 1024, 8, 300
    r = np.random.default_rng(3)
    lens = [int(n) for n in r.integers(200, T + 1, size=B)]
    lens[:3] = [T, 257, 0]

    class Many:
        pass
    c = Many()
    c.B, c.lens, c.bounds = B, lens, [C.cut(r, n, 5, 40) for n in lens]
    M = max(len(b) - 1 for b in c.bounds)
    c.cfg = lc.lc_config_default(levels=1, max_chunks=M, max_tokens=T)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    K, V = (torch.randint(-2 ** 15, 2 ** 15, (B, H, T, 128), dtype=torch.int16, device="cuda", generator=gen) & 0x3fff for _ in range(2))      # (finite as bfloat16)
    c.ws = torch.zeros(lc.lc_workspace_bytes(c.cfg, B, H, H), dtype=torch.uint8, device="cuda")
    buf = torch.zeros(lc.lc_index_bytes(c.cfg, B, H), dtype=torch.uint8, device="cuda")
    c.idx = lc.lc_build_index(c.cfg, K, lens, c.bounds, buf, c.ws)
    w = torch.rand(B, H, M, device="cuda", generator=gen)
    to = [torch.full_like(K, -1) for _ in range(2)]
    for keep in (1 << 30, 150):
        kept = _select(C, c, w, keep, 0)
        for x in to:
            x.fill_(-1)
        lc.lc_evict_rows(c.idx, *kept, K, V, *to)
        _check_rows(c, kept, ((K, to[0]), (V, to[1])), -1, sequences=[0, 1, 2, 511, 1023])
    del c.idx


@pytest.mark.parametrize("bits", [16, 4])
def test_weights_of_more_chunks_than_workgroups(C, bits):
    """64 workgroups of 256 threads go through 20003 chunks' weights."""
    import torch
    r = np.random.default_rng(4)
    n = 20000
    c = C.Cache(112, 2, 1, [n + 2, 7], [np.arange(n + 1), np.arange(8)], extra=3, extra_chunks=3, levels=1)
    w = np.exp(r.standard_normal((2, 2, c.cfg.max_chunks))).astype(np.float32)
    wd, wt = torch.from_numpy(w).cuda(), torch.full((2, 2, c.cfg.max_chunks), -3.0, device="cuda")
    K, V, fill = (c.K, c.V, 5) if bits == 16 else (c.K4, c.V4, 99)
    for keep in (1 << 30, 17000, 3):
        kept = _select(C, c, wd, keep, 0)
        to = [torch.full_like(K, fill) for _ in range(2)]
        wt.fill_(-3.0)
        C.lc.lc_evict_rows(c.idx, *kept, K, V, *to, weights=wd, weights_to=wt)
        _check_rows(c, kept, ((K, to[0]), (V, to[1])), fill)
        for b in range(2):
            pick = kept[0][b, :int(kept[2][b])].cpu().numpy()
            assert np.array_equal(wt[b, :, :len(pick)].cpu().numpy(), w[b][:, pick]) and not wt[b, :, len(pick):].any()
