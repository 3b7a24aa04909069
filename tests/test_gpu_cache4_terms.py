"""The 4-bit attention's softmax and P.V alone, to a few float32 roundings: a probability's third term, its columns and their joining show here and nowhere else."""
import math

import numpy as np
import pytest

import lc_workloads as wl
from oracle import cache4_oracle as c4
from tests import cache4_terms as ct

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("G", range(1, 9))
@pytest.mark.parametrize("T,live,splits", [(300, [3, 40, 130, 299], 1), (300, [3, 40, 130, 299], 0), (20, [0, 5, 17, 19], 0), (2000, [0, 700, 1301, 1999], 9)])
def test_probabilities_to_their_last_bits(G, T, live, splits):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from tests import cache4_common as C
    lc = C.lc
    H = 2
    c = C.Cache(90, H, G, [T], [np.arange(0, T + 1, 10)], splits=splits)
    t, n = c.table([[np.arange(len(c.bounds[0]) - 1)] * H])
    for seed in ct.SEEDS:
        cases = [ct.case(seed, G, T, live), ct.case(seed + 10, G, T, live[::-1])]
        bits = [wl.f32_to_bf16_bits(np.stack([x[i] for x in cases]).astype(np.float32))[None] for i in range(3)]
        assert all(np.array_equal(wl.bf16_bits_to_f64(b[0, h]), cases[h][i]) for i, b in enumerate(bits) for h in range(H))
        lc.lc_cache4_store(C.to_dev(bits[1]), C.to_dev(bits[2]), c.K4, c.V4)
        out, lse = torch.zeros(1, H * G, 128, device="cuda"), torch.zeros(1, H * G, device="cuda")
        lc.lc_sparse_decode4(c.idx, C.to_dev(bits[0].reshape(1, H * G, 128)), c.K4, c.V4, t, n, out, c.ws, lse=lse)
        torch.cuda.synchronize()
        for h, (q, K, V) in enumerate(cases):
            ref, ref_lse, _, _ = c4.attend(q, K, V, np.arange(T))
            off = np.abs(out[0, h * G:(h + 1) * G].cpu().numpy() - ref) / ref
            assert off.max() <= ct.BOUND, (seed, h, off.max() / ct.EPS)
            # the sum's errors, the logarithm's 2 EPS and its own rounding
            far = np.abs(lse[0, h * G:(h + 1) * G].cpu().numpy() - ref_lse)
            assert np.all(far <= ct.BOUND / 2 + 4 * ct.EPS * (1 + np.abs(ref_lse))), (seed, h, far.max() / ct.EPS)
