"""The bound of the 4-bit attention's exact-logit cases: weights in three terms keep it with room to spare, weights in two do not."""
import numpy as np
import pytest

from oracle import cache4_oracle as c4
from tests import cache4_terms as ct


@pytest.mark.parametrize("G", range(1, 9))
def test_a_missing_term_breaks_the_bound(G):
    seen = np.zeros(G)
    for seed in ct.SEEDS:
        q, K, V = ct.case(seed, G, 300, [3, 40, 130, 299])
        some = [0, 3, 40, 130, 299]
        assert np.array_equal(c4.unpack(c4.pack(K[some])), K[some]) and np.array_equal(c4.unpack(c4.pack(V[some])), V[some])
        ref, _, size, _ = c4.attend(q, K, V, np.arange(300))
        assert np.allclose(ref, size, rtol=1e-12)           # nothing cancels
        p = ct.weights(q, K)
        assert np.count_nonzero(p) == 4 * G
        den = p.astype(np.float64).sum(axis=1, keepdims=True)
        off = [np.abs(ct.terms(p, n) @ V / den - ref) / ref for n in (1, 2, 3)]
        assert off[2].max() < 0.2 * ct.BOUND and off[0].min() > ct.BOUND
        seen = np.maximum(seen, off[1].max(axis=1))
    assert np.all(seen > 2 * ct.BOUND)                      # of every head, with one seed or another


def test_three_terms_are_the_value():
    p = np.random.default_rng(0).random(10000).astype(np.float32)
    assert np.array_equal(ct.terms(p, 3), p.astype(np.float64))
