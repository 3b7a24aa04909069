"""A case of the 4-bit attention whose only inexact part is the softmax and the product with the values, so that an error of a few float32 roundings shows.

Keys have one value, queries one, at the same place: a logit is one exact product.  A few live tokens stand among dead ones, whose logits lie millions of powers of two
below and whose weights are exactly zero, so hardly anything is added up.  Values are positive: nothing cancels."""
from __future__ import annotations

import math

import numpy as np

EPS = 2.0 ** -24                # of a float32 operation, at most
SEEDS = (1, 2, 3)
AT = 37                         # the place of a key's and a query's one value

# Relative to out (values are positive), in EPS.  A weight: the argument is d scale - ref in one fused operation, with |d scale| at most .6, scale off by 3 (two constants and
# their product), the reference a whole number at most 1 above: ln 2 (3 * .6 + 2) and 2 of the exponential = 4.7.  Adding up: 3 of a column's sum, 2 of the terms, and per joining
# (wavefronts, splits) 2 of the factor (a power of two by the same instruction) and 4, at most, of the sum = 17; the denominator as many; its reciprocal and the product 3.
BOUND = (2 * 4.7 + 2 * 17 + 3) * EPS


def case(seed, G, T, live):
    """(q [G, 128], keys [T, 128], values [T, 128]) as float64 that bfloat16 and the 4-bit format hold exactly; live: the tokens that weigh something."""
    r = np.random.default_rng([seed, G])
    q = np.zeros((G, 128))
    q[:, AT] = np.round(r.uniform(0.35, 0.75, size=G) * 256) / 256
    K = np.zeros((T, 128))
    K[:, AT] = -6.0 * 2.0 ** 24
    K[live, AT] = r.choice([0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], size=len(live), replace=False)
    V = r.choice([1.0, 1.5, 2.0, 3.0, 4.0, 6.0], size=(T, 128))
    return q, K, V


def weights(q, K):
    """The softmax's numerators as float32 has them at best, relative to a whole power of two not below the largest."""
    x = (q[:, AT:AT + 1] * K[None, :, AT]) / math.sqrt(128) * math.log2(math.e)
    return np.exp2(x - np.ceil(x.max(axis=1, keepdims=True))).astype(np.float32)


def terms(p, n):
    """The sum of the first n of a float32's terms of eight bits, each the upper half of what those before have left."""
    total, left = np.zeros(p.shape), p.astype(np.float32).copy()
    for _ in range(n):
        t = (left.view(np.uint32) & np.uint32(0xffff0000)).view(np.float32)
        total += t
        left = left - t
    return total
