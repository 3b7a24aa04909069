"""Set-up shared by the GPU tests of the 4-bit cache and of the eviction."""
from __future__ import annotations

import math

import numpy as np
import torch

import lc_workloads as wl
from oracle import cache4_oracle as c4
from paper_2603_08453_amd import binding as lc

D = 128


def to_dev(bits):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16).cuda()


def bf16_bits(r, *shape, scale=1.0):
    return wl.f32_to_bf16_bits((r.standard_normal(shape) * scale).astype(np.float32))


def cut(r, n, lo, hi):
    """Chunk boundaries of at most n tokens; what is left over is the open tail."""
    c = np.cumsum(r.integers(lo, hi + 1, size=max(1, n // lo)))
    return np.concatenate([[0], c[c <= n]]).astype(np.int64)


class Cache:
    """A batch with its bfloat16 and its 4-bit cache and an index over the former.  lens, bounds: per sequence.  layout: of the 4-bit cache."""

    def __init__(self, seed, H, G, lens, bounds, extra=0, splits=0, layout="bhtr", k_scale=1.0, v_scale=1.0, levels=2, fanout=4, sink=0, extra_chunks=0, geometry=0):
        r = np.random.default_rng(seed)
        self.r, self.H, self.G, self.B, self.lens, self.bounds = r, H, G, len(lens), list(lens), [np.asarray(b) for b in bounds]
        B, Tc = self.B, max(lens) + extra
        self.Tc = Tc
        self.kb = [bf16_bits(r, H, n, D, scale=k_scale) for n in lens]
        self.vb = [bf16_bits(r, H, n, D, scale=v_scale) for n in lens]
        self.K = torch.zeros(B, H, max(Tc, 1), D, dtype=torch.bfloat16, device="cuda")
        self.V = torch.zeros_like(self.K)
        for b, n in enumerate(lens):
            self.K[b, :, :n] = to_dev(self.kb[b])
            self.V[b, :, :n] = to_dev(self.vb[b])
        most = max(1, max(len(b) - 1 for b in self.bounds)) + extra_chunks
        self.cfg = lc.lc_config_default(levels=levels, fanout=fanout, max_chunks=most, max_tokens=max(Tc, 1), decode_splits=splits, sink_tokens=sink, geometry=geometry)
        self.ws = torch.zeros(lc.lc_workspace_bytes(self.cfg, B, H * G, H), dtype=torch.uint8, device="cuda")
        self.buf = torch.zeros(lc.lc_index_bytes(self.cfg, B, H), dtype=torch.uint8, device="cuda")
        self.idx = lc.lc_build_index(self.cfg, self.K, self.lens, self.bounds, self.buf, self.ws)
        self.K4, self.V4 = (self.narrow(layout) for _ in range(2))
        lc.lc_cache4_store(self.K, self.V, self.K4, self.V4, counts=self.lens)
        torch.cuda.synchronize()

    def narrow(self, layout):
        """Rows never written hold bytes that would be seen: scales 255, no numbers."""
        B, H, T = self.B, self.H, max(self.Tc, 1)
        if layout == "bhtr":
            return torch.full((B, H, T, 68), 255, dtype=torch.uint8, device="cuda")
        if layout == "bthr":
            return torch.full((B, T, H, 68), 255, dtype=torch.uint8, device="cuda").transpose(1, 2)
        return torch.full((B, H, T, 84), 255, dtype=torch.uint8, device="cuda")[..., 4:72]      # "padded"

    def k4(self, b, h):
        return c4.unpack(self.K4[b, h, :self.lens[b]].cpu().numpy())

    def v4(self, b, h):
        return c4.unpack(self.V4[b, h, :self.lens[b]].cpu().numpy())

    def query(self, scale=1.0):
        return bf16_bits(self.r, self.B, self.H * self.G, D, scale=scale)

    def heads(self, qb, b, h):
        return wl.bf16_bits_to_f64(qb[b, h * self.G:(h + 1) * self.G])

    def lists(self, share):
        """Per (sequence, head) an ascending list of about `share` of the chunks."""
        return [[np.flatnonzero(self.r.random(len(self.bounds[b]) - 1) < share) for _ in range(self.H)] for b in range(self.B)]

    def table(self, ids, cap=None, fill=-7):
        cap = cap or max(1, max(len(i) for row in ids for i in row))
        t = np.full((self.B, self.H, cap), fill, dtype=np.int32)
        for b in range(self.B):
            for h in range(self.H):
                t[b, h, :len(ids[b][h])] = ids[b][h]
        n = np.array([[len(i) for i in row] for row in ids], dtype=np.int32).reshape(self.B, self.H)
        return torch.from_numpy(t).cuda(), torch.from_numpy(n).cuda()

    def attend(self, qb, ids, with_lse=True):
        t, n = self.table(ids)
        out = torch.full((self.B, self.H * self.G, D), float("nan"), device="cuda")
        lse = torch.full((self.B, self.H * self.G), float("nan"), device="cuda") if with_lse else None
        lc.lc_sparse_decode4(self.idx, to_dev(qb), self.K4, self.V4, t, n, out, self.ws, lse=lse)
        torch.cuda.synchronize()
        return out.cpu().numpy(), None if lse is None else lse.cpu().numpy()

    def check(self, qb, ids, out, lse, tag=""):
        for b in range(self.B):
            for h in range(self.H):
                rows = c4.active_rows(self.bounds[b], self.lens[b], ids[b][h])
                check_attention(self.heads(qb, b, h), self.k4(b, h), self.v4(b, h), rows, out[b, h * self.G:(h + 1) * self.G],
                                None if lse is None else lse[b, h * self.G:(h + 1) * self.G], (tag, b, h))


EPS = 2.0 ** -24        # of a float32 operation, at most


def check_attention(q, K, V, rows, out, lse, tag):
    """Against float64.  A logit is a sum of 128 exact products in float32: off by up to 130 EPS sum |q_i k_i| / sqrt(d) with the scaling; its
    exponential by that and the instruction's 2 EPS and those of the argument's rounding (up to 127 powers of two below the reference: 2^-17 ln 2 / 2, but only
    where it weighs 2^-127; weight times error is at most 2^-23).  Weights are relative to a sum with the same errors, and products are added up over the tokens in wavefronts and
    splits (at most 64 + 2 T / 32 / 4 roundings of partial sums: counted as 200 EPS at these sizes).  So |out - ref| <= (2 x + 2^-15) sum p |v| with x
    the logits' error, and lse is off by x + 2^-22 |lse| + 2^-18."""
    ref, ref_lse, size, prod = c4.attend(q, K, V, rows)
    x = 130 * EPS * prod
    if len(rows) == 0:
        assert not out.any() and (lse is None or np.all(lse == -math.inf)), tag
        return
    off = np.abs(out.astype(np.float64) - ref)
    assert np.all(off <= (2 * x + 2.0 ** -15) * size + 1e-30), (tag, float((off / np.maximum(size, 1e-300)).max()), x)
    if lse is not None:
        far = np.abs(lse.astype(np.float64) - ref_lse)
        assert np.all(far <= x + 2.0 ** -22 * np.abs(ref_lse) + 2.0 ** -18), (tag, float(far.max()), x)
