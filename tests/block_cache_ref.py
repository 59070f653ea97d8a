"""The block-scaled 8-bit cache in 64 bits on the CPU, written from its definition: e4m3 numbers found in the table of all of them, one power of two
per block and side, the last incomplete block in 16 bits; causal attention over it; eviction.  Shares nothing with the library."""
from __future__ import annotations

import numpy as np
import torch

TB = 64
E4M3 = np.array([(c & 7) / 8 * 2.0 ** -6 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)])
LARGEST = {torch.float16: 65504.0, torch.bfloat16: (2 - 2.0 ** -7) * 2.0 ** 127}


def scale_exponent(top: float) -> int:
    e = -100
    while top > 448.0 * 2.0 ** e:
        e += 1
    return e


def round_block(x: np.ndarray, dtype) -> tuple[np.ndarray, int]:
    """float64 [64, D] -> (the values the block stands for, e)."""
    finite = np.isfinite(x)
    e = scale_exponent(np.abs(np.where(finite, x, 0.0)).max())
    a = np.abs(np.where(finite, x, 0.0)) * 2.0 ** -e
    hi = np.searchsorted(E4M3, a).clip(0, 126)          # first number not below
    lo = np.maximum(hi - 1, 0)
    up, down = E4M3[hi] - a, a - E4M3[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(E4M3[code] * 2.0 ** e > LARGEST[dtype], code - 1, code)
    return np.where(finite, np.copysign(E4M3[code] * 2.0 ** e, x), np.nan), e


class Ref:
    """One cache: the raw tokens of the incomplete block and the values of the complete ones, per (sequence, KV head)."""

    def __init__(self, B, Hq, Hkv, D, Ncap, dtype):
        self.B, self.Hq, self.Hkv, self.D, self.Ncap, self.dtype = B, Hq, Hkv, D, Ncap, dtype
        self.tokens = [[[np.zeros((0, D)), np.zeros((0, D))] for _ in range(Hkv)] for _ in range(B)]
        self.exps = [[[[], []] for _ in range(Hkv)] for _ in range(B)]
        self.score = [[np.zeros(0) for _ in range(Hkv)] for _ in range(B)]
        self.refused = 0

    def len(self, b):
        return len(self.tokens[b][0][0])

    def append(self, k, v, n_new=None):
        k, v = k.double().cpu().numpy(), v.double().cpu().numpy()
        n = k.shape[2]
        for b in range(self.B):
            m = n if n_new is None else min(max(int(n_new[b]), 0), n)
            if self.len(b) + m > self.Ncap:
                self.refused += 1
                continue
            for h in range(self.Hkv):
                self._add(b, h, k[b, h, :m], v[b, h, :m])
                self.score[b][h] = np.concatenate([self.score[b][h], np.zeros(m)])

    def _add(self, b, h, k, v):
        for side, x in enumerate((k, v)):
            t = np.concatenate([self.tokens[b][h][side], x])
            for blk in range(len(self.exps[b][h][side]), len(t) // TB):
                t[blk * TB:(blk + 1) * TB], e = round_block(t[blk * TB:(blk + 1) * TB], self.dtype)
                self.exps[b][h][side].append(e)
            self.tokens[b][h][side] = t

    def values(self, side):
        """[B, Hkv, Ncap, D], zeros behind the lengths."""
        out = np.zeros((self.B, self.Hkv, self.Ncap, self.D))
        for b in range(self.B):
            for h in range(self.Hkv):
                out[b, h, :self.len(b)] = self.tokens[b][h][side]
        return out

    def attention(self, q, n_q=None, scale=0.0, accumulate=False):
        """q [B, Hq, n, D] -> (out, bound of the error of a 32-bit computation of it relative to sum p|v|, sum p|v|), rows behind n_q NaN."""
        q = q.double().cpu().numpy()
        n, G = q.shape[2], self.Hq // self.Hkv
        scale = scale if scale > 0 else 1 / np.sqrt(self.D)
        out, eps, mag = (np.full(q.shape, np.nan) for _ in range(3))
        for b in range(self.B):
            L, m = self.len(b), n if n_q is None else min(max(int(n_q[b]), 0), n)
            for h in range(self.Hkv):
                K, V = self.tokens[b][h]
                for g in range(G):
                    hq = h * G + g
                    seen = np.arange(L)[None, :] <= L - m + np.arange(m)[:, None]
                    x = q[b, hq, :m] @ K.T * scale
                    top = np.where(seen, x, -np.inf).max(axis=1, initial=-np.inf)
                    top = np.where(np.isfinite(top), top, 0.0)
                    p = np.where(seen, np.exp(np.where(seen, x - top[:, None], 0.0)), 0.0)
                    p /= np.maximum(p.sum(axis=1, keepdims=True), 1e-300)
                    out[b, hq, :m], mag[b, hq, :m] = p @ V, p @ np.abs(V)
                    # a score: D products summed in 32 bits (D 2^-24 of their magnitudes), scaled, the maximum subtracted (2^-23 each); the weight:
                    # that, and its exponential (2^-22); twice (weight, sum), and the two sums of t addends, 16 per step
                    size = np.where(seen, np.abs(q[b, hq, :m]) @ np.abs(K).T, 0.0).max(axis=1, initial=0.0)
                    ex = scale * self.D * 2.0 ** -24 * size + 2.0 ** -22 * np.where(seen, np.abs(x), 0.0).max(axis=1, initial=0.0) + 2.0 ** -22
                    eps[b, hq, :m] = (2 * ex + (seen.sum(axis=1) / 16 + 64) * 2.0 ** -23)[:, None]
                    if accumulate:
                        self.score[b][h] += p.sum(axis=0)
        return out, eps, mag

    def evict(self, keep, recent):
        """-> (the cache that keeps the best, kept places [B, Hkv, keep])."""
        new = Ref(self.B, self.Hq, self.Hkv, self.D, self.Ncap, self.dtype)
        kept = np.full((self.B, self.Hkv, keep), -1)
        for b in range(self.B):
            L, count = self.len(b), min(self.len(b), keep)
            sure = min(recent, count)
            for h in range(self.Hkv):
                s = self.score[b][h][:L - sure]
                key = [(1, 0.0) if np.isnan(x) else (0, float(x)) for x in s]
                order = sorted(range(L - sure), key=lambda t: (-key[t][0], -key[t][1], t))[:count - sure]
                at = np.array(sorted(order) + list(range(L - sure, L)), dtype=int)
                kept[b, h, :count] = at
                new._add(b, h, self.tokens[b][h][0][at], self.tokens[b][h][1][at])
                new.score[b][h] = self.score[b][h][at]
        return new, kept


def assert_same_tokens(A, cache, ref, what=""):
    """The library's values, exponents and lengths are the reference's, exactly."""
    k, v = A.akb_unpack(cache)
    lens = cache.lens.cpu().numpy()
    assert lens.tolist() == [ref.len(b) for b in range(ref.B)], what
    for side, got in enumerate((k, v)):
        want = ref.values(side)
        got = got.double().cpu().numpy()[:, :, :ref.Ncap]
        bad = ~((got == want) | (np.isnan(got) & np.isnan(want)))
        assert not bad.any(), f"{what}: {'KV'[side]} differs at {np.argwhere(bad)[:4].tolist()}: {got[bad][:4]} for {want[bad][:4]}"
    exps = cache.exps.cpu().numpy().reshape(ref.B, ref.Hkv, -1, 2)
    for b in range(ref.B):
        for h in range(ref.Hkv):
            for side in (0, 1):
                want = ref.exps[b][h][side]
                assert exps[b, h, :len(want), side].tolist() == want, f"{what}: exponents of {b}, {h}"


def assert_attention(out, ref_out, eps, mag, dtype, what=""):
    """out against the 64-bit result.  32-bit results: eps, and the weights as two 16-bit numbers (half a step of the second: 2^-16 in bfloat16, 2^-22
    in fp16).  16-bit results: a weight is off by half a step of the type, and the result once more."""
    got = out.double().cpu().numpy()
    half = float(torch.finfo(dtype).eps) / 2
    bound = eps * mag + (half ** 2 * mag if out.dtype == torch.float32 else half * mag + half * np.abs(ref_out)) + 1e-30
    if dtype == torch.float16:   # numbers below 2^-14 have fixed steps: half of 2^-24 in a 16-bit result
        bound = bound + (2.0 ** -25 if out.dtype == torch.float16 else 0.0)
    rows = ~np.isnan(ref_out)
    err = np.abs(got - ref_out)[rows]
    assert np.isfinite(got[rows]).all(), f"{what}: not finite"
    worst = float((err / bound[rows]).max()) if err.size else 0.0
    print(f"    {what}: worst error {worst:.3f} of its bound", flush=True)
    assert worst <= 1.0, f"{what}: {worst} of the bound"


def tokens(B, H, n, D, dtype, seed, kind="scales"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(B, H, n, D, generator=g)
    if kind == "scales":
        x = x * torch.pow(10.0, torch.rand(1, H, 1, D, generator=g) * 2 - 1)
    elif kind == "wide":   # every magnitude of the type, zeros among them
        x = x * torch.exp2(torch.rand(B, H, n, D, generator=g) * (40 if dtype == torch.float16 else 200) - (25 if dtype == torch.float16 else 120))
        x[torch.rand(x.shape, generator=g) < 0.02] = 0
    return x.clamp(-LARGEST[dtype], LARGEST[dtype]).to(dtype)
