"""Sequences that share a prefix, are copied, are cut back, or are stored from projections: in 64 bits on the CPU, from the definitions, over the references of block_cache_ref."""
from __future__ import annotations

import numpy as np

from block_cache_ref import Ref, TB


def joined(prefix: Ref, own: Ref) -> Ref:
    """The sequences of `own` with their prefixes' tokens in front."""
    r = Ref(own.B, own.Hq, own.Hkv, own.D, prefix.Ncap + own.Ncap, own.dtype)
    for b in range(own.B):
        for h in range(own.Hkv):
            r.tokens[b][h] = [np.concatenate([prefix.tokens[b // (own.B // prefix.B)][h][side], own.tokens[b][h][side]]) for side in (0, 1)]
    return r


def cut(ref: Ref, b: int, L: int) -> None:
    """Sequence b to its first L tokens: a block that is cut keeps its values."""
    for h in range(ref.Hkv):
        ref.tokens[b][h] = [x[:L] for x in ref.tokens[b][h]]
        ref.exps[b][h] = [e[:L // TB] for e in ref.exps[b][h]]
        ref.score[b][h] = ref.score[b][h][:L]


def fork(src: Ref, dst: Ref, parents, upto) -> None:
    for j in range(dst.B):
        a = j if parents is None else parents[j]
        if not 0 <= a < src.B:
            continue
        L = src.len(a) if upto is None else min(src.len(a), max(upto[j], 0))
        if L > dst.Ncap:
            dst.refused += 1
            continue
        for h in range(src.Hkv):
            dst.tokens[j][h] = [x.copy() for x in src.tokens[a][h]]
            dst.exps[j][h] = [list(e) for e in src.exps[a][h]]
            dst.score[j][h] = src.score[a][h].copy()
        cut(dst, j, L)


def turned(x, places, inv_freq, weight, eps, pairs):
    """x float64 [n, H, D], its tokens' places, frequencies float64 [rot / 2], weight [D] or None -> (normed and turned, sum of the magnitudes of the two addends)."""
    x = x.copy()
    if weight is not None:
        x = x / np.sqrt((x * x).mean(axis=2, keepdims=True) + eps) * weight
    half = len(inv_freq)
    u = np.asarray(places, dtype=np.float64)[:, None, None] * inv_freq[None, None, :]
    a_at, b_at = (np.arange(half) * 2, np.arange(half) * 2 + 1) if pairs else (np.arange(half), np.arange(half) + half)
    a, b = x[:, :, a_at], x[:, :, b_at]
    size = np.abs(x)
    size[:, :, a_at] = size[:, :, b_at] = np.abs(a) + np.abs(b)
    x[:, :, a_at], x[:, :, b_at] = a * np.cos(u) - b * np.sin(u), a * np.sin(u) + b * np.cos(u)
    return x, size
