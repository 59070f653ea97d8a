"""Tokens stored from projections in every way that a call can be shared out: row by row, query heads beside their KV head or apart, past the last-level cache, lengths moved by
tickets or by a launch behind; each type, head size and order of pairs.  All in 64 bits on the GPU; what is stored is compared byte by byte with akb_append of the keys that 64 bits
give (rounded to binary32 and then to the type, as the library does)."""
import numpy as np
import pytest
import torch

import block_cache_ref as R
from test_gpu_block_cache import A, B16, DEV, F16, i32  # noqa: F401
from test_gpu_block_cache_rotated import freqs, projected, weight

pytestmark = pytest.mark.gpu
LENS = [0, 63, 64, 130, 5, 100, 191]

PATHS = [  # dtype, D, sequences, Hq, Hkv, n, ragged, rot, norm, pairs
    # past the last-level cache, every kernel of it
    (F16, 128, 4, 32, 8, 1700, True, 128, True, False),
    (F16, 128, 4, 32, 8, 1700, False, 64, True, True),
    (B16, 128, 4, 32, 8, 1700, False, 128, True, False),
    (B16, 128, 4, 32, 8, 1700, True, 128, False, True),
    (F16, 64, 5, 32, 8, 2800, False, 64, True, False),
    (F16, 64, 5, 32, 8, 2800, True, 32, False, True),
    (B16, 64, 5, 32, 8, 2800, True, 64, True, False),
    (B16, 64, 5, 32, 8, 2800, False, 64, True, True),
    # ... row by row (many sequences), and with query heads apart (few long ones)
    (B16, 128, 1000, 48, 8, 5, True, 128, True, False),
    (F16, 64, 1000, 96, 12, 7, True, 64, True, True),
    (F16, 128, 1, 64, 4, 4200, False, 128, True, False),
    (B16, 64, 2, 128, 8, 4000, True, 48, True, True),
    # query heads apart: groups that four do and do not divide
    *[(t, 128, 3, G * 2, 2, n, True, 128, True, p) for t, G, n, p in ((F16, 5, 9, False), (B16, 5, 70, True), (F16, 8, 70, True), (B16, 8, 200, False), (F16, 16, 200, False), (B16, 16, 9, True),
                                                                     (F16, 11, 64, False), (B16, 11, 63, True))],
    *[(t, 64, 4, G, 1, n, True, 64, True, p) for t, G, n, p in ((F16, 1, 9, False), (B16, 3, 65, True), (F16, 16, 200, True), (B16, 6, 129, False))],
    # query heads beside their KV head, though there are more than four of them or D = 64: too many workgroups
    (F16, 128, 40, 32, 4, 200, True, 128, True, False),
    (B16, 128, 70, 16, 2, 130, True, 96, True, True),
    (F16, 64, 160, 8, 4, 9, True, 64, True, True),
    (B16, 64, 100, 16, 4, 130, True, 64, True, False),
    (F16, 128, 7, 8, 2, 100, True, 128, True, False),
    (B16, 128, 3, 4, 4, 9, True, 128, False, True),
    # row by row, lengths by tickets and by a launch behind
    (F16, 128, 3, 8, 2, 8, True, 128, True, False),
    (B16, 64, 3, 6, 2, 1, False, 64, True, True),
    (B16, 128, 200, 16, 4, 3, True, 128, True, True),
    (F16, 64, 800, 4, 2, 1, False, 64, True, False),
]


def turned(x, places, freq, w, eps, pairs):
    """x float64 [B, n, H, D] at places [B, n] -> (normed and turned, sum of the magnitudes of the two addends)."""
    if w is not None:
        x = x / torch.sqrt((x * x).mean(dim=3, keepdim=True) + eps) * w.double()
    if freq is None:
        return x, x.abs()
    half = freq.numel()
    u = (places.double()[:, :, None] * freq.double())[:, :, None]
    j = torch.arange(half, device=DEV)
    a_at, b_at = (2 * j, 2 * j + 1) if pairs else (j, j + half)
    a, b, size, y = x[..., a_at], x[..., b_at], x.abs(), x.clone()
    size[..., a_at] = size[..., b_at] = a.abs() + b.abs()
    y[..., a_at], y[..., b_at] = a * u.cos() - b * u.sin(), a * u.sin() + b * u.cos()
    return y, size


@pytest.mark.parametrize("case", PATHS, ids=lambda c: f"{str(c[0])[6:]}-D{c[1]}-B{c[2]}-H{c[3]}_{c[4]}-n{c[5]}-rot{c[7]}-norm{int(c[8])}-pairs{int(c[9])}")
@pytest.mark.parametrize("queries", [True, False], ids=["", "keys"])
def test_every_way_to_share_out_a_call(A, case, queries):
    """Queries, with u = 2^-24, relative to the sum of the addends' magnitudes: the root is of a sum of D squares (a lane's eight, each one rounding, and up to four sums
    of lanes), the mean with eps (one more): 13 u, halved by the root, which is itself within 2 u (one unit in the last place): 8.5 u.  Sine and cosine rounded to binary32 and times
    a weight, the channel times the root, their product, the sum: 5 u.  13.5 u, below the 16 u = 2^-20 that is allowed.  Then half a step of the type."""
    dtype, D, B, Hq, Hkv, n, ragged, rot, norm, pairs = case
    print(case, flush=True)
    lens = [LENS[b % len(LENS)] for b in range(B)]
    n_new = [(n, max(1, n // 3), n - 1, min(n, 64 - lens[b] % 64), 0)[b % 5] for b in range(B)] if ragged else [n] * B
    base = [1000 + 7 * b for b in range(B)] if B % 2 else [32768]
    cap = (max(LENS) + n + 63) // 64 * 64
    c, d = (A.BlockCache.allocate(B, Hq, Hkv, D, cap, dtype, score=True) for _ in range(2))
    first = [R.tokens(B, Hkv, max(LENS), D, dtype, s, "plain").to(DEV) for s in (1, 2)]
    for cache in (c, d):
        A.akb_append(cache, *first, i32(lens))
        cache.score.fill_(7.0)
    q, k, v = projected(B, n, Hq, Hkv, D, dtype, 11, B % 2 == 0)
    freq, qw, kw, eps = freqs(rot), weight(D, dtype, 1) if norm else None, weight(D, dtype, 2) if norm else None, 1e-5
    start = torch.full((B, Hq, n, D), 5.0, dtype=dtype, device=DEV)
    taken = torch.arange(n, device=DEV) < i32(n_new)[:, None]
    for t in (q, k, v):   # rows that are not taken may hold anything
        t.masked_fill_(~taken[:, :, None, None], float("nan"))
    out = A.akb_append_rotated(c, q if queries else None, k, v, start if queries else None, inv_freq=freq, n_new=i32(n_new) if ragged else None, q_norm=qw, k_norm=kw, eps=eps,
                               pairs=pairs, base=i32(base))
    places = (i32(lens) + i32(base).repeat_interleave(B // len(base)))[:, None] + torch.arange(n, device=DEV)
    eps = float(np.float32(eps))
    keys, _ = turned(k.double(), places, freq, kw, eps, pairs)
    A.akb_append(d, keys.float().to(dtype).transpose(1, 2).contiguous(), v.transpose(1, 2).contiguous(), i32(n_new))
    del keys
    assert c.lens.tolist() == [x + y for x, y in zip(lens, n_new)] == d.lens.tolist()
    for got, want in zip(A.akb_unpack(c), A.akb_unpack(d)):
        assert torch.equal(got, want)
    whole = torch.arange(cap // 64, device=DEV) < (c.lens // 64)[:, None]
    exps = [x.exps.view(B, Hkv, cap // 64, 2).masked_fill(~whole[:, None, :, None], 0) for x in (c, d)]
    assert torch.equal(*exps) and torch.equal(c.score, d.score) and not c.flags.any()
    if not queries:
        assert out is None
        return
    half = float(torch.finfo(dtype).eps) / 2
    out = out.transpose(1, 2)
    for b in range(0, B, max(1, B // 8)):
        m = n_new[b]
        assert (out[b, m:].float() == 5.0).all()
        want, size = turned(q[b:b + 1, :m].double(), places[b:b + 1, :m], freq, qw, eps, pairs)
        bound = half * want.abs() + 2.0 ** -20 * size * (1 + half) + (2.0 ** -25 if dtype == F16 else 1e-38)
        err = (out[b, :m].double() - want[0]).abs() / bound[0]
        assert not m or float(err.max()) <= 1.0, (b, float(err.max()))


@pytest.mark.parametrize("D,pairs,n", [(128, False, 3), (128, True, 70), (64, False, 70), (64, True, 3), (128, False, 200)])
def test_norm_weights_of_every_size(A, D, pairs, n):
    """bfloat16 weights from 2^-100 to 2^100 on heads from 2^-48 to 2^58: a channel times its weight is beyond binary32 on either side where the normed number times it is not."""
    g = torch.Generator().manual_seed(5)
    H = 8
    sizes = torch.exp2(torch.tensor([-48.0, -40, -20, 0, 20, 40, 50, 58])).view(1, 1, H, 1)
    x = (torch.randn(2, n, H, D, generator=g) * sizes).to(B16).to(DEV)
    w = (torch.exp2(torch.rand(D, generator=g) * 200 - 100) * torch.where(torch.rand(D, generator=g) < 0.5, -1.0, 1.0)).to(B16).to(DEV)
    w[D // 3:D // 3 + 9] = 1.0   # and some that are not
    freq, eps = freqs(D), 1e-37
    c, d = (A.BlockCache.allocate(2, H, H, D, 256, B16) for _ in range(2))
    out = A.akb_append_rotated(c, x, x, x, inv_freq=freq, q_norm=w, k_norm=w, eps=eps, pairs=pairs)
    want, size = turned(x.double(), torch.arange(n, device=DEV).expand(2, n), freq, w, float(np.float32(eps)), pairs)
    A.akb_append(d, want.float().to(B16).transpose(1, 2).contiguous(), x.transpose(1, 2).contiguous())
    for got, stored in zip(A.akb_unpack(c), A.akb_unpack(d)):
        assert torch.equal(got, stored)
    half = 2.0 ** -8
    err = (out.transpose(1, 2).double() - want).abs() / (half * want.abs() + 2.0 ** -20 * size * (1 + half) + 1e-38)
    worst, finite = float(err.max()), bool(torch.isfinite(out).all())
    assert finite and worst <= 1.0, worst
