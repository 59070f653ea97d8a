"""Tokens stored from projections, on the GPU: queries within the bound that their arithmetic gives, keys equal to the 64-bit results rounded once, stored as akb_append
stores them."""
import numpy as np
import pytest
import torch

import block_cache_ref as R
import block_cache_share_ref as S
from test_gpu_block_cache import A, B16, DEV, F16, i32, pair, put  # noqa: F401

pytestmark = pytest.mark.gpu


def projected(B, n, Hq, Hkv, D, dtype, seed, packed, kind="scales"):
    x = R.tokens(B, Hq + 2 * Hkv, n, D, dtype, seed, kind).transpose(1, 2).contiguous().to(DEV)
    parts = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
    return parts if packed else tuple(t.contiguous() for t in parts)


def freqs(rot, theta=10000.0):
    return (theta ** -(torch.arange(rot // 2, dtype=torch.float64) / max(1, rot // 2))).float().to(DEV) if rot else None


def weight(D, dtype, seed):
    return (1 + 0.3 * torch.randn(D, generator=torch.Generator().manual_seed(seed))).to(dtype).to(DEV)


def check_turned(got, x, places, freq, w, eps, pairs, dtype, what=""):
    """got [H, m, D] against x [m, H, D] in 64 bits.  A result is rounded once (half a step).  Before that, relative to the addends' magnitudes: the root
    (its argument, itself, its inverse: 3 x 2^-24), the two products of the norm (2 x 2^-24), sine and cosine (the angle's rounding 2^-25, the series' seven roundings of
    parts below one half of the result, 2^-23 together), the product and the sum (2 x 2^-24): below 12 x 2^-24 < 2^-20."""
    f = np.zeros(0) if freq is None else freq.double().cpu().numpy()
    want, size = S.turned(x.double().cpu().numpy(), places, f, None if w is None else w.double().cpu().numpy(), eps, pairs)
    half = float(torch.finfo(dtype).eps) / 2
    g = got.double().cpu().numpy().transpose(1, 0, 2)
    bound = half * np.abs(want) + 2.0 ** -20 * size * (1 + half) + (2.0 ** -25 if dtype == F16 else 1e-38)
    if w is None and freq is None:
        bound = 0 * bound
    err = np.abs(g - want)
    assert (err <= bound).all(), f"{what}: {float((err / np.maximum(bound, 1e-300)).max())} of its bound at {np.argwhere(err > bound)[:3].tolist()}"


CASES = [  # dtype, D, Hq, Hkv, rot, norm, pairs, packed, lengths before, n, n_new, base
    (B16, 128, 8, 2, 128, True, False, True, [0, 63, 64, 130], 1, None, None),
    (F16, 128, 4, 4, 128, True, False, False, [5, 62], 3, [3, 2], [1000]),
    (F16, 64, 5, 1, 64, True, True, True, [100, 0, 10], 70, [70, 64, 0], [7, 0, 90000]),
    (B16, 64, 16, 1, 32, False, True, False, [60, 1], 200, None, [3000]),
    (B16, 128, 12, 4, 64, False, False, True, [0, 127], 333, [333, 129], None),
    (F16, 128, 2, 2, 16, True, False, True, [64], 64, None, None),
    (F16, 64, 4, 2, 48, True, False, True, [31, 70], 130, [97, 130], [5, 6]),       # a rotation that ends inside an octet's mirror image
    (B16, 128, 4, 1, 0, True, False, True, [33], 100, None, None),                   # norms alone
    (F16, 128, 4, 2, 0, False, False, False, [33, 64, 0], 130, [31, 128, 130], None),   # nothing but the order
    (B16, 64, 2, 2, 64, True, True, True, [1], 1, None, [0]),
    (F16, 128, 32, 2, 112, True, True, True, [10, 20], 6, [6, 0], [1 << 21]),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{str(c[0])[6:]}-D{c[1]}-H{c[2]}_{c[3]}-rot{c[4]}-norm{int(c[5])}-pairs{int(c[6])}-packed{int(c[7])}-n{c[9]}")
def test_append_rotated(A, case):
    dtype, D, Hq, Hkv, rot, norm, pairs, packed, lens, n, n_new, base = case
    B, Ncap, eps = len(lens), max(lens) // 64 * 64 + (n + 127) // 64 * 64, 1e-5
    c, ref = pair(A, B, Hq, Hkv, D, Ncap, dtype, score=True)
    put(A, c, ref, max(max(lens), 1), 3, lens)
    c.score.fill_(7.0)
    q, k, v = projected(B, n, Hq, Hkv, D, dtype, 11, packed)
    if n_new is not None:   # rows that are not taken may hold anything
        for b, m in enumerate(n_new):
            for t in (q, k, v):
                t[b, m:] = float("nan")
    freq, qw, kw = freqs(rot), weight(D, dtype, 1) if norm else None, weight(D, dtype, 2) if norm else None
    more = dict(inv_freq=freq, eps=eps, pairs=pairs, base=i32(base), n_new=i32(n_new))
    turned_k = torch.zeros(B, Hkv, n, D, dtype=dtype)
    start = torch.full((B, Hq, n, D), 5.0, dtype=dtype, device=DEV)
    out = A.akb_append_rotated(c, q, k, v, start, q_norm=qw, k_norm=kw, **more)
    assert out is start
    for b in range(B):
        m = n if n_new is None else n_new[b]
        first = lens[b] + (0 if base is None else base[b // (B // len(base))])
        check_turned(out[b, :, :m], q[b, :m], range(first, first + m), freq, qw, float(np.float32(eps)), pairs, dtype, f"q {b}")
        exact, _ = S.turned(k[b, :m].double().cpu().numpy(), range(first, first + m), np.zeros(0) if freq is None else freq.double().cpu().numpy(),
                            kw.double().cpu().numpy() if norm else None, float(np.float32(eps)), pairs)
        turned_k[b, :, :m] = torch.from_numpy(exact.transpose(1, 0, 2).copy()).float().to(dtype)
        assert (out[b, :, m:].float() == 5.0).all()
    ref.append(turned_k, v.transpose(1, 2), n_new)
    R.assert_same_tokens(A, c, ref)
    score = c.score.view(B, Hkv, Ncap).cpu()
    for b in range(B):
        assert (score[b, :, :lens[b]] == 7.0).all() and not score[b, :, lens[b]:ref.len(b)].any() and (score[b, :, ref.len(b):] == 7.0).all()
    assert not c.flags.any()
    for m in (1, 64):   # and it goes on
        put(A, c, ref, m, 30 + m) if ref.len(0) + m <= Ncap and max(ref.len(b) for b in range(B)) + m <= Ncap else None
    R.assert_same_tokens(A, c, ref)


@pytest.mark.parametrize("dtype", [F16, B16], ids=["fp16", "bf16"])
def test_far_places(A, dtype):
    """Places up to 2^31: the angle is made in 64 bits."""
    base = [0, 1 << 20, (1 << 22) - 1, 99999999, (1 << 31) - 200]
    c, _ = pair(A, 5, 4, 2, 64, 128, dtype)
    q, k, v = projected(5, 40, 4, 2, 64, dtype, 3, True, "plain")
    freq = torch.cat([freqs(62, 500000.0), torch.tensor([0.7390851], device=DEV)])
    out = A.akb_append_rotated(c, q, k, v, inv_freq=freq, base=i32(base))
    for b in range(5):
        check_turned(out[b], q[b], range(base[b], base[b] + 40), freq, None, 0.0, False, dtype, f"base {base[b]}")


@pytest.mark.parametrize("dtype", [F16, B16], ids=["fp16", "bf16"])
def test_norms_of_small_and_large_heads(A, dtype):
    """Heads of the smallest and largest numbers of the type, whose squares 32 bits cannot hold, and of zeros."""
    top, low = R.LARGEST[dtype], 2.0 ** -24 if dtype == F16 else 2.0 ** -133
    x = torch.randn(1, 8, 2, 128, generator=torch.Generator().manual_seed(1)).double()
    sizes = torch.tensor([0.0, low, low * 2 ** 9, 1e-4, 1.0, 300.0, top / 8, top / 64], dtype=torch.float64)
    x = (x * sizes.view(1, 8, 1, 1)).clamp(-top, top).to(dtype).to(DEV)
    c, _ = pair(A, 1, 2, 2, 128, 64, dtype)
    w = weight(128, dtype, 4)
    for eps in (1e-6, 1e-30):
        c.lens.zero_()
        out = A.akb_append_rotated(c, x, x, x, inv_freq=freqs(128), q_norm=w, k_norm=w, eps=eps)
        check_turned(out[0], x[0], range(8), freqs(128), w, float(np.float32(eps)), False, dtype, f"eps {eps}")


def test_refused_sequences_and_missing_queries(A):
    c, ref = pair(A, 4, 4, 2, 128, 128, F16, score=True)
    put(A, c, ref, 128, 1, [100, 128, 0, 64])
    q, k, v = projected(4, 65, 4, 2, 128, F16, 5, True)
    n_new = [29, 1, 65, 64]
    start = torch.full((4, 4, 65, 128), 5.0, dtype=F16, device=DEV)
    out = A.akb_append_rotated(c, q, k, v, start, inv_freq=freqs(128), n_new=i32(n_new))
    assert c.lens.tolist() == [100, 128, 65, 128] and c.flags.cpu().tolist() == [2, 0, 0, 0] + [0] * 4
    assert (out[:2] == 5.0).all()
    for b, first in ((2, 0), (3, 64)):
        check_turned(out[b, :, :n_new[b]], q[b, :n_new[b]], range(first, first + n_new[b]), freqs(128), None, 0.0, False, F16, f"{b}")
    d, _ = pair(A, 4, 4, 2, 128, 128, F16)
    put(A, d, R.Ref(4, 4, 2, 128, 128, F16), 128, 1, [100, 128, 0, 64])
    assert A.akb_append_rotated(d, None, k, v, inv_freq=freqs(128), n_new=i32(n_new)) is None
    assert all(torch.equal(x, y) for x, y in zip(A.akb_unpack(c), A.akb_unpack(d)))
    before = [t.clone().view(torch.uint8) for t in (d.lens, d.k8, d.k_tail)]   # (bits: the tail holds NaN)
    A.akb_append_rotated(d, None, k[:, :0], v[:, :0], inv_freq=freqs(128))
    assert all(torch.equal(x, y.view(torch.uint8)) for x, y in zip(before, (d.lens, d.k8, d.k_tail)))


def test_what_is_not_finite_stays_in_its_head(A):
    c, _ = pair(A, 1, 2, 2, 64, 128, B16)
    x = R.tokens(1, 2, 3, 64, B16, 5, "plain").transpose(1, 2).contiguous()
    clean = x.clone()
    x[0, 1, 0, 3], x[0, 1, 1, 40] = float("nan"), float("inf")
    out = A.akb_append_rotated(c, x.to(DEV), clean.to(DEV), clean.to(DEV), inv_freq=freqs(32))[0].float().cpu()
    bad = ~torch.isfinite(out)
    want = torch.zeros_like(bad)
    want[0, 1, 3] = want[0, 1, 19] = want[1, 1, 40] = True   # channel 3 turns with 19; channel 40 does not turn
    assert torch.equal(bad, want) and out[1, 1, 40] == float("inf")


@pytest.mark.parametrize("n,B", [(1, 3), (1, 400), (130, 3), (130, 60)])
def test_in_a_graph_that_is_replayed(A, n, B):
    """With lengths moved by tickets (few workgroups) and by a launch behind (many)."""
    q, k, v = projected(B, n, 4, 2, 64, F16, 5, True)
    w, freq, base = weight(64, F16, 3), freqs(64), i32([100])
    caches = [A.BlockCache.allocate(B, 4, 2, 64, 640, F16) for _ in range(2)]
    outs = [torch.zeros(B, 4, n, 64, dtype=F16, device=DEV) for _ in range(2)]
    step = lambda i: A.akb_append_rotated(caches[i], q, k, v, outs[i], inv_freq=freq, q_norm=w, k_norm=w, base=base)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        step(0)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=s):
            step(0)
    torch.cuda.current_stream().wait_stream(s)
    caches[0].lens.zero_()
    for turn in range(3):
        graph.replay()
        step(1)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(caches[0].lens, caches[1].lens), f"replay {turn}"
        assert all(torch.equal(x, y) for x, y in zip(A.akb_unpack(caches[0]), A.akb_unpack(caches[1]))), f"replay {turn}"


@pytest.mark.parametrize("n", [3, 100])
def test_a_row_does_not_depend_on_its_neighbours(A, n):
    """Heads of zeros, of the largest numbers, and tokens that are left out change no other row's bits."""
    x = R.tokens(1, 6, n, 128, B16, 5, "plain").transpose(1, 2).contiguous().to(DEV)
    w = weight(128, B16, 3)

    def run(x, n_new=None):
        c = A.BlockCache.allocate(1, 6, 6, 128, 128, B16)
        out = A.akb_append_rotated(c, x, x, x, inv_freq=freqs(128), q_norm=w, k_norm=w, n_new=i32(n_new))
        return out, A.akb_unpack(c)[0][:, :, :n]
    want, keys = run(x)
    y = x.clone()
    y[0, 1, 2], y[0, 0, 5], y[0, 2, 0] = 0, 3e38, 1e-38
    got, _ = run(y)
    same = torch.ones(1, 6, n, dtype=torch.bool)
    same[0, 2, 1] = same[0, 5, 0] = same[0, 0, 2] = False
    assert torch.equal(got[same], want[same]) and not torch.equal(got[~same], want[~same])
    less, _ = run(x, [n - 1])
    assert torch.equal(less[:, :, :n - 1], want[:, :, :n - 1])
