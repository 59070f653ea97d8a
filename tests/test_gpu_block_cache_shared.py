"""Attention of sequences that go on from shared ones, on the GPU against the 64-bit reference of the same tokens in one cache."""
import numpy as np
import pytest
import torch

import block_cache_ref as R
import block_cache_share_ref as S
from test_gpu_block_cache import A, B16, DEV, F16, F32, i32, pair, put  # noqa: F401

pytestmark = pytest.mark.gpu


def caches(A, Bp, B, Hq, Hkv, D, P, N, dtype, first, lens, n=1, seed=1, kind="scales"):
    """A prefix cache with lengths `first` and a cache that goes on from it with lengths `lens`, and their references."""
    up = lambda x: (max(x, 1) + 63) // 64 * 64
    p, pr = pair(A, Bp, Hq, Hkv, D, up(P), dtype)
    c, cr = pair(A, B, Hq, Hkv, D, max(up(N), up(n)), dtype)
    if P:
        put(A, p, pr, P, seed, first, kind=kind)
    if N:
        put(A, c, cr, N, seed + 10, lens, kind=kind)
    c.reserve(n, prefix=p)
    return p, pr, c, cr


def check(A, p, pr, c, cr, n, n_q, out_dtype, what="", seed=9, **more):
    dtype = c.dtype
    q = R.tokens(c.B, c.Hq, n, c.D, dtype, seed, "plain")
    sent = q.clone()
    for b in range(c.B):
        sent[b, :, n if n_q is None else max(n_q[b], 0):] = float("nan")
    start = torch.full(q.shape, 5.0, dtype=out_dtype, device=DEV)
    out = A.akb_attention_shared(p, c, sent.to(DEV), start, n_q=i32(n_q), **more)
    want, eps, mag = S.joined(pr, cr).attention(q, n_q, scale=more.get("scale", 0.0))
    R.assert_attention(out, want, eps, mag, dtype, what)
    assert (out.float().cpu().numpy()[np.isnan(want)] == 5.0).all(), "rows behind n_q are as they were"
    return out


CASES = [  # dtype, out, D, Hq, Hkv, lengths of the prefixes, lengths behind them, n, n_q
    (F16, F32, 128, 4, 4, [100], [1, 63, 64, 65, 200, 0], 1, None),         # an empty sequence: its query token is the prefix's last
    (F16, F16, 128, 8, 2, [64], [1, 70], 1, None),                          # the prefix ends with a block
    (B16, F32, 128, 8, 1, [0], [1, 0, 130], 1, None),                       # no prefix at all; nothing to see
    (B16, B16, 64, 5, 1, [300, 1], [3, 80, 64, 1], 1, None),                # groups of five
    (F16, F32, 64, 16, 1, [1000, 130], [40, 500], 1, None),
    (F16, F16, 128, 32, 8, [700, 65], [5, 9, 100, 64, 1, 33, 128, 2], 1, None),
    (B16, B16, 128, 16, 2, [500], [7, 5, 70, 129, 6, 5, 64, 5], 5, None),   # drafts
    (B16, F32, 128, 8, 2, [129, 64, 3, 0], [7, 3, 70, 2, 0, 1, 9, 4], 7, [7, 5, 7, 0, 3, 7, -1, 9]),   # query tokens that stand in the prefix, or in front of it
    (F16, F32, 64, 4, 2, [200], [90, 150], 90, [90, 33]),                   # questions behind a document
    (B16, B16, 128, 4, 1, [130, 500], [300, 64, 200, 129], 200, [200, 64, 17, 129]),
    (F16, F16, 64, 10, 2, [257], [150, 90, 141], 150, [150, 90, 141]),      # groups of five, row groups that end inside a query token
    (F16, F32, 128, 3, 3, [1], [1], 1, None),
    (B16, B16, 64, 64, 4, [77], [20, 3], 20, [20, 3]),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{str(c[0])[6:]}-{str(c[1])[6:]}-D{c[2]}-H{c[3]}_{c[4]}-P{'_'.join(map(str, c[5]))}-n{c[7]}-{'_'.join(map(str, c[6]))}")
def test_shared_attention(A, case):
    dtype, out_dtype, D, Hq, Hkv, first, lens, n, n_q = case
    p, pr, c, cr = caches(A, len(first), len(lens), Hq, Hkv, D, max(first), max(lens), dtype, first, lens, n)
    check(A, p, pr, c, cr, n, n_q, out_dtype, "out")
    R.assert_same_tokens(A, p, pr, "the prefix is as it was")
    R.assert_same_tokens(A, c, cr, "the cache is as it was")


def test_every_length_around_a_block(A):
    """Prefixes of every length about a block, with few own tokens and with none."""
    for P in (1, 62, 63, 64, 65, 66, 127, 128, 129):
        p, pr, c, cr = caches(A, 1, 4, 4, 2, 64, P, 66, F16, [P], [0, 1, 64, 66], 3)
        check(A, p, pr, c, cr, 3, [1, 3, 2, 3], F32, f"P {P}")


LARGE = [  # dtype, out, D, prefixes, sequences, Hq, Hkv, P, N, n: against 64 bits on the GPU
    (F16, F32, 128, 1, 4, 32, 32, 1024, 60, 1),
    (B16, B16, 128, 1, 64, 32, 8, 9000, 700, 1),
    (F16, F16, 64, 4, 12, 40, 8, 3001, 900, 1),
    (B16, F32, 128, 2, 32, 64, 8, 5000, 300, 4),
    (F16, F32, 64, 3, 6, 16, 4, 2500, 1300, 9),
    (B16, B16, 128, 1, 3, 16, 2, 12000, 400, 300),
    (F16, F16, 128, 2, 300, 4, 4, 640, 70, 1),
    (B16, F32, 128, 1, 2, 8, 8, 700, 20000, 1),        # the own tokens are the longer part
    (B16, B16, 64, 1, 100, 16, 1, 30000, 64, 1),
    (F16, F32, 128, 1, 1, 8, 1, 66000, 500, 2),
    (F16, F16, 128, 8, 8, 12, 4, 300, 900, 100),
    (B16, F32, 128, 1, 20, 32, 8, 3500, 200, 9),       # prompt walks over the prefix, row walks over own tokens
    (F16, F16, 64, 2, 40, 40, 8, 700, 130, 7),
    (F16, F32, 64, 2, 140, 8, 8, 200, 150, 5),         # own walks by a wave alone, in one tile of rows
    (B16, B16, 128, 3, 180, 24, 8, 100, 200, 7),       # ... in two
    (B16, F32, 128, 3, 150, 32, 8, 900, 90, 4),        # prompt walks over the prefix, one tile of own rows
    (F16, F16, 64, 2, 60, 32, 8, 1200, 70, 12),        # ... two tiles
    (B16, F32, 128, 5, 125, 64, 16, 333, 10, 2),       # ... walks that are not cut
    (F16, F32, 64, 8, 560, 32, 8, 130, 66, 1),         # ... of each type and head size
    (F16, F16, 128, 8, 560, 32, 8, 70, 200, 1),
    (B16, F32, 64, 8, 88, 64, 8, 250, 100, 3),
    (F16, F32, 128, 8, 88, 64, 8, 190, 40, 3),
]


@pytest.mark.parametrize("case", LARGE, ids=lambda c: f"{str(c[0])[6:]}-{str(c[1])[6:]}-D{c[2]}-B{c[3]}_{c[4]}-H{c[5]}_{c[6]}-P{c[7]}-N{c[8]}-n{c[9]}")
@pytest.mark.parametrize("ragged", [False, True], ids=["", "ragged"])
def test_large_calls(A, case, ragged):
    dtype, out_dtype, D, Bp, B, Hq, Hkv, P, N, n = case
    print(case, flush=True)
    W, G, up = B // Bp, Hq // Hkv, lambda x: (x + 63) // 64 * 64
    g = torch.Generator(device=DEV).manual_seed(P + N + n)
    p, c = A.BlockCache.allocate(Bp, Hq, Hkv, D, up(P), dtype), A.BlockCache.allocate(B, Hq, Hkv, D, up(N), dtype, n=n)
    c.reserve(n, prefix=p)
    first = [P if not ragged else max(0, P - i * (P // Bp) - 7 * i) for i in range(Bp)]
    lens = [N if not ragged else max(0, N - b * (N // B) - 5 * b) for b in range(B)]
    n_q = [n if not ragged else max(0, n - b % 3 * (n // 2)) for b in range(B)]
    for cache, size in ((p, first), (c, lens)):
        for t in (cache.k_tail, cache.v_tail):
            t.fill_(float("nan"))
        scale = torch.pow(10.0, torch.rand(1, Hkv, 1, D, generator=g, device=DEV) - 0.5)
        k, v = ((torch.randn(cache.B, Hkv, max(size), D, generator=g, device=DEV) * scale).to(dtype) for _ in range(2))
        A.akb_append(cache, k, v, i32(size))
    q = torch.randn(B, Hq, n, D, generator=g, device=DEV).to(dtype)
    out = torch.full(q.shape, 3.0, dtype=out_dtype, device=DEV)
    A.akb_attention_shared(p, c, q, out, n_q=i32(n_q) if ragged else None)
    again = A.akb_attention_shared(p, c, q, torch.full_like(out, 3.0), n_q=i32(n_q) if ragged else None)
    assert torch.equal(out, again), "the same call gives the same bits"
    (KP, VP), (KC, VC) = A.akb_unpack(p), A.akb_unpack(c)
    half = float(torch.finfo(dtype).eps) / 2
    for b in range(0, B, max(1, B // 16)):
        a, m = b // W, n_q[b]
        L = first[a] + lens[b]
        assert (out[b, :, m:].float() == 3.0).all()
        for h in range(0, Hkv, max(1, Hkv // 4)):
            Kd, Vd = (torch.cat([x[a, h, :first[a]], y[b, h, :lens[b]]]).double() for x, y in ((KP, KC), (VP, VC)))
            qd = q[b, h * G:(h + 1) * G, :m].double().reshape(G * m, D)
            past = torch.arange(L, device=DEV)[None] > (L - m + torch.arange(m, device=DEV)).repeat(G)[:, None]
            x = (qd @ Kd.T / D ** 0.5).masked_fill_(past, -float("inf"))
            size = (qd.abs() @ Kd.abs().T).masked_fill_(past, 0.0).amax(dim=1, keepdim=True) if m and L else x.new_zeros(len(qd), 1)
            w = torch.softmax(x, dim=1).nan_to_num_(0.0)
            want, mag = w @ Vd, w @ Vd.abs()
            # as in the reference: products in 32 bits, the scaling and the subtraction, exponentials, sums
            top = x.masked_fill(past, 0.0).abs().amax(dim=1, keepdim=True) if m and L else size
            eps = 2 * (D ** 0.5 * 2.0 ** -24 * size + 2.0 ** -22 * top + 2.0 ** -22) + (L / 16 + 64) * 2.0 ** -23
            bound = eps * mag + (half ** 2 * mag if out_dtype == F32 else half * mag + half * want.abs()) + (2.0 ** -25 if out_dtype == F16 else 0.0) + 1e-30
            got = out[b, h * G:(h + 1) * G, :m].double().reshape(G * m, D)
            assert (((got - want).abs() <= bound).all()), (b, h, float(((got - want).abs() / bound).max()))


def test_scale_and_length_bounds(A):
    p, pr, c, cr = caches(A, 2, 4, 8, 2, 128, 900, 300, F16, [900, 130], [300, 7, 64, 0], 2)
    for max_len, prefix_max_len in ((0, 0), (1, 1), (320, 960), (64, 900), (0, 64)):   # hints: longer sequences are attended whole
        check(A, p, pr, c, cr, 2, None, F32, f"{max_len} {prefix_max_len}", scale=0.3, max_len=max_len, prefix_max_len=prefix_max_len)
    q = R.tokens(4, 8, 1, 128, F16, 2, "plain").to(DEV)
    flat = A.akb_attention_shared(p, c, q[:, :, 0].contiguous())
    assert flat.shape == (4, 8, 128) and torch.equal(flat, A.akb_attention_shared(p, c, q)[:, :, 0])


@pytest.mark.parametrize("n", [1, 9, 60])
def test_scores_far_apart_and_large_values(A, n):
    """Logits of thousands, in the prefix, behind it, or in both; values of the largest size; bfloat16 values of 2^120 in one part only."""
    for dtype in (F16, B16):
        for loud in (0, 1):
            p, pr = pair(A, 1, 2, 1, 128, 256, dtype)
            c, cr = pair(A, 3, 2, 1, 128, 128, dtype)
            for i, (cache, ref, m) in enumerate(((p, pr, 200), (c, cr, 100))):
                k = R.tokens(cache.B, 1, m, 128, dtype, 5 + i, "plain") * (60 if i == loud else 1)
                v = R.tokens(cache.B, 1, m, 128, dtype, 7 + i, "plain") * 2 ** 12
                if dtype == B16 and i != loud:
                    v[:, :, m // 2] *= 2.0 ** 106
                ref.append(k, v)
                A.akb_append(cache, k.to(DEV), v.to(DEV))
            c.reserve(n, prefix=p)
            check(A, p, pr, c, cr, n, None, F32, f"{dtype} loud {loud}")
            check(A, p, pr, c, cr, n, None, dtype, f"{dtype} loud {loud}, 16 bits")


def test_the_prefix_is_what_a_cache_of_all_the_tokens_gives(A):
    """A batch behind a prefix of whole blocks against the same batch whose caches hold the prefix, too: the same numbers in another order of sums."""
    p, pr, c, cr = caches(A, 1, 5, 8, 2, 64, 640, 100, B16, [640], [100, 1, 64, 33, 70], 3)
    whole = A.BlockCache.allocate(5, 8, 2, 64, 768, B16, n=3)
    A.akb_fork(p, whole, i32([0] * 5))
    for b, m in enumerate([100, 1, 64, 33, 70]):
        k, v = (torch.zeros(5, 2, 100, 64, dtype=B16) for _ in range(2))
        for h in range(2):
            k[b, h, :m], v[b, h, :m] = (torch.from_numpy(cr.tokens[b][h][s]).to(B16) for s in (0, 1))
        A.akb_append(whole, k.to(DEV), v.to(DEV), i32([m if i == b else 0 for i in range(5)]))
    q = R.tokens(5, 8, 3, 64, B16, 3, "plain").to(DEV)
    n_q = i32([3, 1, 3, 3, 3])
    ref, eps, mag = S.joined(pr, cr).attention(q.cpu(), [3, 1, 3, 3, 3])
    a, b = A.akb_attention(whole, q, n_q=n_q), A.akb_attention_shared(p, c, q, n_q=n_q)
    R.assert_attention(a, ref, eps, mag, B16, "one cache")
    R.assert_attention(b, ref, eps, mag, B16, "two")


@pytest.mark.parametrize("n", [1, 5, 30])
def test_a_query_that_is_not_finite_stays_with_its_row(A, n):
    """Rows of many sequences lie in one tile: a NaN or an infinity in one is in no other's result."""
    p, pr, c, cr = caches(A, 1, 20, 32, 8, 128, 2000, 100, B16, [2000], [100 - 4 * b for b in range(20)], n)
    q = R.tokens(20, 32, n, 128, B16, 2, "plain").to(DEV)
    want = A.akb_attention_shared(p, c, q).clone()
    q[3, 5, n // 2, 7], q[17, 0, 0, 100] = float("nan"), float("inf")
    got = A.akb_attention_shared(p, c, q)
    same = (got == want).all(dim=-1)
    bad = torch.zeros_like(same)
    bad[3, 5, n // 2] = bad[17, 0, 0] = True
    assert same[~bad].all() and torch.isnan(got[3, 5, n // 2]).all()


def test_two_calls_at_once_on_a_prefix(A):
    """Two batches on two streams, one prefix, a workspace each; and a workspace of NaN bits, prepared, gives the same."""
    p, pr, c0, cr0 = caches(A, 1, 6, 16, 4, 128, 3000, 200, F16, [3000], [200, 3, 77, 64, 1, 130], 4)
    _, _, c1, cr1 = caches(A, 1, 3, 16, 4, 128, 64, 90, F16, [64], [90, 64, 5], 4, seed=3)
    c1.reserve(4, prefix=p)
    qs = [R.tokens(c.B, 16, 4, 128, F16, 2, "plain").to(DEV) for c in (c0, c1)]
    want = [A.akb_attention_shared(p, c, q).clone() for c, q in zip((c0, c1), qs)]
    c0.workspace.fill_(0xFF)
    A.akb_workspace_init(c0.workspace)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in qs], [[] for _ in qs]
    for _ in range(5):
        for i, (s, c) in enumerate(zip(streams, (c0, c1))):
            with torch.cuda.stream(s):
                got[i].append(A.akb_attention_shared(p, c, qs[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i]) for i in (0, 1) for o in got[i])


def test_offsets_beyond_32_bits(A):
    """The last heads of a prefix of 9 GB give what a small prefix with the same tokens gives."""
    D, H = 128, 36
    big, small = (A.BlockCache.allocate(1, H, H, D, Ncap, B16) for Ncap in (1 << 20, 384))
    c = A.BlockCache.allocate(2, H, H, D, 128, B16)
    k, v, q = (R.tokens(m, H, n, D, B16, s).to(DEV) for m, s, n in ((1, 1, 333), (1, 2, 333), (2, 3, 1)))
    A.akb_append(c, *(R.tokens(2, H, 70, D, B16, s).to(DEV) for s in (4, 5)))
    outs = []
    for p in (big, small):
        A.akb_append(p, k, v)
        outs.append(A.akb_attention_shared(p, c.reserve(1, prefix=p), q, prefix_max_len=384))
    assert torch.equal(*outs)
