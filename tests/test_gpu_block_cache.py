"""The block-scaled 8-bit cache on the GPU against its 64-bit reference: what is stored is equal in every bit, attention lies within the bound that the
arithmetic gives, eviction keeps the same tokens."""
import numpy as np
import pytest
import torch

import block_cache_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, B16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def A():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2409_16546_amd import binding
    return binding


def i32(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)


def pair(A, B, Hq, Hkv, D, Ncap, dtype, score=False, n=1):
    print(f"cache B{B} H{Hq}/{Hkv} D{D} Ncap{Ncap} {dtype}", flush=True)
    c = A.BlockCache.allocate(B, Hq, Hkv, D, Ncap, dtype, score=score, n=n)
    for t in (c.k8, c.v8):   # codes that are NaN, and tails that are not finite: nothing behind a length is read
        t.fill_(0x7F)
    c.exps.fill_(120)
    for t in (c.k_tail, c.v_tail):
        t.fill_(float("nan"))
    return c, R.Ref(B, Hq, Hkv, D, Ncap, dtype)


def put(A, c, ref, n, seed, n_new=None, kind="scales"):
    k, v = (R.tokens(c.B, c.Hkv, n, c.D, c.dtype, seed + s, kind) for s in (0, 1))
    ref.append(k, v, n_new)
    if n_new is not None:   # rows that are not taken may hold anything
        for b, m in enumerate(n_new):
            k[b, :, max(m, 0):] = float("nan")
            v[b, :, max(m, 0):] = float("inf")
    A.akb_append(c, k.to(DEV), v.to(DEV), i32(n_new))


# ------------------------------------------------------------------------------------------------------------ store

@pytest.mark.parametrize("dtype", [F16, B16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("steps", [(1,), (63, 1, 1), (64,), (65,), (30, 200, 5), (127, 2, 130), (1,) * 66, (500,)], ids=lambda s: "-".join(map(str, s[:4])))
def test_append_stores_the_references_numbers(A, dtype, D, steps):
    c, ref = pair(A, 2, 4, 2, D, 576, dtype, score=True)
    for i, n in enumerate(steps):
        put(A, c, ref, n, 10 * i + D, kind="wide" if len(steps) == 1 else "scales")
    R.assert_same_tokens(A, c, ref)
    assert not c.flags.any()
    n = ref.len(0)
    assert not c.score.view(2, 2, -1)[:, :, :n].any()


def test_ragged_appends_and_refusals(A):
    c, ref = pair(A, 5, 2, 2, 128, 192, F16, score=True)
    c.score.fill_(7.0)
    for i, (n, n_new) in enumerate([(100, [100, 0, 64, 1, 63]), (92, [92, 92, -3, 92, 1]), (130, [1, 100, 129, 99, 200]), (70, [0, 0, 64, 0, 65])]):
        put(A, c, ref, n, 50 * i, n_new)
    R.assert_same_tokens(A, c, ref)
    assert ref.refused == 3 and c.flags.cpu().tolist() == [3, 0, 0, 0] + [0] * 5
    score = c.score.view(5, 2, 192).cpu()
    for b in range(5):
        assert not score[b, :, :ref.len(b)].any() and (score[b, :, ref.len(b):] == 7.0).all()


@pytest.mark.parametrize("dtype", [F16, B16], ids=["fp16", "bf16"])
def test_extreme_numbers(A, dtype):
    """The largest numbers of the type, the smallest, whole blocks of zeros, values on and beside the borders between codes, and what is not finite."""
    top = R.LARGEST[dtype]
    lo = 2.0 ** -24 if dtype == F16 else 2.0 ** -133
    rows = [torch.full((64, 64), top), torch.full((64, 64), lo), torch.zeros(64, 64), torch.linspace(-top, top, 4096).view(64, 64),
            torch.linspace(0, 448, 4096).view(64, 64) * 2.0 ** -10, torch.tensor([(i % 127 + 0.5) * 2.0 ** -9 for i in range(4096)]).view(64, 64),
            torch.tensor(R.E4M3[np.arange(4096) % 127]).view(64, 64), torch.full((64, 64), 448.0 * 2.0 ** 5), torch.full((64, 64), 450.0),
            torch.tensor([top * 0.97, -top * 0.93, top * 0.88, 1.0]).repeat(1024).view(64, 64)]
    x = torch.cat([r.double().clamp(-top, top) for r in rows]).to(dtype)[None, None]
    bad = x[:, :, :64].clone()
    bad[0, 0, 3, 5], bad[0, 0, 9, 7], bad[0, 0, 40, 63] = float("nan"), float("inf"), float("-inf")
    x = torch.cat([x, bad], dim=2)
    c, ref = pair(A, 1, 1, 1, 64, x.shape[2], dtype)
    ref.append(x, x)
    A.akb_append(c, x.to(DEV), x.to(DEV))
    R.assert_same_tokens(A, c, ref)


def test_the_bytes_do_not_depend_on_how_the_appends_were_cut(A):
    k, v = (R.tokens(3, 2, 333, 128, B16, s).to(DEV) for s in (1, 2))
    caches = []
    for cuts in ([333], [1] * 70 + [263], [64, 64, 64, 64, 64, 13], [50, 200, 83]):
        c, _ = pair(A, 3, 2, 2, 128, 384, B16)
        at = 0
        for n in cuts:
            A.akb_append(c, k[:, :, at:at + n].contiguous(), v[:, :, at:at + n].contiguous())
            at += n
        caches.append(c)
    first = caches[0]
    for c in caches[1:]:
        for name in ("k8", "v8", "exps"):
            assert torch.equal(getattr(c, name), getattr(first, name)), name
        assert all(torch.equal(a, b) for a, b in zip(A.akb_unpack(c), A.akb_unpack(first)))


# -------------------------------------------------------------------------------------------------------- attention

CASES = [  # dtype, out, D, Hq, Hkv, tokens of each sequence, n, n_q
    (F16, F32, 128, 4, 4, [1, 0, 64, 63, 65, 700], 1, None),
    (F16, F16, 128, 8, 2, [1, 0, 64, 200, 1000], 1, None),
    (B16, F32, 128, 8, 1, [129, 128, 1], 1, None),
    (B16, B16, 64, 5, 1, [0, 77, 256], 1, None),
    (F16, F32, 64, 16, 1, [90, 2000], 1, None),
    (F16, F32, 128, 12, 4, [100, 64, 5, 130], 5, None),           # groups of three; a sequence that is all query tokens
    (B16, B16, 128, 8, 2, [70, 300, 2, 0], 7, [7, 3, 7, 2]),       # query tokens that stand in front of the first
    (F16, F16, 128, 2, 2, [150, 64], 150, [150, 64]),              # prompts over themselves
    (B16, B16, 64, 8, 2, [200, 199, 17], 65, [65, 0, 33]),
    (F16, F32, 64, 4, 2, [500, 63], 33, None),
    (B16, F32, 128, 16, 1, [260], 40, None),
    (F16, F16, 128, 4, 1, [1100, 321], 300, [300, 257]),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{str(c[0])[6:]}-{str(c[1])[6:]}-D{c[2]}-H{c[3]}_{c[4]}-n{c[6]}-{'_'.join(map(str, c[5]))}")
@pytest.mark.parametrize("accumulate", [False, True], ids=["", "score"])
def test_attention(A, case, accumulate):
    dtype, out_dtype, D, Hq, Hkv, lens, n, n_q = case
    B, Ncap = len(lens), (max(lens) + 63) // 64 * 64 + 64
    c, ref = pair(A, B, Hq, Hkv, D, max(Ncap, (n + 63) // 64 * 64), dtype, score=accumulate, n=n)
    put(A, c, ref, max(lens), 3, lens)
    q = R.tokens(B, Hq, n, D, dtype, 9, "plain")
    if accumulate:
        c.score.copy_(torch.rand(c.score.shape, generator=torch.Generator().manual_seed(4)))
    before = c.score.clone() if accumulate else None
    start = torch.full(q.shape, 5.0, dtype=out_dtype, device=DEV)
    sent = q.clone()
    for b in range(B):
        sent[b, :, n if n_q is None else n_q[b]:] = float("nan")
    out = A.akb_attention(c, sent.to(DEV), start.clone(), n_q=i32(n_q), accumulate=accumulate)
    want, eps, mag = ref.attention(q, n_q, accumulate=accumulate)
    R.assert_attention(out, want, eps, mag, dtype, "out")
    assert (out.cpu().numpy()[np.isnan(want)] == 5.0).all() if out_dtype != B16 else (out.float().cpu().numpy()[np.isnan(want)] == 5.0).all()
    if accumulate:
        got, was = c.score.double().cpu().numpy().reshape(B, Hkv, -1), before.double().cpu().numpy().reshape(B, Hkv, -1)
        worst = float(np.nanmax(eps)) if np.isfinite(eps).any() else 0.0
        for b in range(B):
            L, rows = ref.len(b), (Hq // Hkv) * n
            for h in range(Hkv):
                add = ref.score[b][h]
                bound = worst * add + rows * 2.0 ** -24 * (1 + add) + 2.0 ** -23 * (1 + add)
                assert (np.abs(got[b, h, :L] - was[b, h, :L] - add) <= bound).all(), (b, h)
                assert (got[b, h, L:] == was[b, h, L:]).all()
    R.assert_same_tokens(A, c, ref, "the cache is as it was")


# kernel and parts, dtype, out, D, B, Hq, Hkv, tokens, ragged, n, ragged n: calls large enough for every way a call is cut, against 64 bits on the GPU
LARGE = [
    ((1, 4), F16, F32, 128, 1, 4, 4, 1000, False, 1, False),         # parts joined by the last workgroup
    ((1, 64), B16, B16, 128, 1, 64, 8, 20000, False, 1, False),      # ... by a launch, many parts
    ((1, 8), B16, F32, 64, 1, 32, 8, 2000, False, 2, False),
    ((1, 2), F16, F32, 64, 300, 4, 1, 600, True, 1, True),           # more sequences than the device would look through
    ((1, 1), F16, F16, 128, 16, 32, 32, 300, True, 1, False),        # whole walks
    ((1, 0), F16, F32, 128, 4, 32, 32, 9000, True, 1, False),        # parts by the lengths
    ((1, 0), B16, B16, 64, 3, 64, 4, 90000, True, 1, False),
    ((2, 11), F16, F32, 128, 3, 64, 8, 5000, True, 5, True),         # two row groups
    ((2, 0), B16, B16, 64, 5, 16, 8, 30000, True, 9, True),
    ((2, 1), F16, F16, 128, 32, 16, 16, 200, True, 40, True),
    ((3, 1), B16, B16, 128, 2, 32, 8, 1100, False, 1100, False),     # prompts over themselves
    ((3, 1), F16, F32, 64, 8, 10, 2, 801, True, 800, True),          # groups of five: row groups that end inside a query token
    ((3, 2), F16, F32, 128, 4, 8, 8, 4099, True, 1000, True),        # chunks in parts
    ((3, 0), B16, F32, 128, 2, 16, 4, 66000, True, 64, False),
    ((2, 4), F16, F16, 64, 1, 16, 2, 6000, False, 333, False),
    ((3, 13), F16, F16, 64, 1, 16, 2, 12000, False, 333, False),
]


@pytest.mark.parametrize("case", LARGE, ids=lambda c: f"kernel{c[0][0]}-parts{c[0][1]}-D{c[3]}-B{c[4]}-H{c[5]}_{c[6]}-N{c[7]}-n{c[9]}")
def test_large_calls(A, case):
    path, dtype, out_dtype, D, B, Hq, Hkv, N, ragged, n, ragged_n = case
    G, Ncap = Hq // Hkv, (N + 63) // 64 * 64
    print(case, flush=True)
    assert A.akb_attention_path(B, Hq, Hkv, D, Ncap, n) == path
    g = torch.Generator(device=DEV).manual_seed(N + n)
    c = A.BlockCache.allocate(B, Hq, Hkv, D, Ncap, dtype, score=True, n=n)
    c.k_tail.fill_(float("nan"))
    c.v_tail.fill_(float("nan"))
    lens = [N if not ragged else max(1, N - b * (N // B) - 7 * b) for b in range(B)]
    n_q = [n if not ragged_n else max(0, n - b * (n // B)) for b in range(B)]
    scale = torch.pow(10.0, torch.rand(1, Hkv, 1, D, generator=g, device=DEV) - 0.5)
    k, v = ((torch.randn(B, Hkv, N, D, generator=g, device=DEV) * scale).to(dtype) for _ in range(2))
    A.akb_append(c, k, v, i32(lens))
    q = torch.randn(B, Hq, n, D, generator=g, device=DEV).to(dtype)
    start = torch.rand(c.score.shape, generator=g, device=DEV)
    c.score.copy_(start)
    out = torch.full(q.shape, 3.0, dtype=out_dtype, device=DEV)
    A.akb_attention(c, q, out, n_q=i32(n_q) if ragged_n else None, accumulate=True)
    K, V = A.akb_unpack(c)
    half = float(torch.finfo(dtype).eps) / 2
    for b in range(B):
        L, m = lens[b], n_q[b]
        assert (out[b, :, m:].float() == 3.0).all()
        for h in range(Hkv):
            Kd, Vd = K[b, h, :L].double(), V[b, h, :L].double()
            qd = q[b, h * G:(h + 1) * G, :m].double().reshape(G * m, D)
            past = torch.arange(L, device=DEV)[None] > (L - m + torch.arange(m, device=DEV)).repeat(G)[:, None]
            x = (qd @ Kd.T / D ** 0.5).masked_fill_(past, -float("inf"))
            size = (qd.abs() @ Kd.abs().T).masked_fill_(past, 0.0).amax(dim=1, keepdim=True) if m else x.new_zeros(0, 1)
            p = torch.softmax(x, dim=1).nan_to_num_(0.0)
            want, mag = p @ Vd, p @ Vd.abs()
            # as in the reference: products in 32 bits, the scaling and the subtraction, exponentials, sums
            top = x.masked_fill(past, 0.0).abs().amax(dim=1, keepdim=True) if m else size
            eps = 2 * (D ** 0.5 * 2.0 ** -24 * size + 2.0 ** -22 * top + 2.0 ** -22) + (L / 16 + 64) * 2.0 ** -23
            bound = eps * mag + (half ** 2 * mag if out_dtype == F32 else half * mag + half * want.abs()) + (2.0 ** -25 if out_dtype == F16 else 0.0) + 1e-30
            got = out[b, h * G:(h + 1) * G, :m].double().reshape(G * m, D)
            assert (((got - want).abs() <= bound).all()), (b, h, float(((got - want).abs() / bound).max()))
            add = p.sum(dim=0)
            rel = float(eps.max()) if m else 0.0
            now, was = c.score.view(B, Hkv, -1)[b, h].double(), start.view(B, Hkv, -1)[b, h].double()
            assert ((now[:L] - was[:L] - add).abs() <= rel * add + (G * m / 16 + 32) * 2.0 ** -23 * (1 + add)).all(), (b, h)
            assert (now[L:] == was[L:]).all()


def test_scale_and_length_bound(A):
    c, ref = pair(A, 2, 4, 2, 128, 1024, F16)
    put(A, c, ref, 900, 1, [900, 130])
    q = R.tokens(2, 4, 1, 128, F16, 2, "plain")
    want = ref.attention(q, scale=0.3)
    for max_len in (0, 1024, 900, 128, 1):   # a hint: longer sequences are attended whole
        R.assert_attention(A.akb_attention(c, q.to(DEV), scale=0.3, max_len=max_len), *want, F16, f"max_len {max_len}")
    flat = A.akb_attention(c, q[:, :, 0].contiguous().to(DEV), scale=0.3)
    assert flat.shape == (2, 4, 128) and torch.equal(flat, A.akb_attention(c, q.to(DEV), scale=0.3)[:, :, 0])


def test_the_same_call_gives_the_same_bits(A):
    c, ref = pair(A, 3, 8, 2, 128, 2048, B16, score=True, n=20)
    put(A, c, ref, 2000, 1, [2000, 70, 900])
    for n in (1, 20):
        q = R.tokens(3, 8, n, 128, B16, 2, "plain").to(DEV)
        runs = []
        for _ in range(3):
            c.score.zero_()
            runs.append((A.akb_attention(c, q, accumulate=True).clone(), c.score.clone()))
        assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(r, runs[0]))


def test_scores_far_apart_and_outlier_values(A):
    """Logits of thousands (one token takes all) and values of the largest size: nothing overflows on the way."""
    for dtype in (F16, B16):
        c, ref = pair(A, 1, 2, 1, 128, 256, dtype)
        k, v = R.tokens(1, 1, 200, 128, dtype, 5, "plain") * 60, R.tokens(1, 1, 200, 128, dtype, 6, "plain") * 2 ** 12
        ref.append(k, v)
        A.akb_append(c, k.to(DEV), v.to(DEV))
        q = R.tokens(1, 2, 3, 128, dtype, 7, "plain") * 40
        c.reserve(3)
        R.assert_attention(A.akb_attention(c, q.to(DEV)), *ref.attention(q), dtype, str(dtype))


@pytest.mark.parametrize("n", [1, 30, 100])
def test_scores_of_logits_far_apart(A, n):
    """Logits of hundreds: rows that fill a tile behind the last one weigh nothing, whatever their products are."""
    c, ref = pair(A, 1, 1, 1, 128, 1600, B16, score=True, n=100)
    k, v = R.tokens(1, 1, 1500, 128, B16, 5, "plain") * 8, R.tokens(1, 1, 1500, 128, B16, 6, "plain")
    ref.append(k, v)
    A.akb_append(c, k.to(DEV), v.to(DEV))
    q = R.tokens(1, 1, n, 128, B16, 7, "plain") * 16
    want, eps, mag = ref.attention(q, accumulate=True)
    R.assert_attention(A.akb_attention(c, q.to(DEV), accumulate=True), want, eps, mag, B16, f"n {n}")
    got, add = c.score.double().cpu().numpy()[:1500], ref.score[0][0]
    assert (np.abs(got - add) <= eps.max() * add + n * 2.0 ** -23).all() and abs(got.sum() - n) <= eps.max() * n + 1500 * n * 2.0 ** -23


def test_offsets_beyond_32_bits(A):
    """The last heads of a cache of 9 GB give what a small cache with the same tokens gives."""
    D, Ncap, H = 128, 1 << 20, 36
    big = A.BlockCache.allocate(1, H, H, D, Ncap, B16, score=True)
    small = A.BlockCache.allocate(1, H, H, D, 384, B16, score=True)
    k, v, q = (R.tokens(1, H, n, D, B16, s).to(DEV) for s, n in ((1, 333), (2, 333), (3, 1)))
    outs = []
    for c in (big, small):
        A.akb_append(c, k, v)
        outs.append(A.akb_attention(c, q, accumulate=True, max_len=384).clone())
    assert torch.equal(*outs)
    assert torch.equal(big.score.view(H, Ncap)[:, :333], small.score.view(H, 384)[:, :333])
    kept = torch.zeros(1, H, 100, dtype=torch.int32, device=DEV)
    for i, c in enumerate((big, small)):
        to = A.BlockCache.allocate(1, H, H, D, 128, B16)
        A.akb_evict(c, to, 100, 10, kept=kept)
        outs[i] = (kept.clone(), *A.akb_unpack(to))
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    # 70000 tokens in one head: blocks far inside the plane
    long = A.BlockCache.allocate(1, 1, 1, D, 1 << 22, F16)
    k = torch.randn(1, 1, 70000, D, device=DEV).to(F16)
    A.akb_append(long, k, k)
    assert int(long.lens) == 70000


# ---------------------------------------------------------------------------------------------------------- eviction

@pytest.mark.parametrize("dtype,D", [(F16, 128), (B16, 64)])
@pytest.mark.parametrize("lens,keep,recent", [([300, 128, 0, 1, 200], 128, 30), ([300, 64, 65, 700, 129], 65, 0), ([90, 200, 500], 200, 200),
                                              ([1500, 64, 1023], 1, 0), ([1100, 3], 1000, 64),
                                              ([40000, 33, 0, 20001, 5000], 5000, 100), ([33000, 8193], 8000, 0)])
def test_evict(A, dtype, D, lens, keep, recent):
    """(More than 32768 tokens of capacity and few heads: a launch per step of the selection.)"""
    B, Ncap = len(lens), max(1536, (max(lens) + 63) // 64 * 64)
    c, ref = pair(A, B, 2, 2, D, Ncap, dtype, score=True)
    put(A, c, ref, max(lens), 3, lens)
    score = torch.rand(B, 2, Ncap, generator=torch.Generator().manual_seed(8))
    score = torch.where(score < 0.3, torch.round(score * 8) / 8, score)     # many equal ones, zeros among them
    score[:, 0] *= torch.exp2(torch.randint(-60, 3, (B, Ncap), generator=torch.Generator().manual_seed(9)).float())
    if lens[0] > 20:
        score[0, 1, 3], score[0, 1, 11], score[0, 1, 17] = float("nan"), float("inf"), -0.0
    c.score.copy_(score.flatten())
    for b in range(B):
        for h in range(2):
            ref.score[b][h] = score[b, h, :lens[b]].double().numpy()
    want, places = ref.evict(keep, recent)
    for with_score in (True, False):
        d, _ = pair(A, B, 2, 2, D, (keep + 127) // 64 * 64, dtype, score=with_score)
        want.Ncap = d.Ncap
        kept = torch.full((B, 2, keep), 99, dtype=torch.int32, device=DEV)
        if with_score:
            A.akb_evict(c.reserve(1, keep), d, keep, recent, kept=kept)
            assert np.array_equal(kept.cpu().numpy(), places)
            got = d.score.view(B, 2, -1).cpu().numpy()
            for b in range(B):
                for h in range(2):
                    assert np.array_equal(got[b, h, :want.len(b)].astype(np.float64), want.score[b][h], equal_nan=True)
        else:
            A.akb_evict(c.reserve(1, keep), d, keep, recent)
        R.assert_same_tokens(A, d, want, f"score {with_score}")
    R.assert_same_tokens(A, c, ref, "the source is as it was")


# ---------------------------------------------------------------------------------------------------------- together

@pytest.mark.parametrize("dtype,D,Hq,Hkv", [(F16, 128, 4, 2), (B16, 64, 3, 1)])
def test_prompt_steps_and_evictions_together(A, dtype, D, Hq, Hkv):
    """A prompt is stored and attends, the cache is brought down to a budget, steps follow, a draft, and the next eviction into the other cache."""
    B = 3
    c, ref = pair(A, B, Hq, Hkv, D, 320, dtype, score=True, n=200)
    d, _ = pair(A, B, Hq, Hkv, D, 320, dtype, score=True, n=200)
    n_new = [200, 131, 64]
    put(A, c, ref, 200, 1, n_new)
    q = R.tokens(B, Hq, 200, D, dtype, 2, "plain")
    R.assert_attention(A.akb_attention(c, q.to(DEV), n_q=i32(n_new), accumulate=True), *ref.attention(q, n_new, accumulate=True), dtype, "prompt")
    for turn in range(2):
        # the reference goes on from the library's scores (they agree to the bounds of the test above; equal scores would be a matter of the last bit)
        for b in range(B):
            for h in range(Hkv):
                ref.score[b][h] = c.score.view(B, Hkv, -1)[b, h, :ref.len(b)].double().cpu().numpy()
        A.akb_evict(c.reserve(200, 100), d, 100, 16)
        ref, _ = ref.evict(100, 16)
        c, d = d, c
        R.assert_same_tokens(A, c, ref, f"turn {turn}: evicted")
        for step in range(30):
            put(A, c, ref, 1, 100 * turn + 3 * step)
            q = R.tokens(B, Hq, 1, D, dtype, 1000 + step, "plain")
            got, want = A.akb_attention(c, q.to(DEV), accumulate=True), ref.attention(q, accumulate=True)
            if step % 10 == 0:
                R.assert_attention(got, *want, dtype, f"turn {turn} step {step}")
        put(A, c, ref, 4, 7 + turn)
        q = R.tokens(B, Hq, 4, D, dtype, 8, "plain")
        R.assert_attention(A.akb_attention(c, q.to(DEV), accumulate=True), *ref.attention(q, accumulate=True), dtype, f"turn {turn}: draft")
        R.assert_same_tokens(A, c, ref, f"turn {turn}: steps stored")


def test_steps_in_hip_graphs_that_share_a_workspace(A):
    """A step (append, attention with scores, eviction into another cache) captured twice, for two caches that share one workspace, and replayed with eager
    work between."""
    def build(seed):
        c, ref = pair(A, 2, 8, 2, 128, 512, F16, score=True)
        put(A, c, ref, 400, seed, [400, 127])
        d, _ = pair(A, 2, 8, 2, 128, 512, F16, score=True)
        return c, d
    k, v, q = (R.tokens(2, h, 1, 128, F16, s).to(DEV) for s, h in ((1, 2), (2, 2), (3, 8)))
    (c0, d0), (c1, d1) = build(10), build(20)
    c1.workspace = c0.reserve(1, 64).workspace
    c0.reserve(1, 64)
    outs = [torch.zeros(2, 8, 1, 128, device=DEV) for _ in range(2)]

    def step(i):
        c, d = ((c0, d0), (c1, d1))[i]
        A.akb_append(c, k, v)
        A.akb_attention(c, q, outs[i], accumulate=True)
        A.akb_evict(c, d, 64, 8, workspace=c0.workspace)

    saved = [[t.clone() for t in (c.lens, c.score, c.k8, c.v8, c.exps, c.k_tail, c.v_tail)] for c in (c0, c1)]

    def restore():
        for c, s in zip((c0, c1), saved):
            for t, x in zip((c.lens, c.score, c.k8, c.v8, c.exps, c.k_tail, c.v_tail), s):
                t.copy_(x)
    eager = []
    for rep in range(3):
        for i in (0, 1):
            step(i)
        eager.append([t.clone() for i, (c, d) in enumerate(((c0, d0), (c1, d1))) for t in (outs[i], c.score, c.lens, d.lens, *A.akb_unpack(d))])
    restore()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.stream(s):
        step(0)
        step(1)
        torch.cuda.synchronize()
        for i in (0, 1):
            with torch.cuda.graph(graphs[i], stream=s):
                step(i)
    torch.cuda.current_stream().wait_stream(s)
    restore()
    other, _ = pair(A, 1, 4, 4, 64, 256, B16)
    for rep in range(3):
        for g in graphs:
            g.replay()
        A.akb_append(other, *(R.tokens(1, 4, 3, 64, B16, 5).to(DEV) for _ in range(2)))   # the program's own eager work
        torch.cuda.synchronize()
        now = [t for i, (c, d) in enumerate(((c0, d0), (c1, d1))) for t in (outs[i], c.score, c.lens, d.lens, *A.akb_unpack(d))]
        assert all(torch.equal(a, b) for a, b in zip(now, eager[rep])), f"replay {rep}"


def test_calls_on_another_stream(A):
    c, ref = pair(A, 2, 4, 2, 128, 256, B16, n=5)
    k, v = (R.tokens(2, 2, 150, 128, B16, s) for s in (1, 2))
    ref.append(k, v)
    q = R.tokens(2, 4, 5, 128, B16, 3, "plain")
    kd, vd, qd = k.to(DEV), v.to(DEV), q.to(DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        A.akb_append(c, kd, vd)
        out = A.akb_attention(c, qd)
    s.synchronize()
    R.assert_attention(out, *ref.attention(q), B16, "stream")


@pytest.mark.parametrize("n", [1, 5, 200])
def test_a_workspace_holds_nothing_but_its_control_words(A, n):
    """A workspace full of NaN bits, prepared, gives the bits that a fresh one gives; so does the one before it, used by calls of other sizes in between."""
    c, ref = pair(A, 2, 8, 2, 128, 4096, B16, score=True, n=200)
    put(A, c, ref, 4000, 1, [4000, 2222])
    q = R.tokens(2, 8, n, 128, B16, 2, "plain").to(DEV)
    d, _ = pair(A, 2, 8, 2, 128, 256, B16, score=True)
    outs = []
    for turn in range(3):
        c.score.zero_()
        if turn == 1:
            c.reserve(200, 200).workspace.fill_(0xFF)
            A.akb_workspace_init(c.workspace)
        out = A.akb_attention(c, q, accumulate=True).clone()
        outs.append((out, c.score.clone()))
        A.akb_evict(c.reserve(200, 200), d, 200, 10)                                    # eviction and other attention in the same workspace
        for other in (1, 3, 64):
            A.akb_attention(c, R.tokens(2, 8, other, 128, B16, 3, "plain").to(DEV))
    assert all(torch.equal(a, b) for o in outs[1:] for a, b in zip(o, outs[0]))


def test_two_calls_at_once(A):
    """Two streams, one cache, a workspace each."""
    c, ref = pair(A, 2, 8, 2, 64, 4096, F16, n=64)
    put(A, c, ref, 4000, 1, [4000, 3999])
    qs = [R.tokens(2, 8, n, 64, F16, 2, "plain").to(DEV) for n in (1, 64)]
    want = [A.akb_attention(c, q).clone() for q in qs]
    spaces = [torch.empty_like(c.workspace) for _ in qs]
    for w in spaces:
        A.akb_workspace_init(w)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in qs], [[] for _ in qs]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(A.akb_attention(c, qs[i], workspace=spaces[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i]) for i in (0, 1) for o in got[i])


def test_a_length_set_to_zero_starts_the_sequence_anew(A):
    c, ref = pair(A, 2, 2, 2, 64, 256, F16, score=True)
    put(A, c, ref, 170, 1)
    c.lens[1] = 0
    fresh = R.Ref(2, 2, 2, 64, 256, F16)
    k, v = (R.tokens(2, 2, 30, 64, F16, s) for s in (5, 6))
    A.akb_append(c, k.to(DEV), v.to(DEV), i32([0, 30]))
    fresh.append(k, v, [0, 30])
    q = R.tokens(2, 2, 1, 64, F16, 7, "plain")
    got = A.akb_attention(c, q.to(DEV), accumulate=True)
    want, old = fresh.attention(q), ref.attention(q)
    R.assert_attention(got[1:], want[0][1:], want[1][1:], want[2][1:], F16, "new")
    R.assert_attention(got[:1], old[0][:1], old[1][:1], old[2][:1], F16, "old")
