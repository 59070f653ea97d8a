"""The block-scaled 8-bit cache on the GPU at calls that its documentation allows and the other tests do not make."""
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


# ------------------------------------------------------------------------------------------ lens and flags aligned to 4 bytes

def at_offset(n, skip):
    """(n int32 that begin 4 skip bytes behind a 16-byte boundary, the words in front, those behind)."""
    all_ = torch.full((n + skip + 9,), 0x5A5A5A5A, dtype=torch.int32, device=DEV)
    assert all_.data_ptr() % 16 == 0
    return all_[skip:skip + n], all_[:skip], all_[skip + n:]


@pytest.mark.parametrize("skip", [0, 1, 2, 3])
@pytest.mark.parametrize("B", [1, 2, 3, 4, 5, 11, 700])
def test_lens_and_flags_aligned_to_4_bytes(A, B, skip):
    print(f"B {B} skip {skip}", flush=True)
    good = A.BlockCache.allocate(B, 2, 2, 64, 128, F16, score=True)
    lens, before, after = at_offset(B, skip)
    flags, fbefore, fafter = at_offset(A.AKV_NFLAGS + B, skip)
    c = A.BlockCache(B, 2, 2, 64, 128, F16, *(torch.empty_like(getattr(good, n)) for n in ("k8", "v8", "exps", "k_tail", "v_tail")), lens, flags,
                     torch.empty_like(good.score))
    A.akb_cache_reset(c)
    c.reserve(2)
    good.reserve(2)
    assert not lens.any() and not flags.any() and not c.score.any()
    k, v = (R.tokens(B, 2, 100, 64, F16, s).to(DEV) for s in (1, 2))
    q = R.tokens(B, 4 // 2, 2, 64, F16, 3).to(DEV)
    n_new = i32([(37 * b) % 101 for b in range(B)])
    outs = []
    for x in (good, c):
        A.akb_append(x, k, v, n_new)
        A.akb_append(x, k, v, n_new)      # more than 64 tokens a call are refused the second time
        outs.append((A.akb_attention(x, q, accumulate=True), x.lens.clone(), x.flags.clone(), *A.akb_unpack(x)))
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    assert B < 3 or int(c.flags[0]) > 0
    for t in (before, after, fbefore, fafter):
        assert (t == 0x5A5A5A5A).all()


@pytest.mark.parametrize("skip", [1, 2, 3])
def test_lens_and_flags_of_the_16_bit_cache_aligned_to_4_bytes(A, skip):
    B = 9
    good = A.Cache.allocate(B, 2, 2, 128, 256)
    c = A.Cache.allocate(B, 2, 2, 128, 256)
    c.lens, before, after = at_offset(B, skip)
    c.flags, fbefore, fafter = at_offset(A.AKV_NFLAGS + B, skip)
    c._struct = None
    A.akv_cache_reset(c)
    assert not c.lens.any() and not c.flags.any()
    k, v = (torch.randn(B, 2, 100, 128, generator=torch.Generator().manual_seed(s)).half().to(DEV) for s in (1, 2))
    n_new = i32([11 * b for b in range(B)])
    for x in (good, c):
        A.akv_append(x, k, v, n_new)
    assert all(torch.equal(getattr(good, n), getattr(c, n)) for n in ("k_hi", "k_mid", "k_lo", "v_hi", "v_mid", "v_lo", "colmax", "lens", "flags"))
    for t in (before, after, fbefore, fafter):
        assert (t == 0x5A5A5A5A).all()


# --------------------------------------------------------------------------------------------------------- workspaces

def test_a_replaced_workspace_stays_until_the_cache_goes(A):
    """Calls on other streams, and captured graphs, may still write the workspace that `reserve` replaces: nobody else gets its memory."""
    c = A.BlockCache.allocate(2, 8, 2, 128, 1024, F16, score=True)
    old = [(c.workspace.data_ptr(), c.workspace.numel())]
    for n in (100, 1000):
        c.reserve(n)
        others = [torch.empty(size, dtype=torch.uint8, device=DEV) for _, size in old for _ in range(4)]
        for x in (*others, c.workspace):
            for at, size in old:
                assert x.data_ptr() + x.numel() <= at or at + size <= x.data_ptr()
        old.append((c.workspace.data_ptr(), c.workspace.numel()))
        del others
    before = c.workspace
    assert c.reserve(5).workspace is before       # large enough: the same one
    sizes = [size for _, size in old]
    assert sizes[2] >= 1.5 * sizes[1] >= 2.25 * sizes[0] - 2   # what is kept is never more than twice the present one


# ------------------------------------------------------------------------------ weights of calls whose bound is too small

@pytest.mark.parametrize("D,B,Hq,Hkv,N,n,max_lens", [
    (128, 2, 4, 2, 900, 1, (0, 900, 128, 1)),            # up to 16 rows: from q . k as it was left
    (64, 2, 4, 2, 900, 5, (0, 128, 1)),
    (128, 2, 4, 2, 900, 60, (0, 128, 1)),                # many rows, one share
    (64, 2, 4, 2, 900, 400, (0, 640, 1)),                # ... several
    (128, 4, 32, 8, 3001, 512, (0, 768)),                # the kernel of many rows
    (128, 1, 2, 1, 20000, 3, (0, 64, 5000)),
])
@pytest.mark.parametrize("dtype,out_dtype", [(F16, F32), (B16, B16)], ids=["fp16-f32", "bf16"])
def test_weights_beyond_the_length_bound(A, D, B, Hq, Hkv, N, n, max_lens, dtype, out_dtype):
    """max_len is a hint: longer sequences are attended whole, and every token of theirs has its weight added."""
    from test_gpu_block_cache_range import check
    g = torch.Generator(device=DEV).manual_seed(N + n)
    c = A.BlockCache.allocate(B, Hq, Hkv, D, (N + 63) // 64 * 64, dtype, score=True, n=n)
    lens = [max(1, N - 271 * b) for b in range(B)]
    n_q = [max(1, n - 7 * b) for b in range(B)]
    A.akb_append(c, *(torch.randn(B, Hkv, N, D, generator=g, device=DEV).to(dtype) for _ in range(2)), i32(lens))
    q = torch.randn(B, Hq, n, D, generator=g, device=DEV).to(dtype)
    start = torch.rand(c.score.shape, generator=g, device=DEV)
    K, V = A.akb_unpack(c)
    for max_len in max_lens:
        print(f"max_len {max_len}: {A.akb_attention_path(B, Hq, Hkv, D, c.Ncap, n, max_len)}", flush=True)
        c.score.copy_(start)
        out = A.akb_attention(c, q, torch.full(q.shape, 3.0, dtype=out_dtype, device=DEV), n_q=i32(n_q), accumulate=True, max_len=max_len)
        check(c, q, out, K, V, lens, n_q, start)


# --------------------------------------------------------------------------------------------------- far inside a plane

@pytest.mark.parametrize("dtype", [F16, B16], ids=["fp16", "bf16"])
def test_long_sequence_in_the_largest_capacity(A, dtype):
    """70000 tokens in one head of a cache of 2^22: every block's bytes are those of the same tokens in a small cache, every call reads them where they are."""
    from test_gpu_block_cache_range import check
    D, N, Ncap = 128, 70000, 1 << 22
    g = torch.Generator(device=DEV).manual_seed(1)
    k, v = ((torch.randn(1, 1, N, D, generator=g, device=DEV) * torch.exp2(3 * torch.randn(1, 1, N, 1, generator=g, device=DEV)).clamp(max=1000)).to(dtype) for _ in range(2))
    c = A.BlockCache.allocate(1, 2, 1, D, Ncap, dtype, score=True, n=200)
    cuts = [0, 1, 30000, 30001, 69999, N]
    for a, b in zip(cuts, cuts[1:]):
        A.akb_append(c, k[:, :, a:b].contiguous(), v[:, :, a:b].contiguous())
    assert int(c.lens) == N and not c.flags.any()
    small = A.BlockCache.allocate(1, 2, 1, D, 256, dtype)
    whole = N // 64
    k8, v8, exps = c.k8.view(-1, 64 * D), c.v8.view(-1, 64 * D), c.exps.view(-1, 2)
    for first in (0, 467, 468, 700, whole - 3):      # three blocks at a time; 30000 and 30001 lie in block 468
        A.akb_cache_reset(small)
        A.akb_append(small, *(x[:, :, first * 64:first * 64 + 192].contiguous() for x in (k, v)))
        assert torch.equal(k8[first:first + 3], small.k8.view(-1, 64 * D)[:3]), first
        assert torch.equal(v8[first:first + 3], small.v8.view(-1, 64 * D)[:3]), first
        assert torch.equal(exps[first:first + 3], small.exps.view(-1, 2)[:3]), first
    K, V = A.akb_unpack(c)
    assert torch.equal(K[:, :, whole * 64:N], k[:, :, whole * 64:]) and torch.equal(V[:, :, whole * 64:N], v[:, :, whole * 64:])
    assert not K[:, :, N:].any() and not V[:, :, N:].any()
    K, V = K[:, :, :N].contiguous(), V[:, :, :N].contiguous()
    for n in (1, 20, 200):
        q = torch.randn(1, 2, n, D, generator=g, device=DEV).to(dtype)
        start = torch.rand(c.score.shape, generator=g, device=DEV)
        c.score.copy_(start)
        out = A.akb_attention(c, q, accumulate=True)
        check(c, q, out, K, V, [N], None, start)
    # eviction: what stays, by the scores as they are now
    keep, recent = 5000, 100
    score = c.score[:N].clone()
    score[1000:2000] = 0.25                          # ties
    c.score[:N].copy_(score)
    d = A.BlockCache.allocate(1, 2, 1, D, 5056, dtype, score=True)
    kept = torch.zeros(1, 1, keep, dtype=torch.int32, device=DEV)
    A.akb_evict(c.reserve(200, keep), d, keep, recent, kept=kept)
    order = torch.sort(score[:N - recent], descending=True, stable=True).indices[:keep - recent]
    want = torch.cat([order.sort().values, torch.arange(N - recent, N, device=DEV)])
    assert torch.equal(kept.view(-1).long(), want)
    assert torch.equal(d.score[:keep], score[want]) and int(d.lens) == keep
    again = A.BlockCache.allocate(1, 2, 1, D, 5056, dtype)   # the kept values, stored anew
    A.akb_append(again, K[:, :, want].contiguous(), V[:, :, want].contiguous())
    assert all(torch.equal(a, b) for a, b in zip(A.akb_unpack(d), A.akb_unpack(again)))


# ------------------------------------------------------------------------ who moves the length: workgroups up to, at and beyond the lines

@pytest.mark.parametrize("B,H,n", [(4, 8, 500), (4, 8, 560), (11, 8, 300), (18, 8, 65), (19, 8, 65), (20, 32, 1), (21, 31, 1), (80, 8, 1), (81, 8, 1)],
                         ids=lambda x: str(x))
def test_ragged_appends_with_refusals_by_ticket_and_by_launch(A, B, H, n):
    D, Ncap = 64, max(192, (2 * n + 63) // 64 * 64)
    print(f"B {B} H {H} n {n}: {B * H * ((63 + n + 63) // 64)} workgroups", flush=True)
    c = A.BlockCache.allocate(B, H, H, D, Ncap, F16, score=True)
    ref = R.Ref(B, H, H, D, Ncap, F16)
    c.score.fill_(7.0)
    rows = torch.Generator().manual_seed(n)
    start = [(Ncap - n, Ncap - n + 1, Ncap, 0, 63, 64)[b % 6] for b in range(B)]   # it just fits, it does not (twice), whatever else
    for turn in range(3):
        n_new = start if turn == 0 else [(n, int(torch.randint(0, n + 1, (1,), generator=rows)), n, 0, n, -2, n + 9)[(b + turn) % 7] for b in range(B)]
        m = max(start) if turn == 0 else n
        k, v = (R.tokens(B, H, m, D, F16, 10 * turn + s) for s in (0, 1))
        ref.append(k, v, n_new)
        A.akb_append(c, k.to(DEV), v.to(DEV), i32(n_new))
    assert ref.refused > 0 and c.flags.cpu().tolist() == [ref.refused, 0, 0, 0] + [0] * B
    R.assert_same_tokens(A, c, ref)
    score = c.score.view(B, H, Ncap).cpu()
    for b in range(B):
        assert not score[b, :, :ref.len(b)].any() and (score[b, :, ref.len(b):] == 7.0).all(), b
