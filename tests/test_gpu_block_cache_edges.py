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
