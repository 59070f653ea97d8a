"""Sequences copied and cut back, on the GPU against the reference: every stored value, exponent and length is equal."""
import pytest
import torch

import block_cache_ref as R
import block_cache_share_ref as S
from test_gpu_block_cache import A, B16, DEV, F16, i32, pair, put  # noqa: F401

pytestmark = pytest.mark.gpu
LENS = [300, 0, 64, 63, 129, 1, 192]


def scored(c, ref, seed):
    """Random scores in both."""
    s = torch.rand(c.B, c.Hkv, c.Ncap, generator=torch.Generator().manual_seed(seed))
    c.score.copy_(s.flatten())
    for b in range(c.B):
        for h in range(c.Hkv):
            ref.score[b][h] = s[b, h, :ref.len(b)].double().numpy()


def same_scores(c, ref):
    got = c.score.view(c.B, c.Hkv, -1).double().cpu().numpy()
    return all((got[b, h, :ref.len(b)] == ref.score[b][h]).all() for b in range(c.B) for h in range(c.Hkv))


@pytest.mark.parametrize("dtype,D", [(F16, 128), (B16, 64), (B16, 128)])
@pytest.mark.parametrize("parents,upto", [(None, None), ([0, 0, 0, 4, 2, 6, 0], None), ([6, 0, 0, 0, 4, 4, 0], [191, 299, 256, 257, 64, 65, 1]),
                                          ([0, 0, 0, 0, 3, 5, 2], [0, -3, 63, 64, 1 << 30, 1, 64]), ([-1, 7, 0, 1 << 30, -(1 << 31), 4, 1], [5] * 7),
                                          (None, [128, 5, 64, 62, 127, 0, 100])])
def test_fork(A, dtype, D, parents, upto):
    c, ref = pair(A, 7, 4, 2, D, 320, dtype, score=True)
    put(A, c, ref, 300, 1, LENS, kind="wide")
    scored(c, ref, 5)
    for with_score in (True, False):
        d, want = pair(A, 7, 4, 2, D, 384, dtype, score=with_score)
        put(A, d, want, 130, 7, [130, 5, 64, 0, 1, 100, 65])
        if with_score:
            scored(d, want, 6)
            before = d.score.clone()
        A.akb_fork(c, d, i32(parents), i32(upto))
        S.fork(ref, want, parents, upto)
        R.assert_same_tokens(A, d, want, f"score {with_score}")
        assert not d.flags.any()
        if with_score:
            assert same_scores(d, want)
            now, was = d.score.view(7, 2, -1), before.view(7, 2, -1)
            assert all(torch.equal(now[b, :, want.len(b):], was[b, :, want.len(b):]) for b in range(7))
        for n in (1, 70, 64):   # the copies go on: what is in the tails is stored with what follows
            put(A, d, want, n, 20 + n)
        R.assert_same_tokens(A, d, want, "with more tokens")
    R.assert_same_tokens(A, c, ref, "the source is as it was")


@pytest.mark.parametrize("N,W", [(320, 1), (4096, 9)])   # copies in runs of blocks, and streamed block by block
def test_fork_from_a_cache_without_scores(A, N, W):
    """The copied tokens have no weight yet, whatever the sequence that they replace had; what is behind them stays; eviction then keeps the tokens that were attended."""
    H, D = 16, 128
    c, d = A.BlockCache.allocate(2, H, H, D, N, F16), A.BlockCache.allocate(2 * W, H, H, D, N, F16, score=True)
    lens = [N - 20, 130]
    A.akb_append(c, *(R.tokens(2, H, N - 20, D, F16, s, "plain").to(DEV) for s in (1, 2)), i32(lens))
    parents, upto = [b % 2 for b in range(2 * W)], [N - 64 * b - 1 for b in range(2 * W)]
    d.score.fill_(7.0)
    A.akb_fork(c, d, i32(parents), i32(upto))
    score, L = d.score.view(2 * W, H, N), d.lens.tolist()
    assert L == [min(lens[a], u) for a, u in zip(parents, upto)]
    for b in range(2 * W):
        assert not score[b, :, :L[b]].any() and (score[b, :, L[b]:] == 7.0).all(), b
    d.reserve(1, keep=64)
    A.akb_attention(d, R.tokens(2 * W, H, 1, D, F16, 3, "plain").to(DEV), accumulate=True)
    e, kept = A.BlockCache.allocate(2 * W, H, H, D, 64, F16, score=True), torch.zeros(2 * W, H, 64, dtype=torch.int32, device=DEV)
    A.akb_evict(d, e, 64, 0, kept=kept)
    for b in (0, 2 * W - 1):
        want = score[b, :, :L[b]].sort(dim=1, descending=True, stable=True).indices[:, :64].sort(dim=1).values
        assert torch.equal(kept[b].long(), want)


@pytest.mark.parametrize("dtype", [F16, B16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
def test_copies_that_pass_the_cache_by(A, dtype, D):
    """More than 128 MiB: blocks one at a time, stored with the non-temporal hint."""
    H, N, L = 16, 4096, [4000, 131, 64, 4096]
    c, d = (A.BlockCache.allocate(B, H, H, D, N, dtype, score=True) for B in (4, 18))
    A.akb_append(c, *(R.tokens(4, H, N, D, dtype, s, "plain").to(DEV) for s in (1, 2)), i32(L))
    c.score.copy_(torch.rand(c.score.shape, generator=torch.Generator().manual_seed(3)))
    d.score.fill_(7.0)
    parents, upto = [b % 4 for b in range(18)], [(1 << 30, 4032, 65, 2049, 1)[b % 5] for b in range(18)]
    A.akb_fork(c, d, i32(parents), i32(upto))
    lens = [min(L[a], u) for a, u in zip(parents, upto)]
    assert d.lens.tolist() == lens
    sides, scores = list(zip(A.akb_unpack(c), A.akb_unpack(d))), [x.score.view(x.B, H, N) for x in (c, d)]
    for b, (a, m) in enumerate(zip(parents, lens)):
        for src, dst in sides:
            assert torch.equal(dst[b, :, :m], src[a, :, :m]), b
        assert torch.equal(scores[1][b, :, :m], scores[0][a, :, :m]) and (scores[1][b, :, m:] == 7.0).all(), b


def test_copies_up_to_the_lengths_that_the_destination_had(A):
    """upto may be dst's own lens, which the call moves."""
    c, ref = pair(A, 7, 4, 2, 128, 320, F16)
    put(A, c, ref, 300, 1, LENS)
    d, want = pair(A, 7, 4, 2, 128, 320, F16)
    put(A, d, want, 130, 7, had := [130, 5, 64, 0, 1, 100, 65])
    A.akb_fork(c, d, i32([0, 0, 0, 4, 2, 6, 0]), d.lens)
    S.fork(ref, want, [0, 0, 0, 4, 2, 6, 0], had)
    R.assert_same_tokens(A, d, want)


def test_fork_into_caches_of_other_sizes(A):
    c, ref = pair(A, 2, 2, 2, 64, 1024, F16)
    put(A, c, ref, 1000, 1, [1000, 130])
    d, want = pair(A, 5, 8, 2, 64, 192, F16)
    put(A, d, want, 10, 2)
    parents, upto = [0, 1, 0, 1, 0], [193, 192, 192, 64, 100]
    A.akb_fork(c, d, i32(parents), i32(upto))
    S.fork(ref, want, parents, upto)
    R.assert_same_tokens(A, d, want)
    assert want.refused == 1 and d.flags.cpu().tolist() == [1, 0, 0, 0] + [0] * 5 and not c.flags.any()
    A.akb_fork(c, d, i32([0] * 5))
    S.fork(ref, want, [0] * 5, None)
    R.assert_same_tokens(A, d, want, "all refused")
    assert d.flags.cpu().tolist() == [6, 0, 0, 0] + [0] * 5
    one, alone = pair(A, 1, 2, 2, 64, 1024, F16)   # and one sequence of several
    A.akb_fork(c, one, i32([0]))
    S.fork(ref, alone, [0], None)
    R.assert_same_tokens(A, one, alone, "one")


@pytest.mark.parametrize("dtype,D,Hkv", [(F16, 128, 2), (B16, 64, 1), (B16, 128, 40)])
def test_truncate(A, dtype, D, Hkv):
    lens = [300, 0, 64, 63, 129, 1, 192, 300, 256, 255, 100, 200]
    keep = [299, 5, 63, 62, 64, 0, 192, 20, 255, -7, 1 << 30, 128]
    c, ref = pair(A, 12, Hkv, Hkv, D, 320, dtype, score=True)
    put(A, c, ref, 300, 1, lens)
    scored(c, ref, 5)
    before = c.score.clone()
    A.akb_truncate(c, i32(keep))
    for b, k in enumerate(keep):
        S.cut(ref, b, min(ref.len(b), max(k, 0)))
    R.assert_same_tokens(A, c, ref)
    assert torch.equal(c.score, before) and not c.flags.any()
    put(A, c, ref, 70, 9, kind="wide")
    R.assert_same_tokens(A, c, ref, "with more tokens")
    A.akb_truncate(c, i32([1 << 20] * 12))   # nothing to cut
    R.assert_same_tokens(A, c, ref, "as it was")
    A.akb_truncate(c, c.lens)
    R.assert_same_tokens(A, c, ref, "to its own lengths")
    A.akb_truncate(c, i32([0] * 12))
    assert not c.lens.any()


def test_every_cut_of_two_blocks(A):
    c, ref = pair(A, 130, 1, 1, 64, 192, F16)
    put(A, c, ref, 129, 3)
    A.akb_truncate(c, i32(list(range(130))))
    for b in range(130):
        S.cut(ref, b, min(b, 129))
    R.assert_same_tokens(A, c, ref)


def test_copies_and_cuts_in_a_graph_and_on_another_stream(A):
    c, ref = pair(A, 4, 2, 2, 128, 320, B16)
    put(A, c, ref, 300, 1, [300, 200, 64, 129])
    d, want = pair(A, 4, 2, 2, 128, 320, B16)
    parents, upto, keep = i32([1, 0, 0, 3]), i32([190, 300, 130, 129]), i32([65, 290, 3, 128])

    def step():
        A.akb_fork(c, d, parents, upto)
        A.akb_truncate(d, keep)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        step()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=s):
            step()
    torch.cuda.current_stream().wait_stream(s)
    for turn in range(3):
        if turn:
            put(A, c, ref, 1 + 5 * turn, 50 + turn)
            parents.copy_(i32([turn, 3, 1, 0]))
        d.k_tail.fill_(float("nan"))
        d.lens.zero_()
        graph.replay()
        torch.cuda.synchronize()
        S.fork(ref, want, parents.tolist(), upto.tolist())
        for b, k in enumerate(keep.tolist()):
            S.cut(want, b, min(want.len(b), k))
        R.assert_same_tokens(A, d, want, f"replay {turn}")


def test_offsets_beyond_32_bits(A):
    """The last heads of caches of 9 GB."""
    D, Ncap, H = 128, 1 << 20, 36
    c, d = (A.BlockCache.allocate(1, H, H, D, Ncap, B16) for _ in range(2))
    small = A.BlockCache.allocate(1, H, H, D, 384, B16)
    k, v = (R.tokens(1, H, 333, D, B16, s).to(DEV) for s in (1, 2))
    A.akb_append(c, k, v)
    A.akb_append(small, k, v)
    A.akb_fork(c, d, None, i32([200]))
    A.akb_truncate(c, i32([200]))
    A.akb_truncate(small, i32([200]))
    e = A.BlockCache.allocate(1, H, H, D, 384, B16)
    for src in (c, d):
        A.akb_fork(src, e)
        assert all(torch.equal(a, b) for a, b in zip(A.akb_unpack(e), A.akb_unpack(small)))
