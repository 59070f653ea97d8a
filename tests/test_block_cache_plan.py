"""How calls of the block-scaled cache's attention are cut, without a GPU (256 compute units are assumed where no device can be asked): the parts of every call fit the
workspace, and the GPU tests reach every kernel with every way its parts are put together."""
import ctypes as C
import os
import random

import pytest

SLOTS = 512                        # workgroups at a time: two per compute unit
GROUP_ROWS = {1: 16, 2: 32, 3: 128}


@pytest.fixture(scope="module")
def A():
    from paper_2409_16546_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2409_16546_amd import build
        build.build_library(verbose=False)
    return binding


def part_floats(rows, D):
    return (2 * rows + 3) // 4 * 4 + rows * D


def device_cut(blocks, walks):
    """Parts of a walk of each sequence where the device cuts by the lengths (blocks of each sequence, walks per sequence)."""
    most = SLOTS - len(blocks) * walks
    q = max(4, -(-sum(blocks) * walks // most))
    return [max(-(-nb // q), 1) for nb in blocks]


def shapes(rng):
    for _ in range(20000):
        G, D = rng.choice([1, 2, 3, 4, 5, 7, 8, 11, 16]), rng.choice([64, 128])
        Hkv, B = rng.choice([1, 2, 3, 4, 7, 8, 16, 32, 64]), int(2 ** rng.uniform(0, 9))
        Ncap = 64 * int(2 ** rng.uniform(0, 16))
        n = min(Ncap, int(2 ** rng.uniform(0, 13)))
        yield B, Hkv * G, Hkv, D, Ncap, n, rng.choice([0, rng.randint(1, Ncap)])
    for items in range(1, 600):    # every number of walks, long ones: the lines of the number of parts
        for G, n in ((1, 1), (4, 5), (4, 33)):
            yield items, G, 1, 128, 1 << 16, n, 0


def test_the_parts_of_every_call_fit_the_workspace(A):
    rng = random.Random(5)
    L = A.lib()
    seen = set()
    for B, Hq, Hkv, D, Ncap, n, max_len in shapes(rng):
        path, parts = A.akb_attention_path(B, Hq, Hkv, D, Ncap, n, max_len)
        how = A.akb_attention_join(B, Hq, Hkv, D, Ncap, n, max_len)
        rows = n * (Hq // Hkv)
        group = min(rows, GROUP_ROWS[path])
        groups = -(-rows // GROUP_ROWS[path])
        items = B * Hkv * groups
        what = (B, Hq, Hkv, D, Ncap, n, max_len, path, parts, how)
        assert (how == 1) == (parts == 1) and how in (1, 2, 3), what
        shape = A.akb_shape(B, Hq, Hkv, D, Ncap, 0)
        room = L.akb_attention_workspace(C.byref(shape), n, 0)
        if parts > 1:
            total = items * parts
        elif parts == 0:
            assert B <= 256 and items * 4 <= SLOTS, what
            walks, total = Hkv * groups, 0
            for lens in ([Ncap] * B, [1] * B, [0] * (B - 1) + [Ncap], [rng.randint(0, Ncap) for _ in range(B)], [int(Ncap ** rng.random()) for _ in range(B)]):
                cut = device_cut([-(-x // 64) for x in lens], walks)
                assert sum(cut) * walks <= SLOTS, what
                total = max(total, sum(cut) * walks)
        else:
            total = 0
        assert total <= 2 * SLOTS, what                                      # the tickets and parts that a workspace holds
        assert 2 * SLOTS * 4 + total * part_floats(group, D) * 4 <= room, what
        seen.add((path, min(parts, 2), how))
    assert seen == {(1, 1, 1), (1, 2, 2), (1, 2, 3), (1, 0, 2), (1, 0, 3), (2, 1, 1), (2, 2, 2), (2, 2, 3), (2, 0, 3), (3, 1, 1), (3, 2, 3), (3, 0, 3)}, seen


def test_a_workspace_for_n_and_its_scores_serves_every_smaller_call(A):
    rng = random.Random(6)
    L = A.lib()
    for B, Hq, Hkv, D, Ncap, n, _ in shapes(rng):
        shape = A.akb_shape(B, Hq, Hkv, D, Ncap, 1)
        for less in {1, max(1, n // 2), max(1, n - 1)}:
            assert L.akb_attention_workspace(C.byref(shape), less, 1) <= L.akb_attention_workspace(C.byref(shape), n, 1), (B, Hq, Hkv, D, Ncap, n, less)


def test_the_gpu_tests_reach_every_kernel_and_join(A):
    from test_gpu_block_cache import LARGE
    from test_gpu_block_cache_joins import JOINS
    reached = set()
    for case in LARGE:
        (path, parts), _, _, D, B, Hq, Hkv, N, _, n, _ = case
        reached.add((path, min(parts, 2), A.akb_attention_join(B, Hq, Hkv, D, (N + 63) // 64 * 64, n)))
    for (path, parts, how), D, B, Hq, Hkv, N, n, _ in JOINS:
        args = (B, Hq, Hkv, D, (N + 63) // 64 * 64, n)
        assert (*A.akb_attention_path(*args), A.akb_attention_join(*args)) == (path, parts, how), args
        reached.add((path, min(parts, 2), how))
    assert reached == {(1, 1, 1), (1, 2, 2), (1, 2, 3), (1, 0, 2), (1, 0, 3), (2, 1, 1), (2, 2, 2), (2, 2, 3), (2, 0, 3), (3, 1, 1), (3, 2, 3), (3, 0, 3)}, reached


def test_join_query_refuses_what_the_path_query_refuses(A):
    assert A.akb_attention_join(1, 6, 4, 64, 64) == 0 and A.akb_attention_join(1, 4, 4, 64, 64, 65) == 0 and A.akb_attention_join(1, 4, 4, 64, 64, 0) == 0
    assert A.akb_attention_join(1, 4, 4, 64, 64, 1, 65) == 0 and A.akb_attention_join(1, 4, 4, 64, 64, 1, -1) == 0
    assert A.akb_attention_join(1, 32, 32, 128, 1024, 1) == 2 and A.akb_attention_join(1, 32, 32, 128, 1024, 1, 64) == 1
