"""Parts of two row tiles that the last workgroup of a row group joins: every split of the work among its threads (rows x channels of a group: more than its
threads, as many, fewer in 2, 4, 8 slices), against 64 bits."""
import pytest
import torch

from test_gpu_block_cache_range import A, DEV, B16, F16, F32, check, i32  # noqa: F401  (A is a fixture)

pytestmark = pytest.mark.gpu

# kernel, parts, join; D, B, Hq, Hkv, tokens, n, query tokens of the sequences
JOINS = [
    ((2, 2, 2), 128, 32, 32, 8, 4096, 5, "all"),        # 20 rows
    ((2, 2, 2), 64, 32, 32, 8, 1500, 5, "ragged"),      # ... 0 to 20 of them
    ((2, 3, 2), 128, 24, 32, 8, 2000, 5, "ragged"),     # three parts
    ((2, 3, 2), 64, 24, 24, 8, 2000, 7, "all"),         # 21 rows, groups of three
    ((2, 2, 2), 128, 16, 32, 8, 2000, 10, "all"),       # a second row group of 8 rows
    ((2, 2, 2), 64, 16, 32, 8, 2000, 10, "all"),
    ((2, 2, 2), 128, 16, 8, 8, 1100, 33, "all"),        # ... of one
    ((2, 2, 2), 64, 16, 8, 8, 1100, 33, "ragged"),
    ((2, 2, 2), 128, 16, 32, 8, 1030, 9, "all"),        # ... of four
    ((2, 2, 2), 64, 16, 32, 8, 1030, 9, "ragged"),
    ((2, 2, 2), 128, 16, 32, 8, 1030, 16, "all"),       # two whole groups
]


@pytest.mark.parametrize("dtype,out_dtype", [(F16, F32), (F16, F16), (B16, F32), (B16, B16)], ids=["fp16-f32", "fp16", "bf16-f32", "bf16"])
@pytest.mark.parametrize("case", JOINS, ids=lambda c: f"parts{c[0][1]}-D{c[1]}-B{c[2]}-H{c[3]}_{c[4]}-N{c[5]}-n{c[6]}-{c[7]}")
def test_parts_joined_by_the_last_workgroup(A, case, dtype, out_dtype):  # noqa: F811
    (path, parts, how), D, B, Hq, Hkv, N, n, which = case
    Ncap = (N + 63) // 64 * 64
    print(case, flush=True)
    assert (*A.akb_attention_path(B, Hq, Hkv, D, Ncap, n), A.akb_attention_join(B, Hq, Hkv, D, Ncap, n)) == (path, parts, how)
    g = torch.Generator(device=DEV).manual_seed(N + n)
    c = A.BlockCache.allocate(B, Hq, Hkv, D, Ncap, dtype, score=True, n=n)
    lens = [max(1, N - b * (N // B)) for b in range(B)]
    n_q = None if which == "all" else [(5 * b) % (n + 1) for b in range(B)]
    A.akb_append(c, *(torch.randn(B, Hkv, N, D, generator=g, device=DEV).to(dtype) for _ in range(2)), i32(lens))
    q = torch.randn(B, Hq, n, D, generator=g, device=DEV).to(dtype)
    start = torch.rand(c.score.shape, generator=g, device=DEV)
    runs = []
    for _ in range(2):   # the second finds the tickets that the first has left
        c.score.copy_(start)
        out = torch.full(q.shape, 3.0, dtype=out_dtype, device=DEV)
        A.akb_attention(c, q, out, n_q=i32(n_q), accumulate=True)
        runs.append((out, c.score.clone()))
    assert all(torch.equal(a, b) for a, b in zip(*runs))
    K, V = A.akb_unpack(c)
    check(c, q, out, K, V, lens, n_q, start, tiny=2.0 ** -25 if out_dtype == F16 else 0.0)
    if n_q is not None:
        assert all((out[b, :, m:].float() == 3.0).all() for b, m in enumerate(n_q))
