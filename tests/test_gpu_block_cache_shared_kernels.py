"""Attention behind shared prefixes by every kernel that there is: each type, result, head size, and kind of walks; against 64 bits on the GPU."""
import pytest

from test_gpu_block_cache_shared import A, B16, F16, F32, test_large_calls as large_call  # noqa: F401

pytestmark = pytest.mark.gpu

FORMS = [  # prefixes, sequences, Hq, Hkv, P, N, n
    (2, 8, 16, 4, 700, 130, 1),      # row walks over prefixes, one tile of own rows
    (2, 8, 16, 4, 700, 130, 6),      # ... two
    (8, 560, 32, 8, 150, 70, 1),     # prompt walks over prefixes, one tile
    (8, 88, 64, 8, 230, 70, 3),      # ... two
    (2, 6, 16, 4, 500, 333, 50),     # one walk over both, cut
    (1, 40, 32, 8, 100, 129, 129),   # ... whole
]
KERNELS = [(dtype, out, D, *form) for dtype in (F16, B16) for out in (F32, dtype) for D in (64, 128) for form in FORMS]


@pytest.mark.parametrize("case", KERNELS, ids=lambda c: f"{str(c[0])[6:]}-{str(c[1])[6:]}-D{c[2]}-B{c[3]}_{c[4]}-H{c[5]}_{c[6]}-P{c[7]}-N{c[8]}-n{c[9]}")
@pytest.mark.parametrize("ragged", [False, True], ids=["", "ragged"])
def test_every_kernel(A, case, ragged):
    large_call(A, case, ragged)
