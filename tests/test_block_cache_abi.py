"""The block-scaled cache's C ABI without a GPU: the header and the binding name the same, sizes are host computations, and calls that cannot be served are
refused before anything is launched."""
import ctypes as C
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ADDR = {n: 0x1000000 * (i + 1) for i, n in enumerate(("k8", "v8", "exps", "k_tail", "v_tail", "score", "lens", "flags"))}
Q, OUT, WS = 0x20000000, 0x30000000, 0x40000000


@pytest.fixture(scope="module")
def A():
    from paper_2409_16546_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2409_16546_amd import build
        build.build_library(verbose=False)
    return binding


@pytest.fixture(scope="module")
def header():
    return re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "akb.h")).read(), flags=re.S)


def test_header_and_binding_name_the_same(A, header):
    names = sorted(set(re.findall(r"\b(akb_[a-z0-9_]+)\s*\(", header)))
    assert names == sorted(A.AKB_EXPORTS)
    for n in names:
        assert getattr(A.lib(), n) is not None
    for struct, cls in (("akb_shape", A.akb_shape), ("akb_cache", A.akb_cache), ("akb_sizes", A.akb_sizes), ("akb_params", A.akb_params)):
        body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (struct, struct), header, flags=re.S).group(1)
        fields = [d.replace("*", " ").split()[-1] for line in body.split(";") if line.strip() for d in line.split(",")]
        assert fields == [f[0] for f in cls._fields_], struct
    assert re.search(r"#define AKB_TB (\d+)", header).group(1) == str(A.AKB_TB) and re.search(r"#define AKB_MAX_G (\d+)", header).group(1) == str(A.AKB_MAX_G)


def test_sizes(A):
    sz = A.akb_layout_sizes(3, 12, 4, 64, 640, torch.bfloat16)
    e = 3 * 4 * 640 * 64
    assert (sz.k8, sz.v8, sz.exps, sz.k_tail, sz.v_tail) == (e, e, 3 * 4 * 10 * 2, 3 * 4 * 64 * 64 * 2, 3 * 4 * 64 * 64 * 2)
    assert (sz.score, sz.lens, sz.flags) == (3 * 4 * 640 * 4, 12, (4 + 3) * 4)
    big = A.akb_layout_sizes(64, 128, 8, 128, 1 << 20)
    assert big.k8 == 64 * 8 * 128 << 20


def test_workspace_of_n_serves_every_smaller_call(A):
    L = A.lib()
    for shape in ((1, 32, 32, 128, 1024, 0), (4, 64, 8, 128, 13056, 1), (200, 16, 1, 64, 4096, 0)):
        s = A.akb_shape(*shape)
        for acc in (0, 1):
            sizes = [L.akb_attention_workspace(C.byref(s), n, acc) for n in (1, 2, 5, 17, 64, 300, 1024)]
            assert sizes == sorted(sizes) and sizes[0] > 0 and all(x % 256 == 0 for x in sizes)
    assert L.akb_evict_workspace(C.byref(s), 100) >= 200 * 100 * 4
    assert L.akb_attention_workspace(C.byref(s), 4097, 0) == 0 and L.akb_evict_workspace(C.byref(s), 0) == 0


@pytest.mark.parametrize("shape", [(0, 4, 4, 128, 64), (1, 4, 3, 128, 64), (1, 4, 4, 96, 64), (1, 4, 4, 128, 100), (1, 34, 2, 128, 64), (1, 4, 4, 128, 0),
                                   (65536, 1, 1, 64, 64), (1, 1, 1, 64, (1 << 22) + 64)])
def test_bad_shapes_are_refused(A, shape):
    with pytest.raises(A.AkvError) as e:
        A.akb_layout_sizes(*shape)
    assert e.value.status == A.AKV_EINVAL and "bad shape" in str(e.value)


def test_refusals_come_before_any_launch(A):
    # the addresses are made up: every call below is turned away by the host
    L = A.lib()
    shape = A.akb_shape(2, 8, 4, 128, 256, 0)
    good = A.akb_cache(shape, **ADDR)
    r = C.byref

    def refused(st, word, status=A.AKV_EINVAL):
        assert st == status and word in L.akv_last_error().decode(), L.akv_last_error()

    def cache(**kw):
        return A.akb_cache(shape, **{**ADDR, **kw})

    for name in ("k8", "v8", "exps", "k_tail", "v_tail", "lens", "flags"):
        refused(L.akb_append(r(cache(**{name: None})), Q, Q, None, 1, None), "NULL")
    for name in ("k8", "v_tail", "score", "exps"):
        refused(L.akb_cache_reset(r(cache(**{name: ADDR[name] + 8})), None), "aligned")
    refused(L.akb_append(None, Q, Q, None, 1, None), "NULL")
    refused(L.akb_append(r(good), Q, None, None, 1, None), "NULL")
    refused(L.akb_append(r(good), Q + 2, Q, None, 1, None), "aligned")
    refused(L.akb_append(r(good), Q, Q, Q + 2, 1, None), "aligned")
    refused(L.akb_append(r(good), Q, Q, None, 257, None), "out of range")
    refused(L.akb_append(r(good), Q, Q, None, -1, None), "out of range")
    assert L.akb_append(r(good), None, None, None, 0, None) == A.AKV_OK

    def attention(c=good, q=Q, n_q=None, n=1, out=OUT, p=None, ws=WS, size=1 << 30):
        return L.akb_attention(r(c), q, n_q, n, out, r(p) if p else None, ws, size, None)
    refused(attention(q=None), "NULL")
    refused(attention(out=OUT + 8), "aligned")
    refused(attention(q=Q + 2), "aligned")
    refused(attention(n_q=Q + 1), "aligned")
    refused(attention(n=257), "out of range")
    refused(attention(p=A.akb_params(0.0, 2, 0, 0)), "out_dtype")
    refused(attention(p=A.akb_params(0.0, 0, 0, 257)), "max_len")
    refused(attention(p=A.akb_params(float("nan"), 0, 0, 0)), "scale")
    refused(attention(p=A.akb_params(float("inf"), 0, 0, 0)), "scale")
    refused(attention(c=cache(score=None), p=A.akb_params(0.0, 0, 1, 0)), "score")
    refused(attention(ws=WS + 16), "aligned", A.AKV_EWORKSPACE)
    refused(attention(ws=None), "needed", A.AKV_EWORKSPACE)
    refused(attention(size=64), "needed", A.AKV_EWORKSPACE)
    assert attention(n=0, q=None, out=None, ws=None) == A.AKV_OK
    many = A.akb_cache(A.akb_shape(128, 64, 4, 64, 1 << 18, 0), **ADDR)
    refused(attention(c=many, n=1 << 17, size=1 << 50), "2^24")

    assert L.akb_workspace_init(None, 1 << 20, None) == A.AKV_EWORKSPACE and L.akb_workspace_init(WS + 8, 1 << 20, None) == A.AKV_EWORKSPACE
    assert L.akb_workspace_init(WS, 16, None) == A.AKV_EWORKSPACE

    to = {n: a + 0x100000000 for n, a in ADDR.items()}

    def evict(src=good, dst=None, keep=100, recent=0, kept=Q, ws=None, size=0, dshape=shape):
        return L.akb_evict(r(src), r(dst or A.akb_cache(dshape, **to)), keep, recent, kept, ws, size, None)
    refused(evict(src=cache(score=None)), "score")
    refused(evict(keep=0), "keep")
    refused(evict(keep=257), "keep")
    refused(evict(recent=101), "recent")
    refused(evict(recent=-1), "recent")
    refused(evict(kept=Q + 1), "aligned")
    refused(evict(kept=None), "needed", A.AKV_EWORKSPACE)
    refused(evict(kept=None, ws=WS + 4, size=1 << 20), "aligned", A.AKV_EWORKSPACE)
    for other in ((3, 8, 4, 128, 256, 0), (2, 8, 2, 128, 256, 0), (2, 8, 4, 64, 256, 0), (2, 8, 4, 128, 256, 1)):
        refused(evict(dshape=A.akb_shape(*other)), "differ")
    refused(evict(dst=good), "share memory")
    refused(evict(dst=A.akb_cache(shape, **{**to, "v8": ADDR["score"]})), "share memory")
    refused(L.akb_unpack(r(good), Q + 4, None, None), "aligned")
    assert L.akb_unpack(r(good), None, None, None) == A.AKV_OK


def test_attention_path_is_a_host_computation_and_the_gpu_cases_reach_what_they_name(A):
    from test_gpu_block_cache import LARGE
    for case in LARGE:   # 256 compute units are assumed where no device can be asked
        path, _, _, D, B, Hq, Hkv, N, _, n, _ = case
        assert A.akb_attention_path(B, Hq, Hkv, D, (N + 63) // 64 * 64, n) == path, case
    assert {c[0][0] for c in LARGE} == {1, 2, 3}
    assert A.akb_attention_path(1, 6, 4, 64, 64)[0] == 0 and A.akb_attention_path(1, 4, 4, 64, 64, 65)[0] == 0 and A.akb_attention_path(1, 4, 4, 64, 64, 1, 65)[0] == 0
    assert A.akb_attention_path(1, 32, 32, 128, 1024, 1, 64) == (1, 1)          # a bound of the lengths: one part
    # the lines: 16 rows, 64 rows, 12 blocks a part
    assert [A.akb_attention_path(8, 32, 8, 128, 8192, n)[0] for n in (4, 5, 16, 17)] == [1, 2, 2, 3]
    assert A.akb_attention_path(8, 32, 8, 128, 2048, 17)[0] == 2


def test_binding_checks_types_and_shapes(A):
    sz = A.akb_layout_sizes(1, 2, 2, 64, 64, torch.float16)
    t = lambda n, dt: torch.zeros(getattr(sz, n) // torch.empty(0, dtype=dt).element_size(), dtype=dt)
    parts = dict(k8=t("k8", torch.uint8), v8=t("v8", torch.uint8), exps=t("exps", torch.int8), k_tail=t("k_tail", torch.float16), v_tail=t("v_tail", torch.float16),
                 lens=t("lens", torch.int32), flags=t("flags", torch.int32))
    c = A.BlockCache(1, 2, 2, 64, 64, torch.float16, **parts)
    with pytest.raises(AssertionError):
        A.BlockCache(1, 2, 2, 64, 128, torch.float16, **parts)                                    # too small
    with pytest.raises(AssertionError):
        A.BlockCache(1, 2, 2, 64, 64, torch.bfloat16, **parts)                                    # tails of the other type
    x = torch.zeros(1, 2, 1, 64, dtype=torch.float16)
    with pytest.raises(AssertionError):
        A.akb_append(c, x.float(), x.float())
    with pytest.raises(AssertionError):
        A.akb_append(c, x[:, :1], x[:, :1])
    with pytest.raises(AssertionError):
        A.akb_attention(c, x.bfloat16())
    with pytest.raises(AssertionError):
        A.akb_evict(c, c, 5, kept=torch.zeros(1, 2, 4, dtype=torch.int32))
