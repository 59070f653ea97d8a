"""Shared prefixes, rotated appends, copies and cuts without a GPU: structs and names, workspaces, which kernels a call takes, and calls that are refused before anything is launched."""
import ctypes as C
import os
import random
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = ("k8", "v8", "exps", "k_tail", "v_tail", "score", "lens", "flags")
ADDR = {n: 0x1000000 * (i + 1) for i, n in enumerate(NAMES)}
OTHER = {n: a + 0x100000000 for n, a in ADDR.items()}
Q, OUT, WS, X = 0x20000000, 0x30000000, 0x40000000, 0x50000000


@pytest.fixture(scope="module")
def A():
    from paper_2409_16546_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2409_16546_amd import build
        build.build_library(verbose=False)
    return binding


@pytest.fixture
def refused(A):
    def check(st, word, status=None):
        assert st == (A.AKV_EINVAL if status is None else status) and word in A.lib().akv_last_error().decode(), A.lib().akv_last_error()
    return check


def test_structs_are_the_headers(A):
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "akb.h")).read(), flags=re.S)
    for struct, cls in (("akb_rotary", A.akb_rotary), ("akb_tokens", A.akb_tokens)):
        body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (struct, struct), header, flags=re.S).group(1)
        fields = [d.replace("*", " ").split()[-1] for line in body.split(";") if line.strip() for d in line.split(",")]
        assert fields == [f[0] for f in cls._fields_], struct


def test_shared_attention_is_refused(A, refused):
    L, r = A.lib(), C.byref
    shape, of = (6, 8, 4, 128, 256, 0), (2, 8, 4, 128, 512, 0)
    good, prefix = A.akb_cache(A.akb_shape(*shape), **ADDR), A.akb_cache(A.akb_shape(*of), **OTHER)

    def call(p=prefix, c=good, q=Q, n_q=None, n=1, out=OUT, par=None, pmax=0, ws=WS, size=1 << 40):
        return L.akb_attention_shared(r(p) if p else None, r(c), q, n_q, n, out, r(par) if par else None, pmax, ws, size, None)
    refused(call(p=None), "NULL")
    refused(call(p=A.akb_cache(A.akb_shape(*of), **{**OTHER, "v8": None})), "NULL")
    for other in ((4, 8, 4, 128, 512, 0), (12, 8, 4, 128, 512, 0), (2, 4, 4, 128, 512, 0), (2, 8, 2, 128, 512, 0), (2, 8, 4, 64, 512, 0), (2, 8, 4, 128, 512, 1)):
        refused(call(p=A.akb_cache(A.akb_shape(*other), **OTHER)), "go together")
        assert L.akb_attention_shared_workspace(r(A.akb_shape(*other)), r(A.akb_shape(*shape)), 1) == 0
        assert L.akb_attention_shared_path(r(A.akb_shape(*other)), r(A.akb_shape(*shape)), 1, 0, 0, None) == 0
    refused(call(par=A.akb_params(0.0, 0, 1, 0)), "accumulate")
    refused(call(par=A.akb_params(0.0, 2, 0, 0)), "out_dtype")
    refused(call(par=A.akb_params(0.0, 0, 0, 257)), "max_len")
    refused(call(par=A.akb_params(float("nan"), 0, 0, 0)), "scale")
    refused(call(pmax=513), "prefix_max_len")
    refused(call(pmax=-1), "prefix_max_len")
    refused(call(n=257), "out of range")
    refused(call(n=-1), "out of range")
    refused(call(q=None), "NULL")
    refused(call(out=OUT + 4), "aligned")
    refused(call(q=Q + 8), "aligned")
    refused(call(n_q=Q + 2), "aligned")
    refused(call(ws=None), "needed", A.AKV_EWORKSPACE)
    refused(call(ws=WS + 16), "aligned", A.AKV_EWORKSPACE)
    need = L.akb_attention_shared_workspace(r(A.akb_shape(*of)), r(A.akb_shape(*shape)), 1)
    refused(call(size=need - 1), "needed", A.AKV_EWORKSPACE)
    assert call(n=0, q=None, out=None, ws=None) == A.AKV_OK
    for bad in ((None, A.akb_shape(*shape), 1), (A.akb_shape(*of), A.akb_shape(*shape), 257), (A.akb_shape(*of), A.akb_shape(*shape), -1)):
        assert L.akb_attention_shared_workspace(r(bad[0]) if bad[0] else None, r(bad[1]), bad[2]) == 0
    for n, ml, pm in ((0, 0, 0), (257, 0, 0), (1, 257, 0), (1, -1, 0), (1, 0, 513), (1, 0, -1)):
        assert L.akb_attention_shared_path(r(A.akb_shape(*of)), r(A.akb_shape(*shape)), n, ml, pm, None) == 0


def part_floats(rows, D):
    return (2 * rows + 3) // 4 * 4 + rows * D


def test_the_parts_of_every_call_fit_a_workspace_for_as_many_tokens_or_more(A):
    """256 compute units are assumed where no device can be asked."""
    rng, L, seen = random.Random(7), A.lib(), set()
    for _ in range(20000):
        G, D, Hkv, Bp = rng.choice([1, 2, 3, 4, 5, 8, 11, 16]), rng.choice([64, 128]), rng.choice([1, 2, 3, 8, 32, 64]), int(2 ** rng.uniform(0, 5))
        W, P, N = int(2 ** rng.uniform(0, 8)), 64 * int(2 ** rng.uniform(0, 14)), 64 * int(2 ** rng.uniform(0, 12))
        n = min(N, int(2 ** rng.uniform(0, 9)))
        args = (Bp, Bp * W, Hkv * G, Hkv, D, P, N, n, rng.choice([0, rng.randint(1, N)]), rng.choice([0, rng.randint(1, P)]))
        path, *parts = A.akb_attention_shared_path(*args)
        assert (path == 3) == (n * G >= 96) and min(parts) >= 1, args
        shapes = A.akb_shape(Bp, Hkv * G, Hkv, D, P, 0), A.akb_shape(Bp * W, Hkv * G, Hkv, D, N, 0)
        floats = 0
        if path == 3:
            walks = Bp * W * Hkv * -(-n * G // 128)
            assert parts[0] == parts[1] and (parts[0] == 1 or walks * parts[0] <= 1024), args
            floats = walks * parts[0] * part_floats(min(n * G, 128), D) if parts[0] > 1 else 0
        else:
            for i, (pairs, rows) in enumerate(((Bp * Hkv, W * n * G), (Bp * W * Hkv, n * G))):
                tile = 128 if i == 0 and path == 2 else (16 if i == 1 and rows <= 16 else 32)
                walks = pairs * -(-rows // tile)
                assert parts[i] == 1 or walks * parts[i] <= 1024, args
                floats += walks * parts[i] * part_floats(tile, D)
        for more in (n, min(N, n + rng.randint(0, 5)), min(N, 2 * n), N):
            room = L.akb_attention_shared_workspace(C.byref(shapes[0]), C.byref(shapes[1]), more)
            assert room % 256 == 0 and 4 * floats + 3 * 256 <= room, (args, more)
        seen.add((path, parts[0] > 1, parts[1] > 1))
    assert seen == {(1, a, b) for a in (False, True) for b in (False, True)} | {(2, False, False), (2, True, False), (3, False, False), (3, True, True)}, seen


def test_the_gpu_tests_reach_every_kernel(A):
    from test_gpu_block_cache_shared import CASES, LARGE
    up, seen = lambda x: (max(x, 1) + 63) // 64 * 64, set()
    for _, out, D, Bp, B, Hq, Hkv, P, N, n in LARGE:
        path, a, b = A.akb_attention_shared_path(Bp, B, Hq, Hkv, D, up(P), up(N), n)
        seen.add((path, a > 1, b > 1, path < 3 and n * (Hq // Hkv) > 16))
    for _, out, D, Hq, Hkv, first, lens, n, _ in CASES:
        path, a, b = A.akb_attention_shared_path(len(first), len(lens), Hq, Hkv, D, up(max(first)), max(up(max(lens)), up(n)), n)
        seen.add((path, a > 1, b > 1, path < 3 and n * (Hq // Hkv) > 16))
    assert {s[0] for s in seen} == {1, 2, 3} and {s[1] for s in seen} == {s[2] for s in seen} == {s[3] for s in seen} == {False, True}, seen
    assert {(s[0], s[3]) for s in seen} == {(1, False), (1, True), (2, False), (2, True), (3, False)}, seen


def test_the_gpu_tests_reach_every_kernel_of_shared_attention(A):
    from test_gpu_block_cache_shared_kernels import FORMS, KERNELS
    up, ways = lambda x: (x + 63) // 64 * 64, []
    for Bp, B, Hq, Hkv, P, N, n in FORMS:
        for D in (64, 128):
            path, a, _ = A.akb_attention_shared_path(Bp, B, Hq, Hkv, D, up(P), up(N), n)
            ways.append((D, path, a > 1 if path == 3 else n * (Hq // Hkv) > 16))
    assert set(ways) == {(D, path, x) for D in (64, 128) for path in (1, 2, 3) for x in (False, True)}
    assert len(KERNELS) == 2 * 2 * len(ways)   # each of them in both types, with both results


def test_the_gpu_tests_reach_every_rotated_append(A):
    """Each kernel (type, head size, order of pairs, past the last-level cache or not) and each way to share a call out, with lengths moved by either means where both occur."""
    from test_gpu_block_cache_rotated_paths import LENS, PATHS
    kernels, ways = set(), set()
    for dtype, D, B, Hq, Hkv, n, _, _, _, pairs in PATHS:
        path, streamed, ticketed = A.akb_append_rotated_path(B, Hq, Hkv, D, (max(LENS) + n + 63) // 64 * 64, n)
        kernels.add((dtype, D, pairs, streamed))
        ways.add((D, path, streamed))
        ways.add((path, ticketed))
        if path == 3:
            ways.add((D, "apart", -(-Hq // Hkv // 4), Hq // Hkv % 4 == 0))
    both = (False, True)
    assert kernels == {(t, D, p, s) for t in (torch.float16, torch.bfloat16) for D in (64, 128) for p in both for s in both}
    assert ways >= {(D, path, s) for D in (64, 128) for path in (1, 2, 3) for s in both} | {(path, t) for path in (1, 2, 3) for t in both}, ways
    assert {w[2:] for w in ways if w[:2] == (128, "apart")} >= {(2, False), (2, True), (3, False), (4, True)} and len({w for w in ways if w[:2] == (64, "apart")}) >= 3, ways
    good = (6, 8, 4, 128, 256)
    assert A.akb_append_rotated_path(*good, 1)[0] == 1 and A.akb_append_rotated_path(*good, 9, False)[0] == 2
    for bad in ((*good, 0), (*good, 257), (6, 8, 3, 128, 256, 1), (1, 256, 256, 64, 1 << 22, 1 << 22)):
        assert A.akb_append_rotated_path(*bad)[0] == 0, bad


def test_rotated_append_is_refused(A, refused):
    L, r = A.lib(), C.byref
    shape = A.akb_shape(6, 8, 4, 128, 256, 0)
    good = A.akb_cache(shape, **ADDR)
    token = 16 * 128

    def call(c=good, n=2, n_new=None, q_out=OUT, no=(), **kw):
        tokens = dict(q=X, k=X + 8 * 256, v=X + 12 * 256, q_seq=2 * token, q_token=token, k_seq=2 * token, k_token=token, v_seq=2 * token, v_token=token, **{})
        turn = dict(q_norm=Q, k_norm=Q, inv_freq=Q, base=Q, n_base=3, rot=128, pairs=0, eps=1e-6)
        for k, v in kw.items():
            (tokens if k in tokens else turn)[k] = v
        return L.akb_append_rotated(r(c), None if "tokens" in no else r(A.akb_tokens(**tokens)), n_new, n, q_out, None if "rotary" in no else r(A.akb_rotary(**turn)), None)
    refused(call(no=("tokens",)), "NULL")
    refused(call(no=("rotary",)), "NULL")
    refused(call(c=A.akb_cache(shape, **{**ADDR, "k_tail": None})), "NULL")
    refused(call(n=257), "out of range")
    refused(call(n=-1), "out of range")
    for rot in (-16, 8, 24, 144):
        refused(call(rot=rot), "multiple of 16")
    refused(call(inv_freq=None), "inv_freq")
    for n_base in (0, -1, 4, 12):
        refused(call(n_base=n_base), "n_base")
    for eps in (-1.0, float("nan"), float("inf")):
        refused(call(eps=eps), "eps")
    refused(call(k=None), "NULL")
    refused(call(v=None), "NULL")
    refused(call(q=None), "NULL")
    refused(call(q_out=None), "NULL")
    for name in ("q", "k", "v"):
        refused(call(**{name: X + 8}), "aligned")
    refused(call(q_out=OUT + 8), "aligned")
    refused(call(q_norm=Q + 8), "aligned")
    refused(call(k_norm=Q + 2), "aligned")
    refused(call(inv_freq=Q + 2), "aligned")
    refused(call(base=Q + 1), "aligned")
    refused(call(n_new=Q + 1), "aligned")
    for name in ("q_seq", "k_token", "v_seq"):
        refused(call(**{name: token + 4}), "strides")
        refused(call(**{name: -token}), "strides")
    refused(call(q_out=X), "shares memory")
    refused(call(q_out=X + 2 * token * 6 * 2 - 16), "shares memory")
    assert call(n=0, k=None, v=None, q=None) == A.AKV_OK
    wide = A.akb_cache(A.akb_shape(1, 256, 256, 64, 1 << 22, 0), **ADDR)
    refused(call(c=wide, n=1 << 22, rot=64, n_base=1), "2^23")


def test_places_and_parents_in_lengths_that_a_call_moves_are_refused(A, refused):
    """Workgroups read them after others may have moved the lengths."""
    L, r = A.lib(), C.byref
    shape = A.akb_shape(6, 8, 4, 128, 256, 0)
    cache, to = A.akb_cache(shape, **ADDR), A.akb_cache(shape, **OTHER)
    tokens = A.akb_tokens(X, X, X, 4096, 2048, 4096, 2048, 4096, 2048)
    for base, n_base in ((ADDR["lens"], 6), (ADDR["lens"] + 20, 1), (ADDR["lens"] - 4, 2)):
        refused(L.akb_append_rotated(r(cache), r(tokens), None, 2, OUT, r(A.akb_rotary(None, None, Q, base, n_base, 128, 0, 0.0)), None), "base shares memory")
    for parents in (OTHER["lens"], OTHER["lens"] + 20, OTHER["lens"] - 20):
        refused(L.akb_fork(r(cache), r(to), parents, None, None), "parents shares memory")


def test_copies_and_cuts_are_refused(A, refused):
    L, r = A.lib(), C.byref
    shape = (2, 8, 4, 128, 256, 0)
    src = A.akb_cache(A.akb_shape(*shape), **ADDR)

    def fork(s=src, d=None, dshape=shape, parents=Q, upto=None, **kw):
        return L.akb_fork(r(s) if s else None, r(d or A.akb_cache(A.akb_shape(*dshape), **{**OTHER, **kw})), parents, upto, None)
    refused(fork(s=None), "NULL")
    refused(fork(lens=None), "NULL")
    for other in ((2, 8, 2, 128, 256, 0), (2, 8, 4, 64, 256, 0), (2, 8, 4, 128, 256, 1)):
        refused(fork(dshape=other), "differ")
    refused(fork(dshape=(3, 8, 4, 128, 256, 0), parents=None), "parents")
    refused(fork(parents=Q + 2), "aligned")
    refused(fork(upto=Q + 1), "aligned")
    refused(fork(d=src), "share memory")
    refused(fork(v8=ADDR["k8"] + 1024), "share memory")
    refused(fork(score=ADDR["lens"] - 1024), "share memory")
    refused(L.akb_truncate(r(src), None, None), "NULL")
    refused(L.akb_truncate(r(src), Q + 2, None), "aligned")
    refused(L.akb_truncate(r(A.akb_cache(A.akb_shape(*shape), **{**ADDR, "k8": ADDR["k8"] + 8})), Q, None), "aligned")


def test_binding_checks_types_and_shapes(A, monkeypatch):
    sz = A.akb_layout_sizes(2, 4, 2, 64, 64, torch.float16)
    t = lambda n, dt: torch.zeros(getattr(sz, n) // torch.empty(0, dtype=dt).element_size(), dtype=dt)
    parts = dict(k8=t("k8", torch.uint8), v8=t("v8", torch.uint8), exps=t("exps", torch.int8), k_tail=t("k_tail", torch.float16), v_tail=t("v_tail", torch.float16),
                 lens=t("lens", torch.int32), flags=t("flags", torch.int32))
    c = A.BlockCache(2, 4, 2, 64, 64, torch.float16, **parts)
    q, k = torch.zeros(2, 3, 4, 64, dtype=torch.float16), torch.zeros(2, 3, 2, 64, dtype=torch.float16)
    i32 = lambda *x: torch.zeros(*x, dtype=torch.int32)
    f = torch.zeros(16)
    for bad in (dict(q=q.float()), dict(k=k.bfloat16()), dict(k=q), dict(q=q[:, :2]), dict(v=k[:1]), dict(inv_freq=f.double()), dict(inv_freq=f.view(4, 4)),
                dict(q_norm=torch.zeros(64)), dict(k_norm=torch.zeros(32, dtype=torch.float16)), dict(base=torch.zeros(2)), dict(n_new=i32(3)), dict(n_new=i32(2).long()),
                dict(q_out=torch.zeros(2, 3, 4, 64, dtype=torch.float16)), dict(q=q.transpose(2, 3).contiguous().transpose(2, 3))):
        args = dict(q=q, k=k, v=k, inv_freq=f, **{})
        args.update(bad)
        with pytest.raises(AssertionError):
            A.akb_append_rotated(c, args.pop("q"), args.pop("k"), args.pop("v"), **args)
    for bad in ((i32(3), None), (i32(2).long(), None), (i32(2), i32(1)), (None, i32(2).float())):
        with pytest.raises(AssertionError):
            A.akb_fork(c, c, *bad)
    for bad in (i32(3), i32(2).long()):
        with pytest.raises(AssertionError):
            A.akb_truncate(c, bad)
    for bad in (dict(q=q.transpose(1, 2).bfloat16()), dict(q=q), dict(q=q.transpose(1, 2), n_q=i32(3)), dict(q=q.transpose(1, 2), out=torch.zeros(2, 4, 3, 64, dtype=torch.bfloat16)),
                dict(q=q.transpose(1, 2), out=torch.zeros(2, 4, 3, 32))):
        with pytest.raises(AssertionError):
            A.akb_attention_shared(c, c, bad.pop("q"), **bad)
    # strides as a projection gives them, slices of one tensor among them; of a dimension of one element they do not count
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda self: True))
    x = torch.zeros(2, 3, 8, 64, dtype=torch.float16)
    assert A._projected(x[:, :, 4:6], c, 3, 2) == (x.data_ptr() + 4 * 64 * 2, 3 * 512, 512)
    assert A._projected(x[:, :1, :4], c, 1, 4)[1:] == (3 * 512, 0)
    assert A._projected(None, c, 3, 2) == (None, 0, 0)
