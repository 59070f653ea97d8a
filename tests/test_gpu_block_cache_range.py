"""The block-scaled 8-bit cache on the GPU at the ends of what its calls may be given: values up to the largest and down to the smallest of the type, in
blocks and in the tail, through every kernel and every way the parts of a call are put together.  Against 64 bits on the GPU."""
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


def check(c, q, out, K, V, lens, n_q=None, start=None, tiny=0.0):
    """out (and the score, where `start` is what it was) against the definition in 64 bits over the values K, V that the cache stands for.  The bound: the products
    of a score in 32 bits, its scaling and the subtraction, the exponential, the sums; the weights in 16 bits (16-bit results; the result is rounded once more) or
    as two 16-bit numbers; `tiny`: steps of numbers that have fixed ones."""
    B, Hq, n, D = q.shape
    G, half = Hq // c.Hkv, float(torch.finfo(c.dtype).eps) / 2
    for b in range(B):
        L, m = lens[b], n if n_q is None else n_q[b]
        for h in range(c.Hkv):
            Kd, Vd = K[b, h, :L].double(), V[b, h, :L].double()
            qd = q[b, h * G:(h + 1) * G, :m].double().reshape(G * m, D)
            past = torch.arange(L, device=DEV)[None] > (L - m + torch.arange(m, device=DEV)).repeat(G)[:, None]
            x = (qd @ Kd.T / D ** 0.5).masked_fill_(past, -float("inf"))
            size = (qd.abs() @ Kd.abs().T).masked_fill_(past, 0.0).amax(dim=1, keepdim=True)
            p = torch.softmax(x, dim=1).nan_to_num_(0.0)
            want, mag = p @ Vd, p @ Vd.abs()
            top = x.masked_fill(past, 0.0).abs().amax(dim=1, keepdim=True)
            eps = 2 * (D ** 0.5 * 2.0 ** -24 * size + 2.0 ** -22 * top + 2.0 ** -22) + (L / 16 + 64) * 2.0 ** -23
            bound = eps * mag + (half ** 2 * mag if out.dtype == F32 else half * mag + half * want.abs()) + tiny
            got = out[b, h * G:(h + 1) * G, :m].double().reshape(G * m, D)
            bad = ~((got - want).abs() <= bound)
            assert not bad.any(), (b, h, bad.nonzero()[:3].tolist(), got[bad][:3].tolist(), want[bad][:3].tolist(), bound[bad][:3].tolist())
            if start is not None:
                now, was = c.score.view(B, c.Hkv, -1)[b, h].double(), start.view(B, c.Hkv, -1)[b, h].double()
                add, rel = p.sum(dim=0), float(eps.max()) if m else 0.0
                assert ((now[:L] - was[:L] - add).abs() <= rel * add + (G * m / 16 + 32) * 2.0 ** -23 * (1 + add)).all(), (b, h)
                assert (now[L:] == was[L:]).all()


# kernel and parts; D, B, Hq, Hkv, tokens, n: the kernels and the ways their parts meet
WAYS = [
    ((1, 1), 128, 2, 4, 2, 200, 1),          # 16 rows, one part
    ((1, 4), 128, 1, 4, 4, 1000, 1),         # ... parts joined by the last workgroup
    ((1, 64), 128, 1, 64, 8, 20000, 1),      # ... by a launch
    ((1, 0), 64, 4, 32, 32, 9000, 1),        # ... parts by the lengths
    ((2, 1), 64, 2, 8, 2, 300, 10),          # 32 rows, one part
    ((2, 2), 128, 32, 32, 8, 4096, 5),       # ... parts joined by the last workgroup
    ((2, 11), 128, 3, 64, 8, 5000, 5),       # ... by a launch
    ((3, 1), 128, 2, 32, 8, 1100, 1100),      # 128 rows, one part
    ((3, 2), 64, 4, 8, 8, 4099, 1000),       # ... parts
]


@pytest.mark.parametrize("out_dtype", [F32, B16], ids=["f32", "bf16"])
@pytest.mark.parametrize("values", ["largest", "near", "blocks", "tail", "some", "small"])
@pytest.mark.parametrize("way", WAYS, ids=lambda w: f"kernel{w[0][0]}-parts{w[0][1]}-D{w[1]}-n{w[6]}")
def test_bfloat16_values_of_every_size(A, way, values, out_dtype):
    """bfloat16 reaches as far as binary32 does: the sums of weights times values stay finite for values up to the largest, and keep their bits for small ones."""
    path, D, B, Hq, Hkv, N, n = way
    Ncap = (N + 63) // 64 * 64
    print(way, values, flush=True)
    assert A.akb_attention_path(B, Hq, Hkv, D, Ncap, n) == path
    score = out_dtype == F32
    c = A.BlockCache.allocate(B, Hq, Hkv, D, Ncap, B16, score=score, n=n)
    g = torch.Generator(device=DEV).manual_seed(N)
    lens = [max(1, N - 37 * b) for b in range(B)]
    lens = [L - 1 if L % 64 == 0 else L for L in lens]   # a tail in every sequence
    k = torch.randn(B, Hkv, N, D, generator=g, device=DEV).to(B16)
    v = torch.randn(B, Hkv, N, D, generator=g, device=DEV).clamp_(-4, 4)
    top = R.LARGEST[B16]
    if values == "largest":
        v = torch.where(torch.arange(D, device=DEV) % 2 == 0, top, -top).expand_as(v)
    elif values == "near":
        v = v * 2.0 ** 113     # no single one is near the end; sums of weights of any size above one are
    elif values in ("blocks", "tail"):
        for b, L in enumerate(lens):
            v[b, :, slice(0, L // 64 * 64) if values == "blocks" else slice(L // 64 * 64, L)] *= 2.0 ** 125
    elif values == "some":
        v[:, :, ::97] *= 2.0 ** 125
    else:
        v = v * 2.0 ** -97
    v = v.to(B16)
    A.akb_append(c, k, v, i32(lens))
    q = torch.randn(B, Hq, n, D, generator=g, device=DEV).to(B16)
    start = torch.rand(c.score.shape, generator=g, device=DEV) if score else None
    if score:
        c.score.copy_(start)
    out = A.akb_attention(c, q, torch.empty(q.shape, dtype=out_dtype, device=DEV), accumulate=score)
    assert torch.isfinite(out).all()
    K, V = A.akb_unpack(c)
    assert values == "small" or float(V.abs().amax()) >= 2.0 ** 114
    check(c, q, out, K, V, lens, start=start, tiny=2.0 ** -120)   # (products and sums below 2^-126, and how they are rounded: a step of 2^-126 is far below)


def test_one_token_comes_back(A):
    """A single token is its own average, whatever its values are: the largest numbers of the type, in the tail."""
    for D in (64, 128):
        for dtype in (F16, B16):
            c = A.BlockCache.allocate(3, 4, 2, D, 64, dtype)
            v = torch.full((3, 2, 1, D), R.LARGEST[dtype], dtype=dtype, device=DEV)
            v[:, 1] = -v[:, 1] / 2
            A.akb_append(c, torch.ones_like(v), v)
            q = torch.ones(3, 4, 1, D, dtype=dtype, device=DEV)
            for out_dtype in (F32, dtype):
                out = A.akb_attention(c, q, torch.empty(q.shape, dtype=out_dtype, device=DEV))
                # one weight, rounded to 16 bits or to two 16-bit numbers, over itself: a number whose rounding is 0 (a power of two, up to the rounding of the
                # exponent's argument, 2^-21)
                want = v.repeat_interleave(2, dim=1).double()
                assert ((out.double() - want).abs() <= want.abs() * 2.0 ** -19).all(), (dtype, out_dtype)


@pytest.mark.parametrize("dtype", [F16, B16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("way", [((1, 1), 128, 8, 16, 1, 40, 1), ((1, 1), 64, 8, 16, 1, 500, 1), ((1, 4), 128, 2, 64, 4, 1000, 1), ((2, 1), 64, 4, 32, 2, 300, 2),
                                 ((2, 2), 128, 32, 32, 8, 1100, 5), ((3, 8), 128, 8, 8, 8, 6200, 65), ((3, 8), 64, 8, 8, 8, 6200, 65)],
                         ids=lambda w: f"kernel{w[0][0]}-parts{w[0][1]}-D{w[1]}-N{w[5]}-n{w[6]}")
def test_32_bit_results_of_two_weights(A, way, dtype):
    """Rows that see two tokens of weights 1 and 2^-x, x below 1, and others of none; the value of the second is 1, of the others 0: the result is 1 / (1 + 2^x).  Off by:
    the two exponents, rounded below 8 (2^-22 each, times ln 2); the exponentials (2^-23 each); the scale, the sum of the weights, the weight itself (22 bits or more), its
    three products, the reciprocal and the product with it (2^-24 each, twice for the weight)."""
    path, D, B, Hq, Hkv, N, n = way
    Ncap = (N + 63) // 64 * 64
    assert A.akb_attention_path(B, Hq, Hkv, D, Ncap, n) == path
    c = A.BlockCache.allocate(B, Hq, Hkv, D, Ncap, dtype, n=n)
    k, v = (torch.zeros(B, Hkv, N, D, dtype=dtype, device=DEV) for _ in range(2))
    k[:, :, :, 0] = -2.0 ** 14                     # times 2^-7 and more: weights below 2^-127
    k[:, :, 0, 0], k[:, :, 1, 0] = 1.0, 0.0
    v[:, :, 1] = 1.0
    A.akb_append(c, k, v)
    x = (torch.arange(B * Hq * n, device=DEV) * 37 % 127 + 1).view(B, Hq, n) / 128   # 1/128 .. 127/128, numbers of 7 bits
    q = torch.zeros(B, Hq, n, D, dtype=dtype, device=DEV)
    q[..., 0] = x.to(dtype)
    scale = float(torch.tensor(0.6931471805599453, dtype=F32))
    out = A.akb_attention(c, q, scale=scale).double()
    want = 1 / (1 + torch.exp(x.double() * scale))[..., None]
    worst = float(((out - want).abs() / want).max())
    print(f"worst {worst:.2e}", flush=True)
    assert worst <= 2 * (2.0 ** -22 * 0.6932 + 2.0 ** -23) + 9 * 2.0 ** -24 + (2.0 ** -22 if dtype == F16 else 0.0)
