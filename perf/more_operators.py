"""The operators that serve several continuations of one prompt from the block-scaled 8-bit cache, as cases that can be timed and compared:
attention of sequences that continue shared ones (a shared prefix is read once for all of them), the step from a model's projections to
stored tokens and turned queries (norms of queries and keys per head, rotary positions, the append), copies of sequences with a length of
their own (sampling, beams), and sequences cut back in place (rejected drafts).

A cache holds complete blocks of 64 tokens as e4m3 numbers with one power of two per block, KV head and side (K, V), and the
tokens of the last, incomplete block in 16 bits (``include/akb.h`` says which byte lies where).  ``prepare`` lays such caches
out with torch alone, so that both forms work on the same bytes:

* the plain form (``own`` false) in elementary torch operations, 32 bits (64 for angles, and for keys, whose values next to a border decide
  a block's exponent), rounded once at the end;
* the library's calls (``own`` true).

``exact`` goes from the same inputs to the results in 64 bits, by the definition and written apart from the plain form.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
TB = 64                      # tokens per block
E_MIN = -100                 # least exponent of a block's scale
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
OUTS = {"f32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
TOP_EXP = {"fp16": 8, "bf16": 120}     # the scale at which 256 times it is no number of the type any more
EPS = 1e-6                             # of the norms
MOST_SCORES = 8 * 32 * 777 * 20778     # query rows x tokens of the largest listed attention
MOST_SHARED = 32768 * 8 * 128          # values of one side of the largest listed prefix
MOST_OWN = 64 * 8 * 1024 * 128         # ... of the largest listed cache of continuations
MOST_TURNED = 4 * 8192 * 48 * 128      # projected values of the largest listed append
MOST_COPIED = 16 * 8 * 8192 * 128      # values of one side of the largest listed copy


# ------------------------------------------------------------------------------------------------------ cases

def _shared(name, Bp, W, Hq, Hkv, P, N, n, dtype, out, *, D=128, data="scales", ragged=True):
    return dict(name=name, kind="shared", Bp=Bp, B=Bp * W, Hq=Hq, Hkv=Hkv, D=D, P=P, N=N, n=n, dtype=dtype, out=out, data=data, ragged=ragged)


def _rotated(name, B, Hq, Hkv, start, n, dtype, *, D=128, rot=128, norm=True, pairs=False, packed=True, base=0, Bp=1, data="scales", ragged=False):
    return dict(name=name, kind="rotated", B=B, Hq=Hq, Hkv=Hkv, D=D, start=start, n=n, dtype=dtype, rot=rot, norm=norm, pairs=pairs, packed=packed,
                base=base, Bp=Bp, data=data, ragged=ragged)


def _fork(name, Bs, Bd, Hkv, N, dtype, *, D=128, cut=0, idle=False, score=False, data="scales", ragged=False):
    return dict(name=name, kind="fork", Bs=Bs, B=Bd, Hkv=Hkv, D=D, N=N, cut=cut, idle=idle, score=score, dtype=dtype, data=data, ragged=ragged)


def _truncate(name, B, Hkv, N, back, dtype, *, D=128, data="scales"):
    return dict(name=name, kind="truncate", B=B, Hkv=Hkv, D=D, N=N, back=back, dtype=dtype, data=data, ragged=True)


def listed() -> list[dict]:
    return [
        # four answers sampled for one short prompt, full heads: the smallest attention call, where latency counts
        _shared("shared_1x4_mha_1k", 1, 4, 32, 32, 1024, 60, 1, "fp16", "f32", data="plain"),
        # a long system prompt before a full batch of conversations
        _shared("shared_1x64_gqa4_32k", 1, 64, 32, 8, 32768, 1000, 1, "bf16", "bf16"),
        # eight prompts of mixed lengths with eight beams each
        _shared("shared_8x8_gqa4_8k", 8, 8, 32, 8, 8192, 500, 1, "fp16", "f32"),
        # drafts of up to five tokens of sixteen conversations behind one document, 64 query heads on 8
        _shared("shared_1x16_draft5_gqa8_13k", 1, 16, 64, 8, 13000, 3001, 5, "fp16", "fp16", data="student"),
        # two documents with four questions each, stored behind them: the most operations
        _shared("shared_2x4_chunk777_20k", 2, 4, 32, 8, 20001, 777, 777, "bf16", "bf16"),
        # one serving step's new token of every sequence, behind a shared prefix: the smallest append
        _rotated("rotated_1", 64, 32, 8, 1000, 1, "bf16", base=32768, ragged=True),
        # a batch of prompts stored from empty: the most bytes
        _rotated("rotated_prompt_8k", 4, 32, 8, 0, 8192, "bf16"),
        # chunks of mixed lengths onto sequences that end anywhere, small heads of which half the channels turn, neighbours in pairs, no norms
        _rotated("rotated_chunk_777_d64", 6, 16, 4, 9001, 777, "fp16", D=64, rot=32, norm=False, pairs=True, packed=False, base=5000, Bp=6, ragged=True),
        # beams of eight prompts put in their new order, behind shared prefixes
        _fork("fork_beams_64x500", 64, 64, 8, 500, "bf16", ragged=True),
        # one prompt handed to sixteen sequences that go on from places of their own; with accumulated weights
        _fork("fork_1x16_prompt_8k", 1, 16, 8, 8192, "fp16", cut=300, score=True),
        # drafts of up to five tokens, some rejected: the smallest call of all
        _truncate("truncate_draft_64", 64, 8, 1000, 5, "bf16"),
        # answers taken back by up to 777 tokens, full heads
        _truncate("truncate_16x32_back_777", 16, 32, 4000, 777, "fp16"),
    ]


def _log(rng, lo, hi):
    """A whole number, its logarithm uniform over [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng) -> dict:
    kind = rng.choice(["shared"] * 5 + ["rotated"] * 3 + ["fork"] * 2 + ["truncate"] * 2)
    D, dtype = rng.choice([64, 128, 128, 128]), rng.choice(["fp16", "bf16"])
    data, ragged = rng.choice(["plain", "scales", "student"]), rng.random() < 0.6
    Hkv = rng.choice([2, 8, 8, 32])
    common = dict(kind=kind, Hkv=Hkv, D=D, dtype=dtype, data=data)
    if kind == "shared":
        G, P, N = rng.choice([1, 1, 2, 4, 4, 5, 8, 16]), _log(rng, 60, min(32768, MOST_SHARED // (Hkv * D))), _log(rng, 1, 4096)
        Bp = _log(rng, 1, max(1, min(8, MOST_SHARED // (Hkv * P * D))))
        W = _log(rng, 1, max(1, min(64, MOST_OWN // (Bp * Hkv * N * D), MOST_SCORES // (Bp * Hkv * G * (P + N)))))
        n = 1
        if rng.random() < 0.5:
            n = _log(rng, 1, max(1, min(1000, N, MOST_SCORES // (Bp * W * Hkv * G * (P + N)))))
        return dict(common, Bp=Bp, B=Bp * W, Hq=Hkv * G, P=P, N=N, n=n, out=rng.choice(["f32", dtype]), ragged=ragged)
    if kind == "rotated":
        G, n, start = rng.choice([1, 2, 4, 4, 5, 8, 16]), _log(rng, 1, 8192), rng.choice([0, rng.randrange(1, 8192)])
        most = MOST_TURNED // D
        n = max(1, min(n, most // (Hkv * (G + 2))))
        B = _log(rng, 1, max(1, min(128, most // (Hkv * max(n * (G + 2), start + n)))))
        base = rng.choice([0, rng.randrange(1, 200000)])
        return dict(common, B=B, Hq=Hkv * G, start=start, n=n, rot=rng.choice([D, D, D // 2, 16 * rng.randrange(0, D // 16 + 1)]), norm=rng.random() < 0.6,
                    pairs=rng.random() < 0.4, packed=rng.random() < 0.5, base=base, Bp=rng.choice([1, B]), ragged=ragged)
    N = _log(rng, 30, 16384)
    if kind == "fork":
        B = _log(rng, 1, max(1, min(64, MOST_COPIED // (Hkv * (N + TB) * D))))
        return dict(common, Bs=_log(rng, 1, B), B=B, N=N, cut=rng.choice([0, 0, _log(rng, 1, N)]), idle=rng.random() < 0.3, score=rng.random() < 0.4, ragged=ragged)
    B = _log(rng, 1, max(1, min(128, MOST_COPIED // (Hkv * (N + TB) * D))))
    return dict(common, B=B, N=N, back=_log(rng, 1, N), ragged=ragged)


# ----------------------------------------------------------------------------------------- the layout of a cache

def _rows(k8):
    """K codes [B, H, NB, 4, D/64, 16, 64] (tile of 16 tokens, 64 channels, token, channel) -> a view [B, H, NB, 4, 16, D/64, 64]."""
    return k8.permute(0, 1, 2, 3, 5, 4, 6)


def _columns(v8):
    """V codes [B, H, NB, D, 4, 4, 4]: of a channel, token 16 t + 4 g + r lies at place [g][t][r] -> a view [B, H, NB, t, g, r, D]."""
    return v8.permute(0, 1, 2, 5, 4, 6, 3)


def _tail_columns(v_tail):
    """The same order in the 16-bit tail of V [B, H, D, 4, 4, 4] -> a view [B, H, t, g, r, D]."""
    return v_tail.permute(0, 1, 4, 3, 5, 2)


def _buffers(B, Hkv, D, Ncap, dtype, score=False):
    NB = -(-Ncap // TB)
    z = lambda *s, t=torch.uint8: torch.zeros(*s, dtype=t, device=DEV)
    return dict(k8=z(B, Hkv, NB, 4, D // 64, 16, 64), v8=z(B, Hkv, NB, D, 4, 4, 4), exps=z(B, Hkv, NB, 2, t=torch.int8),
                k_tail=z(B, Hkv, TB, D, t=TYPES[dtype]), v_tail=z(B, Hkv, D, 4, 4, 4, t=TYPES[dtype]),
                score=z(B, Hkv, NB * TB, t=torch.float32) if score else None, lens=z(B, t=torch.int32), flags=z(4 + B, t=torch.int32))


def _handle(case, c, Hq):
    """The library's cache object over the buffers of `c`."""
    from paper_2409_16546_amd import binding as A
    return A.BlockCache(c["lens"].shape[0], Hq, case["Hkv"], case["D"], c["exps"].shape[2] * TB, TYPES[case["dtype"]], c["k8"], c["v8"], c["exps"],
                        c["k_tail"], c["v_tail"], c["lens"], c["flags"], c["score"])


# ----------------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) & 0x7FFFFFFF)


def _tokens(case, gen, H, n, scales):
    """16-bit [H, n, D] of the case's distribution; `scales`: the channels' sizes [H, 1, D]."""
    x = torch.randn(H, n, case["D"], generator=gen, device=DEV) * scales
    if case["data"] == "student":   # Student-t, three degrees of freedom
        x /= sum(torch.randn(H, n, case["D"], generator=gen, device=DEV).square_() for _ in range(3)).div_(3).sqrt_()
    return x.clamp_(-65504, 65504).to(TYPES[case["dtype"]])


def _scales(case, gen, H):
    shape = (H, 1, case["D"])
    return torch.pow(10.0, torch.rand(shape, generator=gen, device=DEV) * 2 - 1) if case["data"] == "scales" else torch.ones(shape, device=DEV)


def _whole(gen, lo, hi, count):
    return torch.randint(lo, hi + 1, (count,), generator=gen, device=DEV).to(torch.int32)


def _lens(case, gen, N, B):
    return _whole(gen, max(1, N // 4), N, B) if case["ragged"] and N else torch.full((B,), N, dtype=torch.int32, device=DEV)


def _filled(case, gen, B, N, Ncap, score=False):
    """A cache whose B sequences hold up to N tokens."""
    H, D = case["Hkv"], case["D"]
    c = _buffers(B, H, D, Ncap, case["dtype"], score)
    c["lens"].copy_(_lens(case, gen, N, B))
    NB = N // TB
    ks, vs = _scales(case, gen, H), _scales(case, gen, H)
    for b in range(B):
        for side, (scales, view, tail) in enumerate(((ks, _rows(c["k8"])[b], c["k_tail"][b].view(-1, 4, 4, 4, D)),
                                                     (vs, _columns(c["v8"])[b], _tail_columns(c["v_tail"])[b]))):
            for h in range(0, H, 8):   # eight heads at a time keep the temporaries small
                m = min(8, H - h)
                x = _tokens(case, gen, m, (NB + 1) * TB, scales[h:h + 8]).view(m, NB + 1, TB, D)
                codes, e = _pack(x[:, :NB].float(), case["dtype"])
                view[h:h + 8, :NB] = codes.view(m, NB, *view.shape[2:])
                c["exps"][b, h:h + 8, :NB, side] = e
                tail[h:h + 8] = x[:, NB].reshape(tail[h:h + 8].shape)
    if score:
        c["score"].copy_(torch.exp(2 * torch.randn(c["score"].shape, generator=gen, device=DEV)))
    return c


def prepare(case, seed):
    gen = _gen(seed)
    B, Hkv, D, dt = case["B"], case["Hkv"], case["D"], TYPES[case["dtype"]]
    if case["kind"] == "shared":
        Hq, n = case["Hq"], case["n"]
        s = dict(case=case, p=_filled(case, gen, case["Bp"], case["P"], case["P"]), c=_filled(case, gen, B, case["N"], case["N"]))
        s["q"] = torch.randn(B, Hq, n, D, generator=gen, device=DEV).to(dt)
        s["n_q"] = _whole(gen, max(1, n // 3), n, B) if case["ragged"] and n > 1 else None
        s["out"] = torch.zeros(B, Hq, n, D, dtype=OUTS[case["out"]], device=DEV)
        if own:
            s["prefix"], s["handle"] = _handle(case, s["p"], Hq), _handle(case, s["c"], Hq)
            s["handle"].reserve(n, prefix=s["prefix"])
    elif case["kind"] == "rotated":
        start, n, Hq = case["start"], case["n"], case["Hq"]
        s = dict(case=case, c=_filled(case, gen, B, start, start + n + TB))
        s["ends"] = {k: s["c"][k].clone() for k in (("lens", "k_tail", "v_tail") if start and n > 1 else ("lens",))}
        heads = torch.cat([_scales(case, gen, H) for H in (Hq, Hkv, Hkv)])
        x = torch.stack([_tokens(case, gen, Hq + 2 * Hkv, n, heads).transpose(0, 1).contiguous() for _ in range(B)])   # [B, n, heads, D], as a projection gives it
        s["q"], s["k"], s["v"] = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
        if not case["packed"]:
            s["q"], s["k"], s["v"] = (t.contiguous() for t in (s["q"], s["k"], s["v"]))
        s["norms"] = [(1 + 0.2 * torch.randn(D, generator=gen, device=DEV)).to(dt) for _ in range(2)] if case["norm"] else [None, None]
        rot = case["rot"]
        s["freq"] = torch.pow(torch.tensor(10000.0, dtype=torch.float64, device=DEV), -torch.arange(rot // 2, device=DEV).double() / max(1, rot // 2)).float()
        s["base"] = _whole(gen, case["base"] // 2, case["base"], case["Bp"]) if case["base"] else None
        s["n_new"] = _whole(gen, max(1, n // 3), n, B) if case["ragged"] else None
        s["out"] = torch.zeros(B, Hq, n, D, dtype=dt, device=DEV)
        if own:
            s["handle"] = _handle(case, s["c"], Hq)
    elif case["kind"] == "fork":
        N, Bs = case["N"], case["Bs"]
        s = dict(case=case, c=_filled(case, gen, Bs, N, N, case["score"]), d=_buffers(B, Hkv, D, N + TB, case["dtype"], case["score"]))
        s["parents"] = (torch.arange(B, device=DEV) * Bs // B + _whole(gen, -2, 2, B)).clamp(0, Bs - 1).to(torch.int32)   # beams of a prompt lie beside each other
        if case["idle"]:
            s["parents"][torch.rand(B, generator=gen, device=DEV) < 0.2] = -1
        s["upto"] = _whole(gen, N - case["cut"], N, B) if case["cut"] else None
        if own:
            s["handle"], s["to"] = _handle(case, s["c"], Hkv), _handle(case, s["d"], Hkv)
    else:
        s = dict(case=case, c=_filled(case, gen, B, case["N"], case["N"]))
        s["had"] = s["c"]["lens"].clone()
        s["keep"] = (s["had"] - _whole(gen, 0, case["back"], B)).clamp(min=0)
        if own:
            s["handle"] = _handle(case, s["c"], Hkv)
    return s


# ------------------------------------------------------------------------------------------------- the plain form

def _pack(x, dtype):
    """x: [..., 64, D] -> (codes as uint8, exponents as int8 [...]): the least e with max|x| <= 448 2^e, codes to the nearest."""
    m, p = torch.frexp(x.abs().amax(dim=(-2, -1)))
    e = (torch.where(m <= 0.875, p - 9, p - 8)).clamp(min=E_MIN)
    e = torch.where(m == 0, torch.full_like(e, E_MIN), e)
    y = torch.ldexp(x, -e[..., None, None])
    step = torch.ldexp(torch.ones_like(y), (torch.frexp(y).exponent - 4).clamp(min=-9))
    y = torch.round(y / step) * step
    y = torch.where((e == TOP_EXP[dtype])[..., None, None], y.clamp(-240, 240), y)   # 256 times this scale is beyond the type
    return y.to(torch.float8_e4m3fn).view(torch.uint8), e.to(torch.int8)


def _values(view, exps, tail, lens):
    """The stored values as float32 [B, H, NB * 64, D]: blocks, and the tail in the place of the last, incomplete one."""
    B, H, NB, D = *exps.shape[:3], tail.shape[-1]
    x = view.reshape(B, H, NB, TB, D).view(torch.float8_e4m3fn).float()
    x = torch.ldexp(x, exps.int()[..., None, None])
    at = (lens.long() // TB).clamp(max=NB - 1).view(B, 1, 1, 1, 1).expand(B, H, 1, TB, D)
    part = ((lens % TB) > 0).view(B, 1, 1, 1, 1)
    x.scatter_(2, at, torch.where(part, tail.reshape(B, H, 1, TB, D).float(), x.gather(2, at)))
    return x.view(B, H, NB * TB, D)


def _k_values(c):
    return _values(_rows(c["k8"]), c["exps"][..., 0], c["k_tail"], c["lens"])


def _v_values(c):
    """V, zeros behind the lengths."""
    x = _values(_columns(c["v8"]), c["exps"][..., 1], _tail_columns(c["v_tail"]), c["lens"])
    return torch.where(torch.arange(x.shape[2], device=DEV).view(1, 1, -1, 1) < c["lens"].view(-1, 1, 1, 1), x, 0.0)


def _shared_plain(s):
    case, p, c, q = s["case"], s["p"], s["c"], s["q"].float()
    Bp, B, Hq, Hkv, D, n = case["Bp"], case["B"], case["Hq"], case["Hkv"], case["D"], case["n"]
    W, G = B // Bp, Hq // Hkv
    lens, first = c["lens"].view(B, 1, 1, 1, 1), p["lens"].repeat_interleave(W).view(B, 1, 1, 1, 1)
    n_q = lens.new_full((B, 1, 1, 1, 1), n) if s["n_q"] is None else s["n_q"].view(B, 1, 1, 1, 1)
    i = torch.arange(n, device=DEV).view(1, 1, 1, n, 1)
    kp, kc = _k_values(p), _k_values(c)
    P, N = kp.shape[2], kc.shape[2]
    past = lens - n_q + i                                                            # the query token's own place behind the prefix
    tp, tc = torch.arange(P, device=DEV), torch.arange(N, device=DEV)
    seen = torch.cat([(tp <= first + past) & (tp < first) & (i < n_q), (tc <= past) & (tc < lens) & (i < n_q)], dim=4)   # [B, 1, 1, n, P + N]
    rows = q.view(Bp, W, Hkv, G * n, D).transpose(1, 2).reshape(Bp, Hkv, W * G * n, D)   # of all continuations of a prefix
    x = torch.cat([torch.matmul(rows, kp.transpose(2, 3).contiguous()).reshape(Bp, Hkv, W, G, n, P).transpose(1, 2).reshape(B, Hkv, G, n, P),
                   torch.matmul(q.view(B, Hkv, G * n, D), kc.transpose(2, 3).contiguous()).reshape(B, Hkv, G, n, N)], dim=4)
    x = torch.where(seen, x * (1 / math.sqrt(D)), -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    w = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    z = w.sum(dim=-1, keepdim=True)
    w = w / torch.where(z == 0, 1.0, z)
    wp = w[..., :P].reshape(Bp, W, Hkv, G * n, P).transpose(1, 2).reshape(Bp, Hkv, W * G * n, P)
    o = torch.matmul(wp, _v_values(p)).reshape(Bp, Hkv, W, G * n, D).transpose(1, 2).reshape(B, Hkv, G * n, D)
    o = (o + torch.matmul(w[..., P:].reshape(B, Hkv, G * n, N), _v_values(c))).reshape(B, Hq, n, D)
    s["out"].copy_(torch.where((i < n_q).view(B, 1, n, 1), o.to(s["out"].dtype), s["out"]))


def _turn(case, x, weight, cos, sin):
    """x: [B, n, H, D] -> normed per head where there is a weight, its first `rot` channels turned in pairs; in x's type."""
    cos, sin = cos.to(x.dtype), sin.to(x.dtype)
    if weight is not None:
        x = x / torch.sqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * weight.to(x.dtype)
    rot = case["rot"]
    if not rot:
        return x
    x = x.clone()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if case["pairs"] else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, w = a * cos - b * sin, a * sin + b * cos
    a.copy_(u)
    b.copy_(w)
    return x


def _rotated_plain(s):
    case, c = s["case"], s["c"]
    B, Hq, Hkv, D, n, dt = case["B"], case["Hq"], case["Hkv"], case["D"], case["n"], TYPES[case["dtype"]]
    lens = c["lens"].long()
    count = torch.full_like(lens, n) if s["n_new"] is None else s["n_new"].long()
    first = lens if s["base"] is None else lens + s["base"].long().repeat_interleave(B // case["Bp"])
    angle = (first.view(B, 1, 1, 1) + torch.arange(n, device=DEV).view(1, n, 1, 1)).double() * s["freq"].double()   # [B, n, 1, rot / 2]
    cos, sin = torch.cos(angle), torch.sin(angle)
    turned = _turn(case, s["q"].float(), s["norms"][0], cos, sin).transpose(1, 2).to(dt)
    s["out"].copy_(torch.where(torch.arange(n, device=DEV).view(1, 1, n, 1) < count.view(B, 1, 1, 1), turned, s["out"]))
    k, v = _turn(case, s["k"].double(), s["norms"][1], cos, sin).transpose(1, 2).to(dt), s["v"].transpose(1, 2)
    NW = -(-(TB - 1 + n) // TB)                                                     # blocks that an append can touch
    w = torch.arange(NW * TB, device=DEV).view(1, 1, NW * TB, 1)
    had, total = (lens % TB).view(B, 1, 1, 1), (lens % TB + count).view(B, 1, 1, 1)
    src = (w - had).clamp(0, n - 1).expand(B, Hkv, NW * TB, D)
    head = (w[:, :, :TB]).expand(B, Hkv, TB, D)
    new = torch.arange(NW, device=DEV).view(1, NW) < (total.view(B, 1) // TB)         # blocks that are complete now
    blocks = (lens // TB).view(B, 1) + torch.arange(NW, device=DEV).view(1, NW)
    last = (total // TB).view(B, 1, 1, 1).clamp(max=NW - 1)
    slot = last * TB + w[:, :, :TB]                                                 # where the tail's slots lie among the blocks
    keep = (slot < had) | (slot >= total) | (total // TB >= NW)
    for side, (fresh, view, tail) in enumerate(((k, _rows(c["k8"]), c["k_tail"].view(B, Hkv, 4, 4, 4, D)), (v, _columns(c["v8"]), _tail_columns(c["v_tail"])))):
        x = fresh.gather(2, src)
        old = tail.reshape(B, Hkv, TB, D)
        x[:, :, :TB] = torch.where(head < had, old, x[:, :, :TB])
        codes, e = _pack(x.view(B, Hkv, NW, TB, D).float(), case["dtype"])
        b = torch.arange(B, device=DEV).view(B, 1)
        codes = codes.view(B, Hkv, NW, *view.shape[3:]).transpose(1, 2)             # [B, NW, Hkv, ...]
        mask = new.view(B, NW, *(1,) * (codes.dim() - 2))
        view[b, :, blocks] = torch.where(mask, codes, view[b, :, blocks])
        ex = c["exps"][..., side]
        ex[b, :, blocks] = torch.where(new.view(B, NW, 1), e.transpose(1, 2), ex[b, :, blocks])
        tail.copy_(torch.where(keep, old, x.gather(2, slot.expand(B, Hkv, TB, D))).view(tail.shape))
    c["lens"].copy_(lens + count)


def _block_as_tail(c, b, at):
    """Block at[i] of sequence b[i] as the 16-bit tails hold it: K [i, H, 64, D], V [i, H, D, 4, 4, 4]."""
    e = torch.exp2(c["exps"][b, :, at].float())
    k = _rows(c["k8"])[b, :, at].reshape(len(b), c["k8"].shape[1], TB, -1).view(torch.float8_e4m3fn).float() * e[:, :, 0, None, None]
    v = c["v8"][b, :, at].view(torch.float8_e4m3fn).float() * e[:, :, 1, None, None, None, None]
    return k.to(c["k_tail"].dtype), v.to(c["v_tail"].dtype)


def _fork_plain(s):
    case, c, d = s["case"], s["c"], s["d"]
    B, Bs = case["B"], case["Bs"]
    some = s["parents"] >= 0
    from_ = s["parents"].long().clamp(0, Bs - 1)
    had = c["lens"].long()[from_]
    lens = had if s["upto"] is None else torch.minimum(had, s["upto"].long())
    NB = c["exps"].shape[2]
    blocks = (some.view(B, 1) & (torch.arange(NB, device=DEV).view(1, NB) < (lens // TB).view(B, 1))).view(B, 1, NB)
    for name in ("k8", "v8", "exps"):
        to = d[name][:, :, :NB]
        to.copy_(torch.where(blocks.view(B, 1, NB, *(1,) * (to.dim() - 3)), c[name][from_], to))
    # the tail: the source's own, or what one of its blocks stands for
    part, inside = some & (lens % TB > 0), lens // TB < had // TB
    for name, block in zip(("k_tail", "v_tail"), _block_as_tail(c, from_, (lens // TB).clamp(max=NB - 1))):
        ones = (1,) * (block.dim() - 1)
        d[name].copy_(torch.where(part.view(B, *ones), torch.where(inside.view(B, *ones), block, c[name][from_]), d[name]))
    if case["score"]:
        N = c["score"].shape[2]
        keep = (some.view(B, 1) & (torch.arange(N, device=DEV).view(1, N) < lens.view(B, 1))).view(B, 1, N)
        d["score"][:, :, :N] = torch.where(keep, c["score"][from_], d["score"][:, :, :N])
    d["lens"].copy_(torch.where(some, lens, d["lens"].long()))


def _truncate_plain(s):
    c, B = s["c"], s["case"]["B"]
    had = c["lens"].long()
    lens = torch.minimum(had, s["keep"].long())
    inside = (lens % TB > 0) & (lens // TB < had // TB)
    for name, block in zip(("k_tail", "v_tail"), _block_as_tail(c, torch.arange(B, device=DEV), (lens // TB).clamp(max=c["exps"].shape[2] - 1))):
        c[name].copy_(torch.where(inside.view(B, *(1,) * (block.dim() - 1)), block, c[name]))
    c["lens"].copy_(lens)


def run(s):
    case, c = s["case"], s["c"]
    if own:
        from paper_2409_16546_amd import binding as A
    if case["kind"] == "shared":
        if own:
            A.akb_attention_shared(s["prefix"], s["handle"], s["q"], s["out"], n_q=s["n_q"])
        else:
            _shared_plain(s)
        return {"out": s["out"]}
    if case["kind"] == "rotated":
        for k, end in s["ends"].items():   # the sequences end where they ended before
            c[k].copy_(end)
        if own:
            A.akb_append_rotated(s["handle"], s["q"], s["k"], s["v"], s["out"], inv_freq=s["freq"], n_new=s["n_new"], q_norm=s["norms"][0], k_norm=s["norms"][1],
                                 eps=EPS, pairs=case["pairs"], base=s["base"])
        else:
            _rotated_plain(s)
        return {"q": s["out"], **_outputs(c)}
    if case["kind"] == "fork":
        if own:
            A.akb_fork(s["handle"], s["to"], s["parents"], s["upto"])
        else:
            _fork_plain(s)
        return {**_outputs(s["d"]), "score": s["d"]["score"]}
    c["lens"].copy_(s["had"])   # the sequences are as long as they were (a tail that takes a block's values takes the same again)
    if own:
        A.akb_truncate(s["handle"], s["keep"])
    else:
        _truncate_plain(s)
    return {"k_tail": c["k_tail"], "v_tail": c["v_tail"], "lens": c["lens"]}


def _outputs(c):
    """A cache as what it stands for: e4m3 numbers, the exponents of their scales, the tails and lengths."""
    return {"k": c["k8"].view(torch.float8_e4m3fn), "v": c["v8"].view(torch.float8_e4m3fn), "exps": c["exps"], "k_tail": c["k_tail"], "v_tail": c["v_tail"],
            "lens": c["lens"]}


# ----------------------------------------------------------------------------------------------------------- work

def _mean(case, N):
    return N if not case["ragged"] else (max(1, N // 4) + N) / 2


def work(case):
    B, Hkv, D = case["B"], case["Hkv"], case["D"]
    if case["kind"] == "shared":
        n, P, N = case["n"], _mean(case, case["P"]), _mean(case, case["N"])
        m = (max(1, n // 3) + n) / 2 if case["ragged"] and n > 1 else n       # query tokens of a sequence
        kv = Hkv * (case["Bp"] * P + B * N) * (2 * D + 2 / TB)
        io = B * case["Hq"] * m * D * (2 + (4 if case["out"] == "f32" else 2))
        own_seen = m * N - m * (m - 1) / 2 if m <= N else N * (N + 1) / 2
        return {"bytes": kv + io, "flops": 4 * D * B * case["Hq"] * (m * P + own_seen)}
    if case["kind"] == "rotated":
        n = case["n"]
        m = (max(1, n // 3) + n) / 2 if case["ragged"] else n
        out = 2 * D if n >= TB else 4 * D
        return {"bytes": B * m * (case["Hq"] * 4 * D + Hkv * (4 * D + out)), "flops": B * m * (case["Hq"] + Hkv) * (3 * case["rot"] + (4 * D if case["norm"] else 0))}
    per = Hkv * (2 * D + 2 / TB + (4 if case.get("score") else 0))            # bytes of a stored token
    tail = Hkv * 4 * D * TB / 2                                               # ... of half a tail
    if case["kind"] == "fork":
        some = 0.8 if case["idle"] else 1.0
        N = _mean(case, case["N"]) - case["cut"] / 2
        read = min(case["Bs"], B * some)
        return {"bytes": (read + B * some) * (max(0, N - TB / 2) * per + tail), "flops": 0}
    cross = min(1.0, case["back"] / 2 / TB)                                   # the part of the sequences that go back into a complete block
    return {"bytes": B * (cross * 1.5 * tail + 12), "flops": 0}


# ----------------------------------------------------------------------------------------------------- in 64 bits

#: the 127 magnitudes of e4m3 (without infinities), by code
_E4M3 = [((c & 7) / 8 if c < 8 else 1 + (c & 7) / 8) * 2.0 ** (max(c >> 3, 1) - 7) for c in range(127)]


def _exact_block(x, largest):
    """x: float64 [m, 64, D] -> (numbers of e4m3 as float64, exponents): found in the table of all of them."""
    table = torch.tensor(_E4M3, dtype=torch.float64, device=x.device)
    mid = (table[1:] + table[:-1]) / 2
    top = x.abs().flatten(1).amax(dim=1)
    e = torch.full_like(top, float(E_MIN))
    for k in range(E_MIN + 1, 121):
        e = torch.where(top > 448.0 * 2.0 ** (k - 1), float(k), e)
    y = x * torch.exp2(-e).view(-1, 1, 1)
    a = y.abs()
    low = torch.searchsorted(mid, a.contiguous())                   # mid[low - 1] < a <= mid[low]
    tie = (low < 126) & (a == mid[low.clamp(max=125)])
    code = torch.where(tie & (low % 2 == 1), low + 1, low)          # between two: the even one
    code = torch.where(table[code] * torch.exp2(e).view(-1, 1, 1) > largest, code - 1, code)
    return table[code] * torch.sign(y), e


def _exact_tokens(c, b, h, side, n, D, tail=True):
    """The stored values of one head as float64 [n, D], token by token from the layout; tail: the last of them lie in the tail."""
    t = torch.arange(n, device=DEV)
    blk, s = t // TB, t % TB
    full = n // TB * TB if tail else n
    if side == 0:
        codes = c["k8"][b, h].movedim(3, 2).reshape(-1, 4, 16, D)[blk, s // 16, s % 16]
        at = c["k_tail"][b, h][s[full:]]
    else:
        codes = c["v8"][b, h].flatten(2)[blk, :, (s // 4 % 4) * 16 + s // 16 * 4 + s % 4]
        r = s[full:]
        at = c["v_tail"][b, h].flatten(1)[:, (r // 4 % 4) * 16 + r // 16 * 4 + r % 4].T
    table = torch.tensor(_E4M3 + [math.nan], dtype=torch.float64, device=DEV)
    x = table[(codes & 127).long()] * torch.where(codes > 127, -1.0, 1.0).double() * torch.exp2(c["exps"][b, h, blk, side].double()).view(n, 1)
    x[full:] = at.double()
    return x


def _place():
    s = torch.arange(TB, device=DEV)
    return (s // 4 % 4) * 16 + s // 16 * 4 + s % 4


def _exact_tail(c, b, h, side, x):
    """float64 [m, D], m <= 64, into the first slots of a tail of the float64 copies `c`."""
    if side == 0:
        c["k_tail"][b, h, :len(x)] = x
    else:
        c["v_tail"][b, h].view(x.shape[1], TB)[:, _place()[:len(x)]] = x.T


def _exact_copy(c):
    return {**{k: c[k + "8"].view(torch.float8_e4m3fn).double() for k in ("k", "v")}, "exps": c["exps"].clone(), "k_tail": c["k_tail"].double(),
            "v_tail": c["v_tail"].double(), "lens": c["lens"].clone()}


def _exact_turned(case, s, x, weight, first, m):
    """float64 [m, H, D]: the m tokens x [m, H, D], normed and turned as complex numbers, at the places first, first + 1, .."""
    x = x.double()
    if weight is not None:
        x = x * weight.double() * torch.rsqrt((x * x).sum(dim=2, keepdim=True) / case["D"] + EPS)
    half = case["rot"] // 2
    if half:
        turn = torch.polar(torch.ones(m, 1, half, dtype=torch.float64, device=DEV),
                           torch.outer(torch.arange(first, first + m, device=DEV).double(), s["freq"].double()).view(m, 1, half))
        if case["pairs"]:
            z = torch.view_as_complex(x[:, :, :2 * half].reshape(m, -1, half, 2).contiguous()) * turn
            x = torch.cat([torch.view_as_real(z).flatten(2), x[:, :, 2 * half:]], dim=2)
        else:
            z = torch.complex(x[:, :, :half].contiguous(), x[:, :, half:2 * half].contiguous()) * turn
            x = torch.cat([z.real, z.imag, x[:, :, 2 * half:]], dim=2)
    return x


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    B, Hkv, D, dtype = case["B"], case["Hkv"], case["D"], case["dtype"]
    lens = c["lens"].tolist()
    if case["kind"] == "shared":
        n, W, G = case["n"], B // case["Bp"], case["Hq"] // Hkv
        out, first = s["out"].double(), s["p"]["lens"].tolist()
        n_q = [n] * B if s["n_q"] is None else s["n_q"].tolist()
        for p in range(case["Bp"]):
            for h in range(Hkv):
                KP, VP = (_exact_tokens(s["p"], p, h, side, first[p], D) for side in (0, 1))
                for b in range(p * W, (p + 1) * W):
                    K, V = (torch.cat([x, _exact_tokens(c, b, h, side, lens[b], D)]) for side, x in ((0, KP), (1, VP)))
                    L, m = len(K), n_q[b]
                    x = (s["q"][b, h * G:(h + 1) * G, :m].double().reshape(G * m, D) @ K.T / math.sqrt(D)).view(G, m, L)
                    past = torch.arange(L, device=DEV).view(1, L) > (L - m + torch.arange(m, device=DEV)).view(m, 1)
                    x.masked_fill_(past, -math.inf)
                    lse = torch.logsumexp(x, dim=2, keepdim=True)
                    w = torch.where(past, 0.0, torch.exp(x - torch.where(lse == -math.inf, 0.0, lse)))
                    out[b, h * G:(h + 1) * G, :m] = (w.view(G * m, L) @ V).view(G, m, D)
        return {"out": out}
    if case["kind"] == "rotated":
        n, r, out = case["n"], _exact_copy(c), s["out"].double()
        counts = [n] * B if s["n_new"] is None else s["n_new"].tolist()
        base = [0] * B if s["base"] is None else s["base"].repeat_interleave(B // case["Bp"]).tolist()
        largest = float(torch.finfo(TYPES[dtype]).max)
        for b in range(B):
            had, m, at = lens[b] % TB, counts[b], lens[b] // TB
            out[b, :, :m] = _exact_turned(case, s, s["q"][b, :m], s["norms"][0], base[b] + lens[b], m).transpose(0, 1)
            fresh = (_exact_turned(case, s, s["k"][b, :m], s["norms"][1], base[b] + lens[b], m), s["v"][b, :m].double())
            nb = (had + m) // TB
            for h in range(Hkv):
                for side in (0, 1):
                    old = _exact_tokens(c, b, h, side, lens[b], D)[lens[b] - had:]
                    x = torch.cat([old, fresh[side][:, h]])
                    if nb:
                        num, e = _exact_block(x[:nb * TB].to(TYPES[dtype]).double().view(nb, TB, D), largest)
                        if side == 0:
                            r["k"][b, h, at:at + nb] = num.view(nb, 4, 16, D // 64, 64).movedim(3, 2)
                        else:
                            v = num.new_empty(nb, D, TB)
                            v[:, :, _place()] = num.transpose(1, 2)
                            r["v"][b, h, at:at + nb] = v.view(nb, D, 4, 4, 4)
                        r["exps"][b, h, at:at + nb, side] = e.to(torch.int8)
                    _exact_tail(r, b, h, side, x[nb * TB:])
            r["lens"][b] = lens[b] + m
        return {"q": out, **r}
    # copies and cuts: bytes stay what they are, and a block that is cut gives its values to the tail
    src, r = c, _exact_copy(s["d"] if case["kind"] == "fork" else c)
    parents = s["parents"].tolist() if case["kind"] == "fork" else list(range(B))
    upto = s["keep"].tolist() if case["kind"] == "truncate" else [case["N"]] * B if s["upto"] is None else s["upto"].tolist()
    score = s["d"]["score"].double() if case["kind"] == "fork" and case["score"] else None
    for b, a in enumerate(parents):
        if a < 0:
            continue
        L = min(lens[a], upto[b])
        nb = L // TB
        if case["kind"] == "fork":
            for k in ("k", "v"):
                r[k][b, :, :nb] = src[k + "8"][a, :, :nb].view(torch.float8_e4m3fn).double()
            r["exps"][b, :, :nb] = src["exps"][a, :, :nb]
            if score is not None:
                score[b, :, :L] = src["score"][a, :, :L].double()
            if L % TB and nb == lens[a] // TB:
                for k in ("k_tail", "v_tail"):
                    r[k][b] = src[k][a].double()
        if L % TB and nb < lens[a] // TB:
            for h in range(Hkv):
                for side in (0, 1):
                    _exact_tail(r, b, h, side, _exact_tokens(src, a, h, side, (nb + 1) * TB, D, tail=False)[nb * TB:])
        r["lens"][b] = L
    if case["kind"] == "fork":
        return {**r, "score": score}
    return {k: r[k] for k in ("k_tail", "v_tail", "lens")}
