"""The operators of the block-scaled 8-bit cache as cases that can be timed and compared: storing tokens, attention of one or
many query tokens over what is stored, and eviction by accumulated attention weight.

A cache holds complete blocks of 64 tokens as e4m3 numbers with one power of two per block, KV head and side (K, V), and the
tokens of the last, incomplete block in 16 bits (``include/akb.h`` says which byte lies where).  ``prepare`` lays such a cache
out with torch alone, so that both forms work on the same bytes:

* the plain form (``own`` false) in elementary torch operations, 32 bits, rounded once at the end;
* the library's calls (``own`` true).

``exact`` goes from the same inputs to the results in 64 bits, by the definition and written apart from the plain form.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TB = 64                      # tokens per block
E_MIN = -100                 # least exponent of a block's scale
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
OUTS = {"f32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
TOP_EXP = {"fp16": 8, "bf16": 120}     # the scale at which 256 times it is no number of the type any more
MOST_VALUES = 16 * 32 * 8192 * 128     # (sequence, KV head) x tokens x channels of the largest listed cache
MOST_PAIRS = 32 * 8192 * 8192 * 128    # heads x query tokens x stored tokens x channels of the largest listed prompt


# ------------------------------------------------------------------------------------------------------ cases

def _attention(name, B, Hq, Hkv, N, n, dtype, out, *, D=128, data="scales", ragged=False, score=False):
    return dict(name=name, kind="attention", B=B, Hq=Hq, Hkv=Hkv, D=D, N=N, n=n, dtype=dtype, out=out, data=data, ragged=ragged, score=score)


def _append(name, B, Hkv, start, n, dtype, *, D=128, data="scales", ragged=False):
    return dict(name=name, kind="append", B=B, Hkv=Hkv, D=D, start=start, n=n, dtype=dtype, data=data, ragged=ragged)


def _evict(name, B, Hkv, N, keep, recent, dtype, *, D=128, data="scales", ragged=False):
    return dict(name=name, kind="evict", B=B, Hkv=Hkv, D=D, N=N, keep=keep, recent=recent, dtype=dtype, data=data, ragged=ragged)


def listed() -> list[dict]:
    return [
        # one user, a short chat, one layer with full heads: the smallest attention call, where latency counts
        _attention("decode_mha_1k", 1, 32, 32, 1024, 1, "fp16", "f32", data="plain"),
        # a full batch at the benchmark's size, full heads: the most cache bytes
        _attention("decode_mha_8k", 16, 32, 32, 8192, 1, "fp16", "f32"),
        # long documents of mixed lengths, grouped heads; the weights are added up for a later eviction
        _attention("decode_gqa4_128k_score", 4, 32, 8, 131072, 1, "bf16", "bf16", data="student", ragged=True, score=True),
        # a draft of five tokens checked in one call, 64 query heads on 8, mixed odd lengths
        _attention("draft5_gqa8_13k", 3, 64, 8, 13000, 5, "fp16", "fp16", ragged=True),
        # small heads, a batch of short conversations
        _attention("decode_d64_gqa4_3001", 24, 16, 4, 3001, 1, "bf16", "f32", D=64, ragged=True),
        # a whole prompt over itself: the most operations
        _attention("prompt_gqa4_8k", 1, 32, 8, 8192, 8192, "bf16", "bf16"),
        # a chunk of a chunked prompt behind what is stored, chunks of mixed lengths, weights added up
        _attention("chunk_mha_777_of_20k_score", 2, 32, 32, 20001, 777, "fp16", "fp16", ragged=True, score=True),
        # one serving step's new token of every sequence: the smallest call of all
        _append("append_1", 64, 8, 1000, 1, "fp16", ragged=True),
        # a batch of prompts stored from empty
        _append("append_prompt_8k", 8, 8, 0, 8192, "bf16"),
        # chunks of mixed lengths onto sequences that end anywhere
        _append("append_chunk_777", 6, 32, 9001, 777, "fp16", ragged=True),
        # a batch brought down to a budget of 2048 tokens
        _evict("evict_8k_to_2k", 8, 32, 8192, 2048, 512, "fp16"),
        # few heads with very long sequences, odd sizes
        _evict("evict_128k_to_16k", 1, 8, 131001, 16384, 999, "bf16", data="student"),
    ]


def _log(rng, lo, hi):
    """A whole number, its logarithm uniform over [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng) -> dict:
    kind = rng.choice(["attention"] * 6 + ["append"] * 2 + ["evict"] * 2)
    D, dtype = rng.choice([64, 128, 128, 128]), rng.choice(["fp16", "bf16"])
    data, ragged = rng.choice(["plain", "scales", "student"]), rng.random() < 0.5
    if kind == "attention":
        G, N = rng.choice([1, 1, 2, 4, 4, 5, 8, 16]), _log(rng, 60, 131072)
        Hkv = rng.choice([h for h in (2, 8, 8, 32) if h * N * D <= MOST_VALUES])
        B = _log(rng, 1, max(1, min(64, MOST_VALUES // (Hkv * N * D))))
        n = 1
        if rng.random() < 0.5:
            n = _log(rng, 2, max(2, min(8192, N, MOST_PAIRS // (B * Hkv * G * N * 128))))
        return dict(kind=kind, B=B, Hq=Hkv * G, Hkv=Hkv, D=D, N=N, n=n, dtype=dtype, out=rng.choice(["f32", dtype]), data=data, ragged=ragged,
                    score=rng.random() < 0.3)
    if kind == "append":
        n, start = _log(rng, 1, 8192), rng.choice([0, rng.randrange(1, 8192)])
        Hkv = rng.choice([2, 8, 8, 32])
        B = _log(rng, 1, max(1, min(128, 8 * 8 * 16384 * 128 // (Hkv * (start + n) * D))))
        return dict(kind=kind, B=B, Hkv=Hkv, D=D, start=start, n=n, dtype=dtype, data=data, ragged=ragged)
    N = _log(rng, 200, 131072)
    keep = max(64, int(N * rng.choice([0.1, 0.25, 0.5, 0.9])) + rng.randrange(0, 64))
    Hkv = rng.choice([h for h in (2, 8, 8, 32) if h * N * D <= MOST_VALUES // 8])
    B = _log(rng, 1, max(1, min(32, MOST_VALUES // (8 * Hkv * N * D))))
    return dict(kind=kind, B=B, Hkv=Hkv, D=D, N=N, keep=keep, recent=rng.choice([0, 32, keep // 4, keep // 2]), dtype=dtype, data=data, ragged=ragged)


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


def _buffers(B, Hkv, D, Ncap, dtype, score):
    NB = -(-Ncap // TB)
    z = lambda *s, t=torch.uint8: torch.zeros(*s, dtype=t, device=DEV)
    return dict(k8=z(B, Hkv, NB, 4, D // 64, 16, 64), v8=z(B, Hkv, NB, D, 4, 4, 4), exps=z(B, Hkv, NB, 2, t=torch.int8),
                k_tail=z(B, Hkv, TB, D, t=TYPES[dtype]), v_tail=z(B, Hkv, D, 4, 4, 4, t=TYPES[dtype]),
                score=z(B, Hkv, NB * TB, t=torch.float32) if score else None, lens=z(B, t=torch.int32), flags=z(4 + B, t=torch.int32))


def _handle(case, c, Hq, n, keep=0):
    """The library's cache object over the buffers of `c`, with a workspace for calls of up to n query tokens, or of keep tokens."""
    from paper_2409_16546_amd import binding as A
    h = A.BlockCache(case["B"], Hq, case["Hkv"], case["D"], c["exps"].shape[2] * TB, TYPES[case["dtype"]], c["k8"], c["v8"], c["exps"], c["k_tail"],
                     c["v_tail"], c["lens"], c["flags"], c["score"])
    return h.reserve(n, keep)


# ----------------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) & 0x7FFFFFFF)


def _tokens(case, gen, n, scales):
    """16-bit [Hkv, n, D] of the case's distribution; `scales`: the channels' sizes [Hkv, 1, D]."""
    x = torch.randn(case["Hkv"], n, case["D"], generator=gen, device=DEV) * scales
    if case["data"] == "student":   # Student-t, three degrees of freedom
        x /= sum(torch.randn(case["Hkv"], n, case["D"], generator=gen, device=DEV).square_() for _ in range(3)).div_(3).sqrt_()
    return x.clamp_(-65504, 65504).to(TYPES[case["dtype"]])


def _scales(case, gen):
    shape = (case["Hkv"], 1, case["D"])
    return torch.pow(10.0, torch.rand(shape, generator=gen, device=DEV) * 2 - 1) if case["data"] == "scales" else torch.ones(shape, device=DEV)


def _lens(case, gen, N):
    if not case["ragged"] or N == 0:
        return torch.full((case["B"],), N, dtype=torch.int32, device=DEV)
    return torch.randint(max(1, N // 4), N + 1, (case["B"],), generator=gen, device=DEV).to(torch.int32)


def _filled(case, gen, N, Ncap, score):
    """A cache whose sequences hold up to N tokens."""
    c = _buffers(case["B"], case["Hkv"], case["D"], Ncap, case["dtype"], score)
    c["lens"].copy_(_lens(case, gen, N))
    NB = N // TB
    ks, vs = _scales(case, gen), _scales(case, gen)
    for b in range(case["B"]):
        for side, (scales, view, tail) in enumerate(((ks, _rows(c["k8"])[b], c["k_tail"][b].view(-1, 4, 4, 4, case["D"])),
                                                     (vs, _columns(c["v8"])[b], _tail_columns(c["v_tail"])[b]))):
            for h in range(0, case["Hkv"], 8):   # eight heads at a time keep the temporaries small
                part = dict(case, Hkv=min(8, case["Hkv"] - h))
                x = _tokens(part, gen, (NB + 1) * TB, scales[h:h + 8]).view(-1, NB + 1, TB, case["D"])
                codes, e = _pack(x[:, :NB].float(), case["dtype"])
                view[h:h + 8, :NB] = codes.view(len(codes), NB, *view.shape[2:])
                c["exps"][b, h:h + 8, :NB, side] = e
                tail[h:h + 8] = x[:, NB].reshape(tail[h:h + 8].shape)
    return c


def prepare(case, seed):
    gen = _gen(seed)
    B, Hkv, D, dt = case["B"], case["Hkv"], case["D"], TYPES[case["dtype"]]
    if case["kind"] == "attention":
        Hq, n, N = case["Hq"], case["n"], case["N"]
        s = dict(case=case, c=_filled(case, gen, N, N, case["score"]))
        s["q"] = torch.randn(B, Hq, n, D, generator=gen, device=DEV).to(dt)
        s["n_q"] = torch.randint(max(1, n // 3), n + 1, (B,), generator=gen, device=DEV).to(torch.int32) if case["ragged"] and n > 1 else None
        s["out"] = torch.zeros(B, Hq, n, D, dtype=OUTS[case["out"]], device=DEV)
        if case["score"]:
            s["score"] = torch.rand(s["c"]["score"].shape, generator=gen, device=DEV)
        if own:
            s["handle"] = _handle(case, s["c"], Hq, n)
    elif case["kind"] == "append":
        start, n = case["start"], case["n"]
        s = dict(case=case, c=_filled(case, gen, start, start + n + TB, True))
        s["ends"] = {k: s["c"][k].clone() for k in (("lens", "k_tail", "v_tail") if start and n > 1 else ("lens",))}
        ks, vs = _scales(case, gen), _scales(case, gen)
        s["k"] = torch.stack([_tokens(case, gen, n, ks) for _ in range(B)])
        s["v"] = torch.stack([_tokens(case, gen, n, vs) for _ in range(B)])
        s["n_new"] = torch.randint(max(1, n // 3), n + 1, (B,), generator=gen, device=DEV).to(torch.int32) if case["ragged"] else None
        if own:
            s["handle"] = _handle(case, s["c"], Hkv, 1)
    else:
        N = case["N"]
        s = dict(case=case, c=_filled(case, gen, N, N, True))
        score = torch.exp(2 * torch.randn(s["c"]["score"].shape, generator=gen, device=DEV))
        s["c"]["score"].copy_(torch.where(score < 0.05, 0.0, score))   # some tokens that nothing looked at
        s["d"] = _buffers(B, Hkv, D, case["keep"] + TB, case["dtype"], True)
        s["kept"] = torch.zeros(B, Hkv, case["keep"], dtype=torch.int32, device=DEV)
        if own:
            s["handle"], s["to"] = _handle(case, s["c"], Hkv, 1, case["keep"]), _handle(case, s["d"], Hkv, 1)
    return s


# ------------------------------------------------------------------------------------------------- the plain form

def _pack(x, dtype):
    """x: float32 [..., 64, D] -> (codes as uint8, exponents as int8 [...]): the least e with max|x| <= 448 2^e, codes to the nearest."""
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
    return _values(_columns(c["v8"]), c["exps"][..., 1], _tail_columns(c["v_tail"]), c["lens"])


def _attention_plain(s):
    case, c, q = s["case"], s["c"], s["q"]
    B, Hq, Hkv, D, n = case["B"], case["Hq"], case["Hkv"], case["D"], case["n"]
    G, N = Hq // Hkv, c["exps"].shape[2] * TB
    lens = c["lens"].view(B, 1, 1, 1, 1)
    n_q = lens.new_full((B, 1, 1, 1, 1), n) if s["n_q"] is None else s["n_q"].view(B, 1, 1, 1, 1)
    i, t = torch.arange(n, device=DEV).view(1, 1, 1, n, 1), torch.arange(N, device=DEV)
    seen = (t <= lens - n_q + i) & (t < lens) & (i < n_q)                           # [B, 1, 1, n, N]
    v = torch.where((t < lens).view(B, 1, N, 1), _v_values(c), 0.0)
    x = torch.matmul(q.float().view(B, Hkv, G * n, D), _k_values(c).transpose(2, 3).contiguous()).view(B, Hkv, G, n, N) * (1 / math.sqrt(D))
    x = torch.where(seen, x, -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    z = p.sum(dim=-1, keepdim=True)
    p = p / torch.where(z == 0, 1.0, z)
    o = torch.matmul(p.view(B, Hkv, G * n, N), v).view(B, Hq, n, D)
    out = torch.where((i < n_q).view(B, 1, n, 1), o.to(s["out"].dtype), s["out"])
    s["out"].copy_(out)
    if case["score"]:
        c["score"] += p.sum(dim=(2, 3))


def _append_plain(s):
    case, c = s["case"], s["c"]
    B, Hkv, D, n = case["B"], case["Hkv"], case["D"], case["n"]
    lens = c["lens"].long()
    count = torch.full_like(lens, n) if s["n_new"] is None else s["n_new"].long()
    NW = -(-(TB - 1 + n) // TB)                                                     # blocks that an append can touch
    w = torch.arange(NW * TB, device=DEV).view(1, 1, NW * TB, 1)
    had, total = (lens % TB).view(B, 1, 1, 1), (lens % TB + count).view(B, 1, 1, 1)
    src = (w - had).clamp(0, n - 1).expand(B, Hkv, NW * TB, D)
    first = (w[:, :, :TB]).expand(B, Hkv, TB, D)
    new = torch.arange(NW, device=DEV).view(1, NW) < (total.view(B, 1) // TB)         # blocks that are complete now
    blocks = (lens // TB).view(B, 1) + torch.arange(NW, device=DEV).view(1, NW)
    last = (total // TB).view(B, 1, 1, 1).clamp(max=NW - 1)
    slot = last * TB + w[:, :, :TB]                                                 # where the tail's slots lie among the blocks
    keep = (slot < had) | (slot >= total) | (total // TB >= NW)
    for side, (fresh, view, tail) in enumerate(((s["k"], _rows(c["k8"]), c["k_tail"].view(B, Hkv, 4, 4, 4, D)),
                                                (s["v"], _columns(c["v8"]), _tail_columns(c["v_tail"])))):
        x = fresh.gather(2, src)
        old = tail.reshape(B, Hkv, TB, D)
        x[:, :, :TB] = torch.where(first < had, old, x[:, :, :TB])
        codes, e = _pack(x.view(B, Hkv, NW, TB, D).float(), case["dtype"])
        b = torch.arange(B, device=DEV).view(B, 1)
        codes = codes.view(B, Hkv, NW, *view.shape[3:]).transpose(1, 2)             # [B, NW, Hkv, ...]
        mask = new.view(B, NW, 1, 1, 1, 1, 1)[..., :1]
        view[b, :, blocks] = torch.where(mask.view(B, NW, *(1,) * (codes.dim() - 2)), codes, view[b, :, blocks])
        ex = c["exps"][..., side]
        ex[b, :, blocks] = torch.where(new.view(B, NW, 1), e.transpose(1, 2), ex[b, :, blocks])
        tail.copy_(torch.where(keep, old, x.gather(2, slot.expand(B, Hkv, TB, D))).view(tail.shape))
    t = torch.arange(c["score"].shape[2], device=DEV).view(1, 1, -1)
    at = lens.view(B, 1, 1)
    c["score"].masked_fill_((t >= at) & (t < at + count.view(B, 1, 1)), 0.0)
    c["lens"].copy_(lens + count)


def _evict_plain(s):
    case, c, d = s["case"], s["c"], s["d"]
    B, Hkv, D, keep = case["B"], case["Hkv"], case["D"], case["keep"]
    N, NBd = c["score"].shape[2], d["exps"].shape[2]
    lens = c["lens"].long().view(B, 1, 1)
    count = lens.clamp(max=keep)
    t = torch.arange(N, device=DEV).view(1, 1, N)
    score = torch.where(t >= lens - count.clamp(max=case["recent"]), math.inf, c["score"])
    order = torch.sort(torch.where(t < lens, score, -math.inf), dim=2, descending=True, stable=True).indices
    rank = torch.arange(min(keep, N), device=DEV).view(1, 1, -1)
    kept = torch.where(rank < count, order[:, :, :keep], N).sort(dim=2).values
    kept = torch.cat([kept, kept.new_full((B, Hkv, keep - kept.shape[2]), N)], dim=2)
    s["kept"].copy_(torch.where(kept < N, kept, -1))
    at = torch.cat([kept, kept.new_full((B, Hkv, NBd * TB - keep), N)], dim=2).clamp(max=N - 1)
    slot = torch.arange(TB, device=DEV).view(1, 1, TB, 1)
    left = (count % TB).view(B, 1, 1, 1)
    whole = torch.arange(NBd, device=DEV).view(1, 1, NBd) < count // TB
    last = ((count // TB).view(B, 1, 1, 1).clamp(max=NBd - 1) * TB + slot).expand(B, Hkv, TB, D)
    for side, (values, view, tail) in enumerate(((_k_values(c), _rows(d["k8"]), d["k_tail"].view(B, Hkv, 4, 4, 4, D)),
                                                 (_v_values(c), _columns(d["v8"]), _tail_columns(d["v_tail"])))):
        x = values.gather(2, at.view(B, Hkv, NBd * TB, 1).expand(B, Hkv, NBd * TB, D))
        codes, e = _pack(x.view(B, Hkv, NBd, TB, D), case["dtype"])
        view.copy_(torch.where(whole.view(B, 1, NBd, *(1,) * (view.dim() - 3)), codes.view(view.shape), view))
        ex = d["exps"][..., side]
        ex.copy_(torch.where(whole, e, ex))
        tail.copy_(torch.where(slot < left, x.gather(2, last).to(tail.dtype), tail.reshape(B, Hkv, TB, D)).view(tail.shape))
    rows = torch.arange(NBd * TB, device=DEV).view(1, 1, -1)
    d["score"].copy_(torch.where(rows < count, c["score"].gather(2, at), d["score"]))
    d["lens"].copy_(count.view(B))


def run(s):
    case, c = s["case"], s["c"]
    if case["kind"] == "attention":
        if case["score"]:
            c["score"].copy_(s["score"])
        if own:
            from paper_2409_16546_amd import binding as A
            A.akb_attention(s["handle"], s["q"], s["out"], n_q=s["n_q"], accumulate=case["score"])
        else:
            _attention_plain(s)
        return {"out": s["out"], "score": c["score"]} if case["score"] else {"out": s["out"]}
    if case["kind"] == "append":
        for k, end in s["ends"].items():   # the sequences end where they ended before
            c[k].copy_(end)
        if own:
            from paper_2409_16546_amd import binding as A
            A.akb_append(s["handle"], s["k"], s["v"], s["n_new"])
        else:
            _append_plain(s)
        return _outputs(c)
    if own:
        from paper_2409_16546_amd import binding as A
        A.akb_evict(s["handle"], s["to"], case["keep"], case["recent"], kept=s["kept"])
    else:
        _evict_plain(s)
    return {**_outputs(s["d"]), "kept": s["kept"]}


def _outputs(c):
    """A cache as what it stands for: e4m3 numbers, the exponents of their scales, the tails, scores and lengths."""
    return {"k": c["k8"].view(torch.float8_e4m3fn), "v": c["v8"].view(torch.float8_e4m3fn), "exps": c["exps"], "k_tail": c["k_tail"], "v_tail": c["v_tail"],
            "score": c["score"], "lens": c["lens"]}


# ----------------------------------------------------------------------------------------------------------- work

def _mean_len(case, N):
    return N if not case["ragged"] else (max(1, N // 4) + N) / 2


def work(case):
    B, Hkv, D = case["B"], case["Hkv"], case["D"]
    if case["kind"] == "attention":
        n, N = case["n"], _mean_len(case, case["N"])
        m = (max(1, n // 3) + n) / 2 if case["ragged"] and n > 1 else n       # query tokens of a sequence
        m = min(m, N)
        kv = B * Hkv * N * (2 * D + 2 / TB + (8 if case["score"] else 0))
        io = B * case["Hq"] * m * D * (2 + (4 if case["out"] == "f32" else 2))
        return {"bytes": kv + io, "flops": 4 * D * B * case["Hq"] * (m * N - m * (m - 1) / 2)}
    if case["kind"] == "append":
        n = case["n"]
        m = (max(1, n // 3) + n) / 2 if case["ragged"] else n
        out = 2 * D if n >= TB else 4 * D
        return {"bytes": B * Hkv * m * (4 * D + out + 4), "flops": 0}
    L = _mean_len(case, case["N"])
    kept = min(L, case["keep"])
    return {"bytes": B * Hkv * (4 * L + kept * (4 * D + 8)), "flops": 0}


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


def _exact_tokens(c, b, h, side, n, D):
    """The stored values of one head as float64 [n, D], token by token from the layout."""
    t = torch.arange(n, device=DEV)
    blk, s = t // TB, t % TB
    full = n // TB * TB
    if side == 0:
        codes = c["k8"][b, h].movedim(3, 2).reshape(-1, 4, 16, D)[blk, s // 16, s % 16]
        tail = c["k_tail"][b, h][s[full:]]
    else:
        codes = c["v8"][b, h].flatten(2)[blk, :, (s // 4 % 4) * 16 + s // 16 * 4 + s % 4]
        at = s[full:]
        tail = c["v_tail"][b, h].flatten(1)[:, (at // 4 % 4) * 16 + at // 16 * 4 + at % 4].T
    table = torch.tensor(_E4M3 + [math.nan], dtype=torch.float64, device=DEV)
    x = table[(codes & 127).long()] * torch.where(codes > 127, -1.0, 1.0).double() * torch.exp2(c["exps"][b, h, blk, side].double()).view(n, 1)
    x[full:] = tail.double()
    return x


def _exact_cache(c, b, h, side, x, D, dtype, first):
    """Stores float64 tokens x[m, D] at place `first` (the beginning of a block) of head (b, h) of the float64 copies `c`."""
    m = x.shape[0]
    nb = m // TB
    largest = float(torch.finfo(TYPES[dtype]).max)
    num, e = _exact_block(x[:nb * TB].view(nb, TB, D), largest) if nb else (x.new_zeros(0, TB, D), x.new_zeros(0))
    at = first // TB
    s = torch.arange(TB, device=DEV)
    place = (s // 4 % 4) * 16 + s // 16 * 4 + s % 4
    if side == 0:
        c["k"][b, h, at:at + nb] = num.view(nb, 4, 16, D // 64, 64).movedim(3, 2)
    else:
        v = num.new_empty(nb, D, TB)
        v[:, :, place] = num.transpose(1, 2)
        c["v"][b, h, at:at + nb] = v.view(nb, D, 4, 4, 4)
    c["exps"][b, h, at:at + nb, side] = e.to(torch.int8)
    return x[nb * TB:]


def _exact_copy(c):
    return {**{k: c[k + "8"].view(torch.float8_e4m3fn).double() for k in ("k", "v")}, "exps": c["exps"].clone(), "k_tail": c["k_tail"].double(),
            "v_tail": c["v_tail"].double(), "score": c["score"].double(), "lens": c["lens"].clone()}


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    B, Hkv, D, dtype = case["B"], case["Hkv"], case["D"], case["dtype"]
    lens = c["lens"].tolist()
    slots = torch.arange(TB, device=DEV)
    place = (slots // 4 % 4) * 16 + slots // 16 * 4 + slots % 4
    if case["kind"] == "attention":
        n, G = case["n"], case["Hq"] // Hkv
        out, score = s["out"].double(), s["score"].double() if case["score"] else None
        n_q = [n] * B if s["n_q"] is None else s["n_q"].tolist()
        for b in range(B):
            L, m = lens[b], n_q[b]
            for h in range(Hkv):
                K, V = (_exact_tokens(c, b, h, side, L, D) for side in (0, 1))
                for g in range(G):
                    x = s["q"][b, h * G + g, :m].double() @ K.T / math.sqrt(D)
                    past = torch.arange(L, device=DEV).view(1, L) > (L - m + torch.arange(m, device=DEV)).view(m, 1)
                    x.masked_fill_(past, -math.inf)
                    lse = torch.logsumexp(x, dim=1, keepdim=True)
                    p = torch.where(past, 0.0, torch.exp(x - torch.where(lse == -math.inf, 0.0, lse)))
                    out[b, h * G + g, :m] = p @ V
                    if score is not None:
                        score[b, h, :L] += p.sum(dim=0)
        return {"out": out, "score": score} if case["score"] else {"out": out}
    if case["kind"] == "append":
        r = _exact_copy(c)
        counts = [case["n"]] * B if s["n_new"] is None else s["n_new"].tolist()
        for b in range(B):
            had, m = lens[b] % TB, counts[b]
            for h in range(Hkv):
                for side, fresh in enumerate((s["k"], s["v"])):
                    tail = r["k_tail"][b, h, :had] if side == 0 else r["v_tail"][b, h].flatten(1)[:, place[:had]].T
                    x = torch.cat([tail, fresh[b, h, :m].double()])
                    rest = _exact_cache(r, b, h, side, x, D, dtype, lens[b] - had)
                    if side == 0:
                        r["k_tail"][b, h, :len(rest)] = rest
                    else:
                        r["v_tail"][b, h].view(D, TB)[:, place[:len(rest)]] = rest.T
            r["score"][b, :, lens[b]:lens[b] + m] = 0
            r["lens"][b] = lens[b] + m
        return r
    d = s["d"]
    r = _exact_copy(d)
    kept = torch.full_like(s["kept"], -1)
    for b in range(B):
        L, m = lens[b], min(lens[b], case["keep"])
        sure = min(case["recent"], m)
        for h in range(Hkv):
            sc = c["score"][b, h, :L].double()
            order = np.lexsort((np.arange(L - sure), -sc[:L - sure].cpu().numpy()))[:m - sure]   # by score, then by place
            at = torch.cat([torch.from_numpy(np.sort(order)).to(DEV), torch.arange(L - sure, L, device=DEV)])
            kept[b, h, :m] = at.to(torch.int32)
            r["score"][b, h, :m] = sc[at]
            for side in (0, 1):
                rest = _exact_cache(r, b, h, side, _exact_tokens(c, b, h, side, L, D)[at], D, dtype, 0)
                if side == 0:
                    r["k_tail"][b, h, :len(rest)] = rest
                else:
                    r["v_tail"][b, h].view(D, TB)[:, place[:len(rest)]] = rest.T
        r["lens"][b] = m
    return {**r, "kept": kept}
