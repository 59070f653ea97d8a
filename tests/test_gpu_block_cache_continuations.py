"""Several continuations of prompts as a server runs them: prompts stored from projections and attended, copies, steps behind the shared prefixes, beams put in a new order, drafts checked and cut
back; against the 64-bit reference all along, eagerly and in a graph."""
import numpy as np
import pytest
import torch

import block_cache_ref as R
import block_cache_share_ref as S
from test_gpu_block_cache import A, B16, DEV, F16, i32, pair  # noqa: F401
from test_gpu_block_cache_rotated import check_turned, freqs, projected, weight

pytestmark = pytest.mark.gpu


class Side:
    """A cache, its reference, and how its tokens are turned."""

    def __init__(self, A, B, Hq, Hkv, D, Ncap, dtype, pairs):
        self.A, (self.c, self.r) = A, pair(A, B, Hq, Hkv, D, Ncap, dtype)
        self.freq, self.qw, self.kw, self.pairs = freqs(D), weight(D, dtype, 1), weight(D, dtype, 2), pairs

    def store(self, n, seed, n_new=None, base=None):
        """n new projected tokens of every sequence -> their turned queries; the reference takes the keys' 64-bit results, rounded once."""
        c = self.c
        q, k, v = projected(c.B, n, c.Hq, c.Hkv, c.D, c.dtype, seed, True, "plain")
        lens = [self.r.len(b) for b in range(c.B)]
        out = self.A.akb_append_rotated(c, q, k, v, inv_freq=self.freq, q_norm=self.qw, k_norm=self.kw, eps=1e-6, pairs=self.pairs, n_new=i32(n_new), base=base)
        base = [0] * c.B if base is None else base.repeat_interleave(c.B // len(base)).tolist()
        turned = torch.zeros(c.B, c.Hkv, n, c.D, dtype=c.dtype)
        for b in range(c.B):
            m = n if n_new is None else n_new[b]
            at = range(base[b] + lens[b], base[b] + lens[b] + m)
            eps = float(np.float32(1e-6))
            x, _ = S.turned(k[b, :m].double().cpu().numpy(), at, self.freq.double().cpu().numpy(), self.kw.double().cpu().numpy(), eps, self.pairs)
            turned[b, :, :m] = torch.from_numpy(x.transpose(1, 0, 2).copy()).float().to(c.dtype)
            check_turned(out[b, :, :m], q[b, :m], at, self.freq, self.qw, eps, self.pairs, c.dtype, f"q {b}")
        self.r.append(turned, v.transpose(1, 2), n_new)
        return out


@pytest.mark.parametrize("dtype,D,Hq,Hkv,pairs", [(F16, 128, 4, 2, False), (B16, 64, 6, 2, True)])
def test_prompts_beams_and_drafts(A, dtype, D, Hq, Hkv, pairs):
    P, W = 2, 3
    prompt, beams, other = (Side(A, b, Hq, Hkv, D, cap, dtype, pairs) for b, cap in ((P, 256), (P * W, 128), (P * W, 128)))
    first = [200, 131]
    q = prompt.store(200, 1, n_new=first)
    prompt.c.reserve(200)
    R.assert_attention(A.akb_attention(prompt.c, q, n_q=i32(first)), *prompt.r.attention(q.cpu(), first), dtype, "prompts")
    # the first new token of every beam comes from the prompt's last query: its sequence has no token of its own yet
    beams.c.reserve(5, prefix=prompt.c)
    last = torch.stack([q[b // W, :, first[b // W] - 1] for b in range(P * W)])
    R.assert_attention(A.akb_attention_shared(prompt.c, beams.c, last[:, :, None].contiguous()), *S.joined(prompt.r, beams.r).attention(last[:, :, None].cpu()), dtype, "the last of the prompt")
    rng = np.random.default_rng(3)
    for turn in range(4):
        for step in range(14):
            q = beams.store(1, 100 * turn + step + 10, base=prompt.c.lens)
            got = A.akb_attention_shared(prompt.c, beams.c, q)
            if step % 7 == 0:
                R.assert_attention(got, *S.joined(prompt.r, beams.r).attention(q.cpu()), dtype, f"turn {turn} step {step}")
        parents = [b // W * W + int(rng.integers(W)) for b in range(P * W)]      # the beams that stay, some of them twice
        A.akb_fork(beams.c, other.c, i32(parents))
        S.fork(beams.r, other.r, parents, None)
        beams, other = other, beams
        R.assert_same_tokens(A, beams.c, beams.r, f"turn {turn}: new order")
        beams.c.reserve(5, prefix=prompt.c)
        m = [int(x) for x in rng.integers(1, 6, P * W)]                          # drafts of one to five tokens, of which some stay
        q = beams.store(5, 1000 + turn, n_new=m, base=prompt.c.lens)
        R.assert_attention(A.akb_attention_shared(prompt.c, beams.c, q, n_q=i32(m)), *S.joined(prompt.r, beams.r).attention(q.cpu(), m), dtype, f"turn {turn}: drafts")
        keep = [beams.r.len(b) - int(rng.integers(0, m[b] + 1)) for b in range(P * W)]
        A.akb_truncate(beams.c, i32(keep))
        for b, k in enumerate(keep):
            S.cut(beams.r, b, k)
        R.assert_same_tokens(A, beams.c, beams.r, f"turn {turn}: cut back")
    # one beam of each prompt goes on alone, in a cache that holds its prompt, too
    alone = Side(A, P, Hq, Hkv, D, 448, dtype, pairs)
    A.akb_fork(prompt.c, alone.c)
    S.fork(prompt.r, alone.r, None, None)
    R.assert_same_tokens(A, alone.c, alone.r, "the prompts copied")
    alone.c.reserve(3)
    q = alone.store(3, 5000)
    R.assert_attention(A.akb_attention(alone.c, q), *alone.r.attention(q.cpu()), dtype, "alone")
    R.assert_same_tokens(A, prompt.c, prompt.r, "the prefixes are as they were")


def test_steps_in_graphs_that_share_a_workspace(A):
    """A step (rotated append, attention behind the prefix, beams in a new order, a cut) captured for two batches that share a workspace, replayed with eager work between."""
    dtype, Hq, Hkv, D = B16, 8, 2, 128
    prompt = Side(A, 1, Hq, Hkv, D, 1024, dtype, False)
    prompt.store(1000, 1)
    batches = []
    for seed, B in ((2, 6), (3, 4)):
        s, d = (Side(A, B, Hq, Hkv, D, 256, dtype, False) for _ in range(2))
        s.store(62, seed, n_new=[62 - b for b in range(B)])
        x = projected(B, 2, Hq, Hkv, D, dtype, seed + 10, True, "plain")
        batches.append(dict(s=s, d=d, x=x, q=torch.zeros(B, Hq, 2, D, dtype=dtype, device=DEV), out=torch.zeros(B, Hq, 2, D, device=DEV),
                            parents=i32([(b * 5 + 1) % B for b in range(B)]), keep=i32([70 - 3 * b for b in range(B)])))
    ws = batches[0]["s"].c.reserve(2, prefix=prompt.c).workspace
    assert ws.numel() >= A.lib().akb_attention_shared_workspace(prompt.c.struct().shape, batches[1]["s"].c.struct().shape, 2)

    def step(i):
        t = batches[i]
        A.akb_append_rotated(t["s"].c, *t["x"], t["q"], inv_freq=prompt.freq, q_norm=prompt.qw, k_norm=prompt.kw, base=prompt.c.lens)
        A.akb_attention_shared(prompt.c, t["s"].c, t["q"], t["out"], workspace=ws)
        A.akb_fork(t["s"].c, t["d"].c, t["parents"])
        A.akb_truncate(t["d"].c, t["keep"])
    names = ("lens", "k8", "v8", "exps", "k_tail", "v_tail")
    saved = [[getattr(t["s"].c, n).clone() for n in names] for t in batches]

    def restore():
        for t, s in zip(batches, saved):
            for n, x in zip(names, s):
                getattr(t["s"].c, n).copy_(x)
            t["d"].c.lens.zero_()
    see = lambda: [x.clone() for t in batches for x in (t["q"], t["out"], t["s"].c.lens, t["d"].c.lens, *A.akb_unpack(t["s"].c), *A.akb_unpack(t["d"].c))]
    eager = []
    for _ in range(3):
        for i in (0, 1):
            step(i)
        eager.append(see())
    restore()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.stream(s):
        step(0)
        step(1)
        torch.cuda.synchronize()
        for i in (0, 1):
            with torch.cuda.graph(graphs[i], stream=s):
                step(i)
    torch.cuda.current_stream().wait_stream(s)
    restore()
    for rep in range(3):
        for g in graphs:
            g.replay()
        A.akb_attention(prompt.c.reserve(1), torch.zeros(1, Hq, 1, D, dtype=dtype, device=DEV))   # the program's own eager work
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(see(), eager[rep])), f"replay {rep}"
