// The block-scaled 8-bit cache: sequences copied to others and cut back in place (rules and layout: include/akb.h).
#include "akb_common.h"

namespace akb {

constexpr int kThreads = 256;

// One side of a block on its way to a 16-bit tail: 16 codes become 32 bytes per thread and turn, in the orders that both already have (K: a token's run of channels; V: a
// channel's tokens)
template <class T, int D> struct TailSide {
    static constexpr int kTurns = D * 4 / kThreads;
    u32x4_t w[kTurns];
    int e;
    __device__ __forceinline__ void load(const akb_cache& c, size_t block, bool is_v, int tid)
    {
        const u32x4_t* from = reinterpret_cast<const u32x4_t*>((is_v ? c.v8 : c.k8) + block * (kTB * D));
#pragma unroll
        for (int k = 0; k < kTurns; ++k) w[k] = from[tid + k * kThreads];
        e = c.exps[block * 2 + (is_v ? 1 : 0)];
    }
    __device__ __forceinline__ void store(const akb_cache& d, size_t bh, bool is_v, int tid) const
    {
        const float s = pow2(e);
        uint16_t* to = (is_v ? d.v_tail : d.k_tail) + bh * kTB * D;
#pragma unroll
        for (int k = 0; k < kTurns; ++k) {
            const int p = tid + k * kThreads, run = p >> 2, token = run / (16 * (D / 64)) * 16 + run % 16, i = run / 16 % (D / 64);   // k8: [4][D / 64][16] runs of 64 channels
            u32x4_t* out = reinterpret_cast<u32x4_t*>(to + (is_v ? p * 16 : token * D + i * 64 + (p & 3) * 16));
            out[0] = cvt8<T>(w[k][0], w[k][1], s);
            out[1] = cvt8<T>(w[k][2], w[k][3], s);
        }
    }
};

// `pieces` of 16 bytes, PER of them per thread and turn, all asked for before the first is stored
template <int PER, bool NT> __device__ __forceinline__ void copy(const uint8_t* from, uint8_t* to, int pieces, int tid)
{
    const u32x4_t* f = reinterpret_cast<const u32x4_t*>(from);
    u32x4_t* t = reinterpret_cast<u32x4_t*>(to);
    for (int i0 = tid; i0 < pieces; i0 += PER * kThreads) {
        u32x4_t x[PER];
#pragma unroll
        for (int k = 0; k < PER; ++k) x[k] = f[min(i0 + k * kThreads, pieces - 1)];
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            if (i0 + k * kThreads >= pieces) break;
            if (NT) __builtin_nontemporal_store(x[k], t + i0 + k * kThreads);
            else t[i0 + k * kThreads] = x[k];
        }
    }
}

// A copy is bound by memory, 16 bytes out for 16 in: 7.0 TB/s where one source goes to many, 6.1 where each has its own (a plain copy moves 5.4).
// One workgroup per (chunk of blocks, side, KV head, sequence of the destination).  The complete blocks of a (sequence, KV head) lie one behind the other, so a chunk is a run of bytes.
template <class T, int D, bool NT>
__global__ __launch_bounds__(kThreads) void fork_kernel(akb_cache c, akb_cache d, const int32_t* __restrict__ parents, const int32_t* __restrict__ upto, int chunk)
{
    const int tid = threadIdx.x, h = blockIdx.y, j = blockIdx.z, first = (blockIdx.x >> 1) * chunk;
    const bool is_v = blockIdx.x & 1;
    const int a = parents ? parents[j] : j;
    if (a < 0 || a >= c.shape.B) return;
    const int had = seq_len(c, a), len = upto ? min(had, max(upto[j], 0)) : had;
    const bool front = blockIdx.x == 0 && h == 0 && tid == 0;
    if (len > d.shape.Ncap) {
        if (front) atomicAdd(&d.flags[AKV_FLAG_OVERFLOW], 1);
        return;
    }
    const size_t from = size_t(a) * c.shape.Hkv + h, to = size_t(j) * d.shape.Hkv + h, from0 = from * (c.shape.Ncap / kTB), to0 = to * (d.shape.Ncap / kTB);
    const int whole = len / kTB, n = min(chunk, whole - first);
    if (front) d.lens[j] = len;
    if (n > 0) {
        copy<4, NT>((is_v ? c.v8 : c.k8) + (from0 + first) * (kTB * D), (is_v ? d.v8 : d.k8) + (to0 + first) * (kTB * D), n * (kTB * D / 16), tid);
        if (!is_v && tid < 2 * n) d.exps[(to0 + first) * 2 + tid] = c.exps[(from0 + first) * 2 + tid];
    }
    if (is_v && d.score)   // (from a cache without scores: of tokens that no weight has been counted for, as the appends store them)
        for (int t = first * kTB + tid; t < min(len, (first + chunk) * kTB); t += kThreads)
            d.score[to * d.shape.Ncap + t] = c.score ? c.score[from * c.shape.Ncap + t] : 0.f;
    if (len % kTB && whole >= first && whole < first + chunk) {   // the incomplete block
        if (whole < had / kTB) {
            TailSide<T, D> s;
            s.load(c, from0 + whole, is_v, tid);
            s.store(d, to, is_v, tid);
        } else copy<2, false>(reinterpret_cast<const uint8_t*>((is_v ? c.v_tail : c.k_tail) + from * kTB * D), reinterpret_cast<uint8_t*>((is_v ? d.v_tail : d.k_tail) + to * kTB * D), kTB * D / 8, tid);
    }
}

hipError_t launch_fork(const akb_cache& src, const akb_cache& dst, const int32_t* parents, const int32_t* upto, hipStream_t st)
{
    // (a copy that ends with the source's capacity has no incomplete block; one that the destination has no room for is refused by the first workgroups)
    const int blocks = std::min(src.shape.Ncap, dst.shape.Ncap) / kTB;
    // Copies that are more than half of the last-level cache are stored with the non-temporal hint and shared out by single blocks; smaller ones, which the next step reads,
    // without it and in runs of eight.  Single blocks with the hint / eight without: one prompt of 8192 tokens to 16 sequences of 8 heads (268 MB) 40.8 / 60 us, 16 to 16 88
    // / 105; 64 sequences of up to 500 tokens that change places (67 MB) 27.7 / 14.3, with the next step's attention 33.3 / 26.1.
    const bool streamed = size_t(dst.shape.B) * dst.shape.Hkv * blocks * kTB * dst.shape.D * 2 > (size_t(128) << 20);
    const int chunk = streamed ? 1 : 8;
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(2 * ((blocks + chunk - 1) / chunk), dst.shape.Hkv, dst.shape.B), dim3(kThreads), 0, st, src, dst, parents, upto, chunk); };
    auto pick = [&](auto plain, auto hinted) { streamed ? launch(hinted) : launch(plain); };
    if (src.shape.dtype == AKB_FP16) src.shape.D == 64 ? pick(fork_kernel<Fp16, 64, false>, fork_kernel<Fp16, 64, true>) : pick(fork_kernel<Fp16, 128, false>, fork_kernel<Fp16, 128, true>);
    else src.shape.D == 64 ? pick(fork_kernel<Bf16, 64, false>, fork_kernel<Bf16, 64, true>) : pick(fork_kernel<Bf16, 128, false>, fork_kernel<Bf16, 128, true>);
    return hipGetLastError();
}

// A workgroup has `heads` KV heads of a sequence.  A sequence that stays inside its incomplete block, or ends with a block, only gets its length; which of its workgroups reads
// the old length and which the new makes no difference then.  Where a block goes to the tail, all have to have read the old one: the last by ticket moves it.
template <class T, int D>
__global__ __launch_bounds__(kThreads) void truncate_kernel(akb_cache c, const int32_t* __restrict__ keep, int heads)
{
    const int tid = threadIdx.x, h0 = blockIdx.x * heads, b = blockIdx.y;
    const int had = seq_len(c, b), len = min(had, max(keep[b], 0)), blk = len / kTB;
    if (len % kTB == 0 || blk == had / kTB) {
        if (blockIdx.x == 0 && tid == 0) c.lens[b] = len;
        return;
    }
    __syncthreads();   // (the length has been read by all waves)
    if (tid == 0 && atomicAdd(&c.flags[AKV_NFLAGS + b], 1) == int(gridDim.x) - 1) {
        c.flags[AKV_NFLAGS + b] = 0;
        c.lens[b] = len;
    }
    const int end = min(h0 + heads, c.shape.Hkv);
    for (int h = h0; h < end; h += 2) {   // two heads, both sides, at a time: all their codes are asked for before the first is stored
        TailSide<T, D> s[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const size_t bh = size_t(b) * c.shape.Hkv + min(h + (i >> 1), end - 1);
            s[i].load(c, bh * (c.shape.Ncap / kTB) + blk, i & 1, tid);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (h + (i >> 1) < end) s[i].store(c, size_t(b) * c.shape.Hkv + h + (i >> 1), i & 1, tid);
    }
}

constexpr int kTickets = 8;   // of a sequence, at most
hipError_t launch_truncate(const akb_cache& c, const int32_t* keep, hipStream_t st)
{
    // (16 sequences of 32 heads in 32, 8 and 2 workgroups each, with the copy that sets the lengths: 11.7, 9.8 and 17.9 us)
    const int heads = (c.shape.Hkv + kTickets - 1) / kTickets;
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((c.shape.Hkv + heads - 1) / heads, c.shape.B), dim3(kThreads), 0, st, c, keep, heads); };
    if (c.shape.dtype == AKB_FP16) c.shape.D == 64 ? launch(truncate_kernel<Fp16, 64>) : launch(truncate_kernel<Fp16, 128>);
    else c.shape.D == 64 ? launch(truncate_kernel<Bf16, 64>) : launch(truncate_kernel<Bf16, 128>);
    return hipGetLastError();
}

}  // namespace akb
