// The block-scaled 8-bit cache: sequences copied to others and cut back in place (rules and layout: include/akb.h).
#include "akb_common.h"

namespace akb {

constexpr int kThreads = 256;

// Block `block` of c as the 16-bit tail `bh` of d holds it: 16 codes become 32 bytes per thread and turn, in the orders that both already have (K: a token's run of
// channels; V: a channel's tokens).
template <class T, int D> __device__ __forceinline__ void block_to_tail(const akb_cache& c, size_t block, const akb_cache& d, size_t bh, int tid)
{
    const float ks = pow2(c.exps[block * 2]), vs = pow2(c.exps[block * 2 + 1]);
    for (int p = tid; p < D * 4; p += kThreads) {
        const u32x4_t k = *reinterpret_cast<const u32x4_t*>(c.k8 + block * (kTB * D) + p * 16), v = *reinterpret_cast<const u32x4_t*>(c.v8 + block * (kTB * D) + p * 16);
        const int run = p >> 2, token = run / (16 * (D / 64)) * 16 + run % 16, i = run / 16 % (D / 64);   // k8: [4][D / 64][16] runs of 64 channels
        u32x4_t* kt = reinterpret_cast<u32x4_t*>(d.k_tail + bh * kTB * D + token * D + i * 64 + (p & 3) * 16);
        u32x4_t* vt = reinterpret_cast<u32x4_t*>(d.v_tail + bh * kTB * D + p * 16);
        kt[0] = cvt8<T>(k[0], k[1], ks);
        kt[1] = cvt8<T>(k[2], k[3], ks);
        vt[0] = cvt8<T>(v[0], v[1], vs);
        vt[1] = cvt8<T>(v[2], v[3], vs);
    }
}

// One workgroup per (chunk of blocks, KV head, sequence of the destination).  The complete blocks of a (sequence, KV head) lie one behind the other, so a chunk is two runs of bytes.
constexpr int kChunk = 4;   // blocks
template <class T, int D>
__global__ __launch_bounds__(kThreads) void fork_kernel(akb_cache c, akb_cache d, const int32_t* __restrict__ parents, const int32_t* __restrict__ upto)
{
    const int tid = threadIdx.x, h = blockIdx.y, j = blockIdx.z, chunk = blockIdx.x;
    const int a = parents ? parents[j] : j;
    if (a < 0 || a >= c.shape.B) return;
    const int had = seq_len(c, a), len = upto ? min(had, max(upto[j], 0)) : had;
    if (len > d.shape.Ncap) {
        if (chunk == 0 && h == 0 && tid == 0) atomicAdd(&d.flags[AKV_FLAG_OVERFLOW], 1);
        return;
    }
    const size_t from = size_t(a) * c.shape.Hkv + h, to = size_t(j) * d.shape.Hkv + h, from0 = from * (c.shape.Ncap / kTB), to0 = to * (d.shape.Ncap / kTB);
    const int whole = len / kTB, first = chunk * kChunk, n = min(kChunk, whole - first);
    if (chunk == 0 && h == 0 && tid == 0) d.lens[j] = len;
    if (n > 0) {
        const u32x4_t *k = reinterpret_cast<const u32x4_t*>(c.k8 + (from0 + first) * (kTB * D)), *v = reinterpret_cast<const u32x4_t*>(c.v8 + (from0 + first) * (kTB * D));
        u32x4_t *ko = reinterpret_cast<u32x4_t*>(d.k8 + (to0 + first) * (kTB * D)), *vo = reinterpret_cast<u32x4_t*>(d.v8 + (to0 + first) * (kTB * D));
        for (int i = tid; i < n * (kTB * D / 16); i += kThreads) {
            ko[i] = k[i];
            vo[i] = v[i];
        }
        if (tid < 2 * n) d.exps[(to0 + first) * 2 + tid] = c.exps[(from0 + first) * 2 + tid];
    }
    if (c.score && d.score)
        for (int t = first * kTB + tid; t < min(len, (first + kChunk) * kTB); t += kThreads) d.score[to * d.shape.Ncap + t] = c.score[from * c.shape.Ncap + t];
    if (len % kTB && whole >= first && whole < first + kChunk) {   // the incomplete block
        if (whole < had / kTB) {
            block_to_tail<T, D>(c, from0 + whole, d, to, tid);
        } else {
            const u32x4_t *k = reinterpret_cast<const u32x4_t*>(c.k_tail + from * kTB * D), *v = reinterpret_cast<const u32x4_t*>(c.v_tail + from * kTB * D);
            u32x4_t *ko = reinterpret_cast<u32x4_t*>(d.k_tail + to * kTB * D), *vo = reinterpret_cast<u32x4_t*>(d.v_tail + to * kTB * D);
            for (int i = tid; i < kTB * D / 8; i += kThreads) {
                ko[i] = k[i];
                vo[i] = v[i];
            }
        }
    }
}

hipError_t launch_fork(const akb_cache& src, const akb_cache& dst, const int32_t* parents, const int32_t* upto, hipStream_t st)
{
    // (a copy that ends with the source's capacity has no incomplete block; one that the destination has no room for is refused by the first workgroups)
    const int blocks = std::min(src.shape.Ncap, dst.shape.Ncap) / kTB;
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((blocks + kChunk - 1) / kChunk, dst.shape.Hkv, dst.shape.B), dim3(kThreads), 0, st, src, dst, parents, upto); };
    if (src.shape.dtype == AKB_FP16) src.shape.D == 64 ? launch(fork_kernel<Fp16, 64>) : launch(fork_kernel<Fp16, 128>);
    else src.shape.D == 64 ? launch(fork_kernel<Bf16, 64>) : launch(fork_kernel<Bf16, 128>);
    return hipGetLastError();
}

// One workgroup per (KV head, sequence).  A sequence that stays inside its incomplete block, or ends with a block, only gets its length; which of its workgroups reads
// the old length and which the new makes no difference then.  Where a block goes to the tail, all have to have read the old one: the last by ticket moves it.
template <class T, int D>
__global__ __launch_bounds__(kThreads) void truncate_kernel(akb_cache c, const int32_t* __restrict__ keep)
{
    const int tid = threadIdx.x, h = blockIdx.x, b = blockIdx.y;
    const int had = seq_len(c, b), len = min(had, max(keep[b], 0)), blk = len / kTB;
    if (len % kTB == 0 || blk == had / kTB) {
        if (h == 0 && tid == 0) c.lens[b] = len;
        return;
    }
    __syncthreads();   // (the length has been read by all waves)
    if (tid == 0 && atomicAdd(&c.flags[AKV_NFLAGS + b], 1) == int(gridDim.x) - 1) {
        c.flags[AKV_NFLAGS + b] = 0;
        c.lens[b] = len;
    }
    const size_t bh = size_t(b) * c.shape.Hkv + h;
    block_to_tail<T, D>(c, bh * (c.shape.Ncap / kTB) + blk, c, bh, tid);
}

hipError_t launch_truncate(const akb_cache& c, const int32_t* keep, hipStream_t st)
{
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(c.shape.Hkv, c.shape.B), dim3(kThreads), 0, st, c, keep); };
    if (c.shape.dtype == AKB_FP16) c.shape.D == 64 ? launch(truncate_kernel<Fp16, 64>) : launch(truncate_kernel<Fp16, 128>);
    else c.shape.D == 64 ? launch(truncate_kernel<Bf16, 64>) : launch(truncate_kernel<Bf16, 128>);
    return hipGetLastError();
}

}  // namespace akb
