// Eviction from the block-scaled 8-bit cache by accumulated attention weight (rules and layout: include/akb.h).
#include "akb_common.h"

namespace akb {

constexpr int kSelThreads = 1024;
constexpr int kBins = 2048;

// order of binary32 numbers as unsigned integers; zeros of either sign are equal, a NaN is the largest
__device__ __forceinline__ uint32_t order_key(float f)
{
    if (f != f) return 0xFFFFFFFFu;
    const uint32_t u = float_bits(f + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// inclusive prefix sum over the workgroup (every thread calls it); total in *sum
__device__ __forceinline__ int block_scan(int v, int* wave_s, int* sum)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int x = akv::wave_scan_add(v);
    __syncthreads();   // wave_s may still be read from the call before
    if (lane == 63) wave_s[wave] = x;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < kSelThreads / 64; ++w) {
        const int t = wave_s[w];
        before += w < wave ? t : 0;
        all += t;
    }
    *sum = all;
    return x + before;
}

// Which tokens of a (sequence, KV head) stay: one workgroup each.  The place among the sorted scores is found 11, 11 and 10 bits at a
// time (counts of each value of the bits among the scores that agree in the bits above), then one pass writes the kept tokens' places in
// their order: those above the threshold, of those at it the first.
__global__ __launch_bounds__(kSelThreads) void select_kernel(akb_cache c, akb_cache d, int keep, int recent, int32_t* __restrict__ kept)
{
    __shared__ int hist[kBins];
    __shared__ int wave_s[kSelThreads / 64];
    __shared__ int found_s[2];
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const size_t bh = size_t(b) * c.shape.Hkv + h;
    const int len = seq_len(c, b), count = min(len, keep), sure = min(recent, count);
    const int pool = len - sure;          // tokens to choose from
    int need = count - sure;              // of which this many stay
    const float* score = c.score + bh * c.shape.Ncap;
    uint32_t prefix = 0;
    if (need < pool && need > 0) {
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bits = pass == 2 ? 10 : 11;
            for (int i = tid; i < kBins; i += kSelThreads) hist[i] = 0;
            __syncthreads();
            for (int t = tid; t < pool; t += kSelThreads) {
                const uint32_t k = order_key(score[t]);
                if (pass == 0 || (k >> (shift + bits)) == prefix) atomicAdd(&hist[(k >> shift) & ((1u << bits) - 1)], 1);
            }
            __syncthreads();
            // from the largest value down: thread i has values 2 i, 2 i + 1 counted from the top
            const int top = kBins - 1 - 2 * tid, h0 = hist[top], h1 = hist[top - 1];
            int all;
            const int upto = block_scan(h0 + h1, wave_s, &all), before = upto - h0 - h1;
            if (before < need && need <= upto) {
                const bool first = need <= before + h0;
                found_s[0] = first ? top : top - 1;
                found_s[1] = first ? before : before + h0;
            }
            __syncthreads();
            prefix = (prefix << bits) | uint32_t(found_s[0]);
            need -= found_s[1];
            __syncthreads();
        }
    }
    const bool all_stay = count - sure >= pool, none = count - sure <= 0;
    int32_t* out = kept + bh * keep;
    int done = 0, ties = 0;               // written; tokens at the threshold passed
    if (all_stay) {
        for (int t = tid; t < count; t += kSelThreads) out[t] = t;
    } else {
        if (!none)
            for (int base = 0; base < pool; base += kSelThreads) {
                const int t = base + tid;
                const uint32_t k = t < pool ? order_key(score[t]) : 0u;
                const int tie = t < pool && k == prefix ? 1 : 0;
                int all_ties, all_keep;
                const int rank = block_scan(tie, wave_s, &all_ties);
                const int stays = t < pool && (k > prefix || (tie && ties + rank <= need)) ? 1 : 0;
                const int at = block_scan(stays, wave_s, &all_keep);
                if (stays) out[done + at - 1] = t;
                done += all_keep;
                ties += all_ties;
            }
        for (int i = tid; i < sure; i += kSelThreads) out[count - sure + i] = len - sure + i;
    }
    for (int i = count + tid; i < keep; i += kSelThreads) out[i] = -1;
    if (h == 0 && tid == 0) d.lens[b] = count;
}

// one stored value of channel ch of token t, exact
template <class T, int D> __device__ __forceinline__ float stored(const akb_cache& c, size_t bh, int len, int t, int ch, bool is_v)
{
    const int blk = t / kTB, s = t % kTB;
    if (blk < len / kTB) {
        const size_t block = bh * (c.shape.Ncap / kTB) + blk;
        const uint32_t code = is_v ? c.v8[block * (kTB * D) + ch * kTB + v_place(s)] : c.k8[block * (kTB * D) + k_place<D>(s, ch)];
        return T::lo(T::template cvt2<false>(code, pow2(c.exps[block * 2 + (is_v ? 1 : 0)])));
    }
    return T::to_float(is_v ? c.v_tail[(bh * D + ch) * kTB + v_place(s)] : c.k_tail[(bh * kTB + s) * D + ch]);
}

// A block of the destination: one workgroup of 2 D threads per (block, side, KV head, sequence); a thread has the four tokens of a
// dword of V's order in eight channels, as in the append.
template <class T, int D>
__global__ __launch_bounds__(2 * D) void gather_kernel(akb_cache c, akb_cache d, int keep, const int32_t* __restrict__ kept)
{
    constexpr int kOct = D / 8, kWaves = 2 * D / 64;
    __shared__ uint32_t max_s[kWaves];
    __shared__ int from_s[kTB];
    const int tid = threadIdx.x, h = blockIdx.y, b = blockIdx.z, blk = blockIdx.x >> 1;
    const bool is_v = blockIdx.x & 1;
    const size_t bh = size_t(b) * c.shape.Hkv + h;
    const int len = seq_len(c, b), count = min(len, keep);
    if (blk * kTB >= count) return;
    if (tid < kTB) {
        const int i = blk * kTB + tid, t = i < count ? kept[bh * keep + i] : -1;
        from_s[tid] = t;
        if (!is_v && d.score && t >= 0) d.score[bh * d.shape.Ncap + i] = c.score[bh * c.shape.Ncap + t];
    }
    __syncthreads();
    const int oct = tid % kOct, grp = tid / kOct, t0 = (grp & 3) * 16 + (grp >> 2) * 4;
    float x[4][8];
    float mx = 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int t = from_s[t0 + r];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[r][e] = t >= 0 ? stored<T, D>(c, bh, len, t, oct * 8 + e, is_v) : 0.f;
            const float a = fabsf(x[r][e]);
            if (a < __builtin_inff()) mx = fmaxf(mx, a);
        }
    }
    if ((blk + 1) * kTB <= count) {
        mx = akv::wave_max(mx);
        if ((tid & 63) == 0) max_s[tid >> 6] = float_bits(mx);
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) mx = fmaxf(mx, bits_float(max_s[w]));
        const int e = scale_exponent(mx);
        const float inv = pow2(-e), most = most_code<T>(e);
        const size_t block = bh * (d.shape.Ncap / kTB) + blk;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < 8; ++i) x[r][i] = to_code<T>(x[r][i], inv, most);
        if (!is_v) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                *reinterpret_cast<u32x2_t*>(d.k8 + block * (kTB * D) + k_place<D>(t0 + r, oct * 8)) =
                    u32x2_t{pack_codes(x[r][0], x[r][1], x[r][2], x[r][3]), pack_codes(x[r][4], x[r][5], x[r][6], x[r][7])};
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) *reinterpret_cast<uint32_t*>(d.v8 + block * (kTB * D) + (oct * 8 + i) * kTB + grp * 4) = pack_codes(x[0][i], x[1][i], x[2][i], x[3][i]);
        }
        if (tid == 0) d.exps[block * 2 + (is_v ? 1 : 0)] = (int8_t)e;
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (from_s[t0 + r] < 0) continue;
            if (!is_v) {
                *reinterpret_cast<u32x4_t*>(d.k_tail + (bh * kTB + t0 + r) * D + oct * 8) =
                    u32x4_t{T::pack(x[r][0], x[r][1]), T::pack(x[r][2], x[r][3]), T::pack(x[r][4], x[r][5]), T::pack(x[r][6], x[r][7])};
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) d.v_tail[(bh * D + oct * 8 + i) * kTB + grp * 4 + r] = (uint16_t)T::from_float(x[r][i]);
            }
        }
    }
}

hipError_t launch_evict(const akb_cache& src, const akb_cache& dst, int keep, int recent, int32_t* kept, hipStream_t st)
{
    const akb_shape& s = src.shape;
    hipLaunchKernelGGL(select_kernel, dim3(s.Hkv, s.B), dim3(kSelThreads), 0, st, src, dst, keep, recent, kept);
    if (hipError_t e = hipGetLastError()) return e;
    const int blocks = (std::min(keep, s.Ncap) + kTB - 1) / kTB;
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(2 * blocks, s.Hkv, s.B), dim3(2 * s.D), 0, st, src, dst, keep, kept); };
    if (s.dtype == AKB_FP16) s.D == 64 ? launch(gather_kernel<Fp16, 64>) : launch(gather_kernel<Fp16, 128>);
    else s.D == 64 ? launch(gather_kernel<Bf16, 64>) : launch(gather_kernel<Bf16, 128>);
    return hipGetLastError();
}

}  // namespace akb
