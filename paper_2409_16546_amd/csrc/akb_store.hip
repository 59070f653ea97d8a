// The block-scaled 8-bit cache: tokens stored, and given back as 16-bit values (rules and layout: include/akb.h).
#include "akb_pack.h"

namespace akb {

// One workgroup of 2 D threads per (block that the call touches, KV head, sequence), for both sides; the lanes of a wave read whole rows.
//   A complete block takes the tokens that the tail held and new ones.
//   The incomplete last block goes to the tail, by the workgroups of the first block alone: they are the ones that read the tail.
// Who moves the length: with few workgroups the last of the sequence by ticket (every one has read the old length by then), as in the
// append of the 16-bit cache; otherwise a launch behind this one.
template <class T, int D, bool NT>
__global__ __launch_bounds__(2 * D) void append_kernel(akb_cache c, const uint16_t* __restrict__ k_new, const uint16_t* __restrict__ v_new,
                                                       const int32_t* __restrict__ n_new, int n, int ticketed)
{
    __shared__ PackLds<D> lds;
    const int tid = threadIdx.x, h = blockIdx.y, b = blockIdx.z;
    const int j = blockIdx.x;
    const int Hkv = c.shape.Hkv, Ncap = c.shape.Ncap;
    const int len = akb::seq_len(c, b);
    const int cnt = n_new ? min(max(n_new[b], 0), n) : n;
    if (cnt == 0) return;
    if (len + cnt > Ncap) {   // the sequence is left unchanged
        if (ticketed && blockIdx.x == 0 && h == 0 && tid == 0) atomicAdd(&c.flags[AKV_FLAG_OVERFLOW], 1);
        return;
    }
    int ticket = -1;
    if (ticketed) {   // drawn once all waves of the workgroup have read the length, looked at when it leaves
        __syncthreads();
        if (tid == 0) ticket = atomicAdd(&c.flags[AKV_NFLAGS + b], 1);
    }
    const size_t bh = size_t(b) * Hkv + h;
    const int first = len / kTB, had = len % kTB, total = had + cnt;   // counted from the start of block `first`
    const BlockLane<D> at(tid);
    const int t0 = at.t0;
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const bool is_v = side == 1;
        const uint16_t* fresh = (is_v ? v_new : k_new) + bh * n * D;
        auto load_fresh = [&](int w) -> u32x4_t {             // token w counted from the start of block `first`
            if (w < had || w >= total) return u32x4_t{0, 0, 0, 0};
            const u32x4_t* p = reinterpret_cast<const u32x4_t*>(fresh + size_t(w - had) * D + at.oct * 8);
            return NT ? __builtin_nontemporal_load(p) : *p;
        };
        if ((j + 1) * kTB <= total) {
            u32x4_t x[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = load_fresh(j * kTB + t0 + r);
            if (j == 0 && had > 0) {
                const bool old[4] = {t0 < had, t0 + 1 < had, t0 + 2 < had, t0 + 3 < had};
                const int token[4] = {t0, t0 + 1, t0 + 2, t0 + 3};
                load_tail<D, true>(c, bh, is_v, x, old, token);
            }
            if (is_v) __syncthreads();   // K's block has been packed
            pack_block<T, D, NT>(c, bh * (Ncap / kTB) + first + j, is_v, x, lds);
        }
        if (j == 0 && total % kTB) {   // the incomplete block: its new tokens go to the tail (what of the old ones is needed has been read)
            __syncthreads();
            const int last = total / kTB * kTB;
            u32x4_t x[4];
            bool store[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[r] = load_fresh(last + t0 + r);
                store[r] = last + t0 + r >= had && last + t0 + r < total;
            }
            store_tail<D>(c, bh, is_v, x, store);
        }
    }
    if (c.score && tid < kTB) {   // the new tokens' scores
        const int w = j * kTB + tid;
        if (w >= had && w < total) c.score[bh * Ncap + first * kTB + w] = 0.f;
    }
    if (ticket == int(gridDim.x) * Hkv - 1) {   // the last workgroup of the sequence (thread 0 of it)
        c.flags[AKV_NFLAGS + b] = 0;
        c.lens[b] = len + cnt;
    }
}

// behind the append: the lengths move, refusals are counted
__global__ __launch_bounds__(256) void append_lens_kernel(akb_cache c, const int32_t* __restrict__ n_new, int n)
{
    for (int b = threadIdx.x; b < c.shape.B; b += 256) {
        const int len = seq_len(c, b), cnt = n_new ? min(max(n_new[b], 0), n) : n;
        if (len + cnt <= c.shape.Ncap) c.lens[b] = len + cnt;
        else atomicAdd(&c.flags[AKV_FLAG_OVERFLOW], 1);
    }
}

// Who moves the lengths of an append of n tokens: the workgroups' tickets, or a launch behind.
// A ticket per workgroup or a launch behind, us of calls one after the other.  One block per head, where the workgroups arrive as they were launched: 512 workgroups of 64
// sequences 6.0 / 8.3 and of 16 sequences 7.9 / 8.3, 640 of 80 and of 20 sequences 6.2 / 8.2 and 8.3 / 8.3, 768 of 96 and of 24 6.3 / 8.3 and 10.2 / 8.3, 1024 7.1 / 8.1
// and 11.8 / 8.1.  Several blocks: 96 workgroups 8.2 / 10.3, 192 9.4 / 10.4, 272 11.0 / 11.6, 288 11.7 / 11.6, 384 10.8 / 10.3 and 13.1 / 11.6, 576 15.7 / 11.7.  (Of one side
// per workgroup they would be twice as many, and gain nothing: 8 x 8 pairs 8192 tokens 77 us.)
bool append_ticketed(const akb_shape& s, int n)
{
    const int blocks = (kTB - 1 + n + kTB - 1) / kTB;
    return long(blocks) * s.Hkv * s.B <= (blocks == 1 ? 640 : 288);
}
hipError_t launch_append_lens(const akb_cache& c, const int32_t* n_new, int n, hipStream_t st)
{
    hipLaunchKernelGGL(append_lens_kernel, dim3(1), dim3(256), 0, st, c, n_new, n);
    return hipGetLastError();
}

hipError_t launch_append(const akb_cache& c, const uint16_t* k_new, const uint16_t* v_new, const int32_t* n_new, int n, hipStream_t st)
{
    if (n == 0) return hipSuccess;
    const int blocks = (kTB - 1 + n + kTB - 1) / kTB;
    const dim3 grid(blocks, c.shape.Hkv, c.shape.B);
    const bool ticketed = append_ticketed(c.shape, n);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(2 * c.shape.D), 0, st, c, k_new, v_new, n_new, n, ticketed ? 1 : 0); };
    // New tokens that are more than half of the last-level cache are read and their codes stored with the non-temporal hint; fewer may still lie there as they were
    // made, and their codes are wanted there next.  Plain / with the hint: 8 x 8 pairs 8192 tokens (268 MB) 76.7 / 68.8 us, 6 x 32 pairs up to 777 tokens (76 MB at most, read again and again) 28.9 / 33.8.
    const bool streamed = size_t(c.shape.B) * c.shape.Hkv * n * c.shape.D * 4 > (size_t(128) << 20);
    auto pick = [&](auto plain, auto hinted) { streamed ? launch(hinted) : launch(plain); };
    if (c.shape.dtype == AKB_FP16) c.shape.D == 64 ? pick(append_kernel<Fp16, 64, false>, append_kernel<Fp16, 64, true>) : pick(append_kernel<Fp16, 128, false>, append_kernel<Fp16, 128, true>);
    else c.shape.D == 64 ? pick(append_kernel<Bf16, 64, false>, append_kernel<Bf16, 64, true>) : pick(append_kernel<Bf16, 128, false>, append_kernel<Bf16, 128, true>);
    if (hipError_t e = hipGetLastError()) return e;
    return ticketed ? hipSuccess : launch_append_lens(c, n_new, n, st);
}

// The append of a block backwards: one workgroup of 2 D threads per (block, side, KV head, sequence).
template <class T, int D>
__global__ __launch_bounds__(2 * D) void unpack_kernel(akb_cache c, uint16_t* __restrict__ k_out, uint16_t* __restrict__ v_out)
{
    constexpr int kOct = D / 8, kStride = kTB / 4 + 1;
    __shared__ uint32_t codes_s[D * kStride];
    const int tid = threadIdx.x, NB = c.shape.Ncap / kTB, blk = blockIdx.x >> 1;
    const bool is_v = blockIdx.x & 1;
    const size_t bh = size_t(blockIdx.z) * c.shape.Hkv + blockIdx.y, block = bh * NB + blk;
    uint16_t* out = is_v ? v_out : k_out;
    if (!out) return;
    const int len = seq_len(c, blockIdx.z);
    const int oct = tid % kOct, grp = tid / kOct, t0 = (grp & 3) * 16 + (grp >> 2) * 4;
    u32x4_t x[4] = {};
    if (blk < len / kTB) {
        const float s = pow2(c.exps[block * 2 + (is_v ? 1 : 0)]);
        if (!is_v) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const u32x2_t w = *reinterpret_cast<const u32x2_t*>(c.k8 + block * (kTB * D) + k_place<D>(t0 + r, oct * 8));
                x[r] = cvt8<T>(w[0], w[1], s);
            }
        } else {
            for (int p = tid; p < D * 4; p += 2 * D) {
                const u32x4_t w = *reinterpret_cast<const u32x4_t*>(c.v8 + block * (kTB * D) + p * 16);
                uint32_t* d = codes_s + (p >> 2) * kStride + (p & 3) * 4;
#pragma unroll
                for (int i = 0; i < 4; ++i) d[i] = w[i];
            }
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t w = codes_s[(oct * 8 + e) * kStride + grp];   // tokens t0 .. t0 + 3 of channel 8 oct + e
                const uint32_t a = T::template cvt2<false>(w, s), d = T::template cvt2<true>(w, s), sh = 16 * (e & 1);
                x[0][e >> 1] |= (a & 0xFFFFu) << sh;
                x[1][e >> 1] |= (a >> 16) << sh;
                x[2][e >> 1] |= (d & 0xFFFFu) << sh;
                x[3][e >> 1] |= (d >> 16) << sh;
            }
        }
    } else if (blk == len / kTB && len % kTB) {
        const uint16_t* tail = (is_v ? c.v_tail : c.k_tail) + bh * kTB * D;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (t0 + r >= len % kTB) continue;
            if (!is_v) {
                x[r] = *reinterpret_cast<const u32x4_t*>(tail + (t0 + r) * D + oct * 8);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[r][e >> 1] |= uint32_t(tail[(oct * 8 + e) * kTB + grp * 4 + r]) << (16 * (e & 1));
            }
        }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) *reinterpret_cast<u32x4_t*>(out + (block * kTB + t0 + r) * D + oct * 8) = x[r];
}

hipError_t launch_unpack(const akb_cache& c, uint16_t* k_out, uint16_t* v_out, hipStream_t st)
{
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(2 * (c.shape.Ncap / kTB), c.shape.Hkv, c.shape.B), dim3(2 * c.shape.D), 0, st, c, k_out, v_out); };
    if (c.shape.dtype == AKB_FP16) c.shape.D == 64 ? launch(unpack_kernel<Fp16, 64>) : launch(unpack_kernel<Fp16, 128>);
    else c.shape.D == 64 ? launch(unpack_kernel<Bf16, 64>) : launch(unpack_kernel<Bf16, 128>);
    return hipGetLastError();
}

}  // namespace akb
