// A block of 64 tokens x D channels in the registers of a workgroup of 2 D threads: a thread holds the four tokens 16 t + 4 g .. + 3 (a dword of V's
// order) of eight channels, as 16-bit numbers.  What the append and the eviction do with it.
#pragma once

#include "akb_common.h"

namespace akb {

template <int D> struct BlockLane {
    int oct, grp, t0;   // channels 8 oct .. + 7; dword grp of a V channel: tokens t0 .. t0 + 3
    __device__ __forceinline__ BlockLane(int tid) : oct(tid % (D / 8)), grp(tid / (D / 8)), t0((grp & 3) * 16 + (grp >> 2) * 4) {}
};
template <int D> struct PackLds {
    static constexpr int kStride = kTB / 4 + 1;   // of a V channel, padded by a dword
    uint32_t codes[D * kStride];
    uint32_t max[2 * D / 64];
};

template <bool NT, class V> __device__ __forceinline__ void put(V v, uint8_t* p)
{
    if (NT) __builtin_nontemporal_store(v, reinterpret_cast<V*>(p));
    else *reinterpret_cast<V*>(p) = v;
}
// A complete block: maximum over the workgroup, e, codes.  K leaves straight from the registers (8 bytes of a token's 64-channel run), V through LDS,
// so that its 16-byte pieces are stored by neighbouring lanes.  NT: with the non-temporal hint.
template <class T, int D, bool NT>
__device__ __forceinline__ void pack_block(const akb_cache& c, size_t block, bool is_v, const u32x4_t (&x)[4], PackLds<D>& lds)
{
    constexpr int kStride = PackLds<D>::kStride;
    const int tid = threadIdx.x;
    const BlockLane<D> at(tid);
    auto over_workgroup = [&](uint32_t mx) {
        mx = akv::wave_max_int(int(mx));
        if ((tid & 63) == 0) lds.max[tid >> 6] = mx;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 2 * D / 64; ++w) mx = max(mx, lds.max[w]);
        return mx;
    };
    uint32_t two = 0;   // magnitudes of the even and the odd channels
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) two = akv::max_halves(two, x[r][i] & 0x7FFF7FFFu);
    uint32_t mx = over_workgroup(max(two & 0xFFFFu, two >> 16));
    const bool finite = mx < T::kInf;
    if (!finite) {   // infinities and NaN do not count
        mx = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) mx = max(mx, max(finite_mag<T>(x[r][i] & 0xFFFFu), finite_mag<T>(x[r][i] >> 16)));
        __syncthreads();   // lds.max is written again
        mx = over_workgroup(mx);
    }
    const int e = scale_exponent(T::to_float(mx));
    const float scale = pow2(e);
    uint32_t code[8];   // K: two words of each token; V: a word of each channel
    if (finite && e < T::kTopExp) {   // |x| <= 448 2^e: two numbers are one instruction
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (!is_v) {
                    code[2 * r + i] = T::template code2<true>(T::template code2<false>(0, x[r][2 * i], scale), x[r][2 * i + 1], scale);
                } else {
                    const int ch = 2 * r + i;
                    const uint32_t sel = ch & 1 ? 0x07060302u : 0x05040100u;   // this channel of two tokens
                    code[ch] = T::template code2<true>(T::template code2<false>(0, __builtin_amdgcn_perm(x[1][ch >> 1], x[0][ch >> 1], sel), scale),
                                                       __builtin_amdgcn_perm(x[3][ch >> 1], x[2][ch >> 1], sel), scale);
                }
            }
    } else {
        const float inv = pow2(-e), most = most_code<T>(e);
        float y[4][8];
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                y[r][2 * i] = to_code(T::lo(x[r][i]), inv, most);
                y[r][2 * i + 1] = to_code(T::hi(x[r][i]), inv, most);
            }
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                code[2 * r + i] = is_v ? pack_codes(y[0][2 * r + i], y[1][2 * r + i], y[2][2 * r + i], y[3][2 * r + i])
                                       : pack_codes(y[r][4 * i], y[r][4 * i + 1], y[r][4 * i + 2], y[r][4 * i + 3]);
    }
    if (!is_v) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            put<NT>(u32x2_t{code[2 * r], code[2 * r + 1]}, c.k8 + block * (kTB * D) + k_place<D>(at.t0 + r, at.oct * 8));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) lds.codes[(at.oct * 8 + i) * kStride + at.grp] = code[i];
        __syncthreads();
        for (int p = tid; p < D * 4; p += 2 * D) {   // 16-byte pieces
            const uint32_t* s = lds.codes + (p >> 2) * kStride + (p & 3) * 4;
            put<NT>(u32x4_t{s[0], s[1], s[2], s[3]}, c.v8 + block * (kTB * D) + p * 16);
        }
    }
    if (tid == 0) c.exps[block * 2 + (is_v ? 1 : 0)] = (int8_t)e;
}

// Tokens of the incomplete block: those of the thread's four that `store` names
template <int D>
__device__ __forceinline__ void store_tail(const akb_cache& c, size_t bh, bool is_v, const u32x4_t (&x)[4], const bool (&store)[4])
{
    const BlockLane<D> at(threadIdx.x);
    uint16_t* tail = (is_v ? c.v_tail : c.k_tail) + bh * kTB * D;
    if (is_v && store[0] && store[1] && store[2] && store[3]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t sel = e & 1 ? 0x07060302u : 0x05040100u;
            *reinterpret_cast<u32x2_t*>(tail + (at.oct * 8 + e) * kTB + at.grp * 4) =
                u32x2_t{__builtin_amdgcn_perm(x[1][e >> 1], x[0][e >> 1], sel), __builtin_amdgcn_perm(x[3][e >> 1], x[2][e >> 1], sel)};
        }
        return;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (!store[r]) continue;
        if (!is_v) {
            *reinterpret_cast<u32x4_t*>(tail + (at.t0 + r) * D + at.oct * 8) = x[r];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) tail[(at.oct * 8 + e) * kTB + at.grp * 4 + r] = (uint16_t)(x[r][e >> 1] >> (16 * (e & 1)));
        }
    }
}

// ... and those that `want` names, read back into x; RUN: token[r] = t0 + r, a dword pair of V's order
template <int D, bool RUN>
__device__ __forceinline__ void load_tail(const akb_cache& c, size_t bh, bool is_v, u32x4_t (&x)[4], const bool (&want)[4], const int (&token)[4])
{
    const BlockLane<D> at(threadIdx.x);
    const uint16_t* tail = (is_v ? c.v_tail : c.k_tail) + bh * kTB * D;
    if (RUN && is_v) {
        u32x2_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = *reinterpret_cast<const u32x2_t*>(tail + (at.oct * 8 + e) * kTB + at.grp * 4);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i)   // half r % 2 of dword r / 2 of channels 2 i, 2 i + 1
                if (want[r]) x[r][i] = __builtin_amdgcn_perm(w[2 * i + 1][r >> 1], w[2 * i][r >> 1], r & 1 ? 0x07060302u : 0x05040100u);
        return;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (!want[r]) continue;
        if (!is_v) {
            x[r] = *reinterpret_cast<const u32x4_t*>(tail + token[r] * D + at.oct * 8);
        } else {
            const uint16_t* p = tail + at.oct * 8 * kTB + v_place(token[r]);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[r][i] = p[2 * i * kTB] | uint32_t(p[(2 * i + 1) * kTB]) << 16;
        }
    }
}

}  // namespace akb
