// Shared declarations of the block-scaled 8-bit cache (layout and rules: include/akb.h).
#pragma once

#include "../../include/akb.h"
#include "akv_common.h"

namespace akb {

using akv::align256;

constexpr int kTB = AKB_TB;
constexpr int kEMin = -100;        // least exponent of a block's scale
constexpr float kMaxCode = 448.f;  // largest e4m3 number

// host launchers, each defined next to its kernels
hipError_t launch_append(const akb_cache& c, const uint16_t* k_new, const uint16_t* v_new, const int32_t* n_new, int n, hipStream_t st);
hipError_t launch_unpack(const akb_cache& c, uint16_t* k_out, uint16_t* v_out, hipStream_t st);
size_t evict_workspace(const akb_shape& s, int keep);
hipError_t launch_evict(const akb_cache& src, const akb_cache& dst, int keep, int recent, int32_t* kept, char* ws, hipStream_t st);   // kept: or NULL

struct AttentionArgs {
    akb_cache c;
    const uint16_t* q;
    const int32_t* n_q;
    int n;
    void* out;
    int out_dtype;
    int accumulate;
    int max_len;
    float c2;       // scale * log2(e)
    char* ws;
};
size_t attention_workspace(const akb_shape& s, int n, bool accumulate);
size_t attention_tickets();   // bytes at the front of a workspace that are zero between calls
int attention_path(const akb_shape& s, int n, int max_len, int32_t* parts);   // akb_attention_path
int attention_join(const akb_shape& s, int n, int max_len);                    // akb_attention_join
hipError_t launch_attention(const AttentionArgs& a, hipStream_t st);
size_t shared_workspace(const akb_shape& prefix, const akb_shape& s, int n);
int shared_path(const akb_shape& prefix, const akb_shape& s, int n, int max_len, int prefix_max_len, int32_t* parts);   // akb_attention_shared_path
hipError_t launch_shared(const akb_cache& prefix, int prefix_max_len, const AttentionArgs& a, hipStream_t st);
bool append_ticketed(const akb_shape& s, int n);   // the appends' workgroups move the lengths themselves
hipError_t launch_append_lens(const akb_cache& c, const int32_t* n_new, int n, hipStream_t st);   // otherwise: behind them
int rotated_path(const akb_shape& s, int n, bool queries, int32_t* how);   // akb_append_rotated_path
hipError_t launch_append_rotated(const akb_cache& c, const akb_tokens& x, const int32_t* n_new, int n, uint16_t* q_out, const akb_rotary& r, hipStream_t st);
hipError_t launch_fork(const akb_cache& src, const akb_cache& dst, const int32_t* parents, const int32_t* upto, hipStream_t st);
hipError_t launch_truncate(const akb_cache& c, const int32_t* keep, hipStream_t st);

#if defined(__HIPCC__)
using akv::bits_float;
using akv::float_bits;
using akv::u32x2_t;
using akv::u32x4_t;
using akv::f32x4_t;

typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short s16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

// place of token t (0..63) of a block in a channel of V
__host__ __device__ __forceinline__ int v_place(int t) { return ((t >> 2) & 3) * 16 + (t >> 4) * 4 + (t & 3); }
// byte of (token t, channel d) in a block of K
template <int D> __host__ __device__ __forceinline__ int k_place(int t, int d) { return (t >> 4) * (16 * D) + (d >> 6) * 1024 + (t & 15) * 64 + (d & 63); }

__device__ __forceinline__ float pow2(int e) { return bits_float(uint32_t(e + 127) << 23); }   // -126 <= e <= 127

// The two 16-bit types.  cvt2 / cvt8: e4m3 numbers times a power of two, exact (four significant bits, within the type's range).
struct Fp16 {
    using x8 = f16x8_t;
    static constexpr uint32_t kInf = 0x7C00u;
    static constexpr int kTopExp = 8;   // 256 times 2^8 is beyond the type
    static constexpr bool kWide = false;   // numbers as far apart as those of binary32
    __device__ static __forceinline__ float to_float(uint32_t h) { return (float)__builtin_bit_cast(_Float16, (uint16_t)h); }
    template <bool HI> __device__ static __forceinline__ uint32_t cvt2(uint32_t w, float s) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, s, HI)); }
    __device__ static __forceinline__ uint32_t pack(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{a, b}), f16x2_t)); }
    // two numbers over a power of two, to the nearest e4m3 numbers, in the low or the high half of a word
    template <bool HI> __device__ static __forceinline__ uint32_t code2(uint32_t old, uint32_t w, float s) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(__builtin_bit_cast(s16x2_t, old), __builtin_bit_cast(f16x2_t, w), s, HI)); }
    __device__ static __forceinline__ float lo(uint32_t w) { return (float)__builtin_bit_cast(f16x2_t, w).x; }
    __device__ static __forceinline__ float hi(uint32_t w) { return (float)__builtin_bit_cast(f16x2_t, w).y; }
    __device__ static __forceinline__ f32x4_t mfma16(u32x4_t a, u32x4_t b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0); }
    __device__ static __forceinline__ f32x16_t mfma32(u32x4_t a, u32x4_t b, f32x16_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0); }
};
struct Bf16 {
    using x8 = bf16x8_t;
    static constexpr uint32_t kInf = 0x7F80u;
    static constexpr int kTopExp = 120;
    static constexpr bool kWide = true;
    __device__ static __forceinline__ float to_float(uint32_t h) { return bits_float(h << 16); }
    template <bool HI> __device__ static __forceinline__ uint32_t cvt2(uint32_t w, float s) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, HI)); }
    __device__ static __forceinline__ uint32_t pack(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{a, b}), bf16x2_t)); }
    template <bool HI> __device__ static __forceinline__ uint32_t code2(uint32_t old, uint32_t w, float s) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(__builtin_bit_cast(s16x2_t, old), __builtin_bit_cast(bf16x2_t, w), s, HI)); }
    __device__ static __forceinline__ float lo(uint32_t w) { return bits_float(w << 16); }
    __device__ static __forceinline__ float hi(uint32_t w) { return bits_float(w & 0xFFFF0000u); }
    __device__ static __forceinline__ f32x4_t mfma16(u32x4_t a, u32x4_t b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0); }
    __device__ static __forceinline__ f32x16_t mfma32(u32x4_t a, u32x4_t b, f32x16_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0); }
};
// eight e4m3 numbers (two words) times s, as eight 16-bit numbers
template <class T> __device__ __forceinline__ u32x4_t cvt8(uint32_t w0, uint32_t w1, float s)
{
    return u32x4_t{T::template cvt2<false>(w0, s), T::template cvt2<true>(w0, s), T::template cvt2<false>(w1, s), T::template cvt2<true>(w1, s)};
}

// magnitude bits of a 16-bit number for a block's maximum: infinities and NaN do not count
template <class T> __device__ __forceinline__ uint32_t finite_mag(uint32_t h) { const uint32_t m = h & 0x7FFFu; return m < T::kInf ? m : 0u; }
// the least e >= -100 with amax <= 448 2^e = 1.75 2^(e + 8)
__device__ __forceinline__ int scale_exponent(float amax)
{
    const uint32_t u = float_bits(amax);
    return max(int(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0), kEMin);
}
// x 2^-e as the conversion to e4m3 takes it: within +-448 (+-240 where the code above would stand for a number beyond the type), NaN for what is not finite
__device__ __forceinline__ float to_code(float x, float inv, float most)
{
    const float y = x * inv;
    return fabsf(x) < __builtin_inff() ? fminf(fmaxf(y, -most), most) : __builtin_nanf("");
}
template <class T> __device__ __forceinline__ float most_code(int e) { return e == T::kTopExp ? 240.f : kMaxCode; }
__device__ __forceinline__ uint32_t pack_codes(float a, float b, float c, float d)
{
    return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true));
}

// the larger of a value and that of the lane 16 / 32 further (mod the pairs of rows / the halves), in both
__device__ __forceinline__ float max_lane16(float v)
{
    const auto s = __builtin_amdgcn_permlane16_swap(float_bits(v), float_bits(v), false, false);
    return fmaxf(bits_float(s[0]), bits_float(s[1]));
}
__device__ __forceinline__ float max_lane32(float v)
{
    const auto s = __builtin_amdgcn_permlane32_swap(float_bits(v), float_bits(v), false, false);
    return fmaxf(bits_float(s[0]), bits_float(s[1]));
}
// A barrier for data in LDS alone: loads from memory that are in flight stay so (__syncthreads waits for them)
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// tokens of sequence b
__device__ __forceinline__ int seq_len(const akb_cache& c, int b) { return min(max(c.lens[b], 0), c.shape.Ncap); }
#endif

}  // namespace akb
