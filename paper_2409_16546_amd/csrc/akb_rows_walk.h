// The walk of few query rows over blocks of the block-scaled 8-bit cache: what a wave holds of its rows, how codes go to the matrix units.
#pragma once

#include "akb_rows.h"

namespace akb {

constexpr int kTileRows = 16;

// A block of K or V as the matrix instructions take it: lane (token t % 16 or channel % 16, quarter): 16 codes
// NT: with the non-temporal hint
template <bool NT> __device__ __forceinline__ u32x4_t load_codes(const uint8_t* p)
{
    const u32x4_t* w = reinterpret_cast<const u32x4_t*>(p);
    return NT ? __builtin_nontemporal_load(w) : *w;
}
template <int D, bool NT> struct KCodes {
    u32x4_t w[4][D / 64];
    uint32_t e;   // exponents of the block's K and of its V (the scales are made where they are used: made here, the load would be waited for here)
    __device__ __forceinline__ void load(const akb_cache& c, size_t block, int lane)
    {
        const uint8_t* p = c.k8 + block * (kTB * D) + (lane & 15) * 64 + (lane >> 4) * 16;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < D / 64; ++i) w[t][i] = load_codes<NT>(p + t * (16 * D) + i * 1024);
        e = *reinterpret_cast<const uint16_t*>(c.exps + block * 2);
    }
};
template <int D, bool NT> struct VCodes {
    u32x4_t w[D / 16];
    __device__ __forceinline__ void load(const akb_cache& c, size_t block, int lane)
    {
        const uint8_t* p = c.v8 + block * (kTB * D) + (lane & 15) * 64 + (lane >> 4) * 16;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) w[i] = load_codes<NT>(p + i * 1024);
    }
};

// A query row as the operand of S^T: step k of 32 channels, lane group g: channels 64 (k / 2) + 16 g + 8 (k % 2) .. + 7 (the order in which K's codes come)
template <int D> __device__ __forceinline__ void load_query(u32x4_t (&q)[D / 32], const uint16_t* row, int lane)
{
#pragma unroll
    for (int k = 0; k < D / 32; ++k) q[k] = row ? *reinterpret_cast<const u32x4_t*>(row + 64 * (k >> 1) + 16 * (lane >> 4) + 8 * (k & 1)) : u32x4_t{0, 0, 0, 0};
}

// Running state of a row tile in one wave: lane (row l % 16, g): channels 16 i + 4 g .. + 3 of O, the row's maximum, its share of the sum
template <class T, int D> struct RowState {
    u32x4_t q[D / 32];
    f32x4_t o[D / 16];
    float m, z;
    int limit;
    __device__ __forceinline__ void init(const uint16_t* qrow, int lim, int lane)
    {
        load_query<D>(q, qrow, lane);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[i] = f32x4_t{0, 0, 0, 0};
        m = -__builtin_inff();
        z = 0.f;
        limit = lim;
    }
    // S^T of 64 tokens -> weights (unit: the bits of the largest); ph[u]: tokens 32 u .. + 31 as the operand of the second product, pl: what 16 bits lack of them, pr: what
    // those lack (bfloat16)
    template <bool EXACT> __device__ __forceinline__ void weights(f32x4_t (&s)[4], int first, bool masked, float c2, float unit, int lane, u32x4_t (&ph)[2], u32x4_t (&pl)[2], u32x4_t (&pr)[2])
    {
        float mx = -__builtin_inff();
        const int seen = limit - first - 4 * (lane >> 4);   // counted from the lane's first token
        if (masked) {
            asm volatile("");   // (a branch: without it all blocks are asked, 50 instructions of some 180; few are masked where the caller knows what every row sees)
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (16 * t + r >= seen) s[t][r] = -__builtin_inff();
        }
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[t][r]);
        mx = max_lane32(max_lane16(mx));
        const float now = fmaf(mx, c2, -unit);
        if (__any(now > m + kSlackBits)) {
            const float up = fmaxf(m, now), a = __builtin_amdgcn_exp2f(m - (up == -__builtin_inff() ? 0.f : up));
            z *= a;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) o[i] *= a;
            m = up;
        }
        const float base = m == -__builtin_inff() ? 0.f : m;   // nothing seen yet: all weights are 2^-inf
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[t][r] = __builtin_amdgcn_exp2f(fmaf(s[t][r], c2, -base));
                sum += s[t][r];
            }
        z += sum;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float p0 = s[2 * u + (k >> 1)][2 * (k & 1)], p1 = s[2 * u + (k >> 1)][2 * (k & 1) + 1];
                ph[u][k] = T::pack(p0, p1);
                if (!EXACT) continue;
                const float l0 = p0 - T::lo(ph[u][k]), l1 = p1 - T::hi(ph[u][k]);
                pl[u][k] = T::pack(l0, l1);
                if (T::kWide) pr[u][k] = T::pack(l0 - T::lo(pl[u][k]), l1 - T::hi(pl[u][k]));
            }
    }
};

// q . k of 64 tokens for the score, [tile of 16 tokens][row][16]: a store covers whole lines; lane (row, g) has four runs of four tokens.  (Without the hint: the score
// kernel finds them in the last-level cache, which the codes of large calls pass by.  4 x 8 pairs of up to 131072 tokens 161 / 151 us.)
__device__ __forceinline__ void store_logits(float* block, const f32x4_t (&s)[4], int rows, int row, int lane)
{
    if (row >= rows) return;
#pragma unroll
    for (int t = 0; t < 4; ++t) *reinterpret_cast<f32x4_t*>(block + (t * rows + row) * 16 + 4 * (lane >> 4)) = s[t];
}

// Blocks lo + at, lo + at + STEP, .. below hi of (sequence, KV head) bh, which has len tokens, for RT tiles of 16 rows, `all_see` tokens of which every row sees.
// logits: where the products are left for the score (one tile of `rows` rows), or NULL.
template <class T, int D, bool EXACT, int RT, bool NT, int STEP>
__device__ __forceinline__ void walk_rows(const akb_cache& c, size_t bh, RowState<T, D> (&st)[RT], int lo, int hi, int len, int all_see, float c2, int lane, int at, float* logits,
                                          int rows)
{
    const int whole = min(hi, len / kTB);   // blocks in 8 bits
    const size_t block0 = bh * (c.shape.Ncap / kTB);
    int blk = lo + at;
    KCodes<D, NT> kc;
    if (blk < whole) kc.load(c, block0 + blk, lane);
    for (; blk < whole; blk += STEP) {
        VCodes<D, NT> vc;
        vc.load(c, block0 + blk, lane);
        uint32_t e = kc.e;
        asm volatile("" : "+v"(e));   // (known to be the same in all lanes, it would be moved to a scalar register where it is asked for, and the codes that are asked for before it waited for there)
        const float k_scale = pow2(int8_t(e)), v_scale = pow2(int8_t(e >> 8)), unit = weight_bits<T>(v_scale >= pow2(kLargeExp));
        f32x4_t s[RT][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int k = 0; k < RT; ++k) s[k][t] = f32x4_t{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                const u32x4_t x = cvt8<T>(kc.w[t][i >> 1][2 * (i & 1)], kc.w[t][i >> 1][2 * (i & 1) + 1], k_scale);
#pragma unroll
                for (int k = 0; k < RT; ++k) s[k][t] = T::mfma16(x, st[k].q[i], s[k][t]);
            }
        }
        if (blk + STEP < whole) kc.load(c, block0 + blk + STEP, lane);
        if (RT == 1 && logits) store_logits(logits + size_t(blk) * kTB * rows, s[0], rows, lane & 15, lane);
        const bool masked = (blk + 1) * kTB > all_see;
        u32x4_t ph[RT][2], pl[RT][2], pr[RT][2];
#pragma unroll
        for (int k = 0; k < RT; ++k) st[k].template weights<EXACT>(s[k], blk * kTB, masked, c2, unit, lane, ph[k], pl[k], pr[k]);
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const u32x4_t v = cvt8<T>(vc.w[i][2 * u], vc.w[i][2 * u + 1], v_scale);
#pragma unroll
                for (int k = 0; k < RT; ++k) {
                    st[k].o[i] = T::mfma16(v, ph[k][u], st[k].o[i]);
                    if (EXACT) st[k].o[i] = T::mfma16(v, pl[k][u], st[k].o[i]);
                    if (EXACT && T::kWide) st[k].o[i] = T::mfma16(v, pr[k][u], st[k].o[i]);
                }
            }
    }
    if (blk < hi) {   // the incomplete block, in 16 bits
        const uint16_t *kt = c.k_tail + bh * kTB * D, *vt = c.v_tail + bh * kTB * D;
        const int g = lane >> 4, left = len - blk * kTB;
        u32x4_t v[D / 16][2];
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int u = 0; u < 2; ++u) v[i][u] = *reinterpret_cast<const u32x4_t*>(vt + (16 * i + (lane & 15)) * kTB + 16 * g + 8 * u);
        f32x4_t s[RT][4] = {};
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                const u32x4_t x = *reinterpret_cast<const u32x4_t*>(kt + (16 * t + (lane & 15)) * D + 64 * (i >> 1) + 16 * g + 8 * (i & 1));
#pragma unroll
                for (int k = 0; k < RT; ++k) s[k][t] = T::mfma16(x, st[k].q[i], s[k][t]);
            }
        if (RT == 1 && logits) store_logits(logits + size_t(blk) * kTB * rows, s[0], rows, lane & 15, lane);
        uint32_t large = 0;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {   // what lies behind the length may be anything: zero, so that a weight of zero makes zero of it
                const int t = 16 * (2 * u + (e >> 1)) + 4 * g + 2 * (e & 1);
                const uint32_t stored = t + 1 < left ? 0xFFFFFFFFu : (t < left ? 0xFFFFu : 0u);
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    v[i][u][e] &= stored;
                    if (T::kWide) large |= large_values(v[i][u][e]);
                }
            }
        const float unit = weight_bits<T>(__any(large & kLargeValues));
        u32x4_t ph[RT][2], pl[RT][2], pr[RT][2];
#pragma unroll
        for (int k = 0; k < RT; ++k) st[k].template weights<EXACT>(s[k], blk * kTB, true, c2, unit, lane, ph[k], pl[k], pr[k]);
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int k = 0; k < RT; ++k) {
                    st[k].o[i] = T::mfma16(v[i][u], ph[k][u], st[k].o[i]);
                    if (EXACT) st[k].o[i] = T::mfma16(v[i][u], pl[k][u], st[k].o[i]);
                    if (EXACT && T::kWide) st[k].o[i] = T::mfma16(v[i][u], pr[k][u], st[k].o[i]);
                }
    }
}

}  // namespace akb
