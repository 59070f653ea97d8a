// Tokens from a model's projections into the block-scaled 8-bit cache: norms per head, rotary positions, the append (rules and layout: include/akb.h).
//
// Keys are normed and turned in 64 bits, rounded to binary32 and from there to the 16-bit type: their largest number decides a block's exponent, and in 32 bits throughout one key
// in some thousand came out as another 16-bit number.  (What the step between costs: a key whose binary32 number is the middle of two 16-bit ones, one in some 2^13 in binary16 and
// 2^16 in bfloat16, may be off by 2^-25 of itself more than half a step.)  Queries are normed and turned in 32 bits, by the same angles, sine and cosine rounded to binary32.
// Bound by memory where it is large (4 x 8192 tokens of 32 + 16 heads: 738 MB in 151 to 163 us by the card, 4.5 to 4.9 TB/s, where a plain copy moves 5.1 in and out; without norms
// and with 16 channels turned 147), by the chain of loads, sums and stores of a workgroup where it is small.
// A row (a token of a head) lies in D / 8 lanes, eight channels in each; a workgroup has a block's 64 tokens, 16 rows at a time.  Sine and cosine are made by their power series
// for a thread's first token (half of them by the lane of the other channels of the pairs), and turned on by 16 tokens, in 64 bits, for the next.
#include "akb_pack.h"

namespace akb {

constexpr int kApart = 4;   // query heads of a workgroup of their own
struct TurnArgs {
    akb_cache c;
    akb_tokens x;
    akb_rotary r;
    const int32_t* n_new;
    int n;
    uint16_t* q_out;
    int ticketed;
    // Workgroups of a sequence: `blocks` x KV heads, each of which has 64 tokens of a KV head and, unless `apart`, of its query heads; where apart, as many for every
    // kApart of the query heads (`apart` parts); where the tokens are few, `rows` that have 16 rows each
    int blocks, apart, rows;
};
typedef double f64x2_t __attribute__((ext_vector_type(2)));

// cos, sin of place x freq: the angle brought into +-pi/4 (pi / 2 in two parts), then the sums of the power series, cut where the next term is below 2^-50.
__device__ __forceinline__ f64x2_t cos_sin(double place, float freq)
{
    constexpr double kTwoOverPi = 0.63661977236758134308, kHalfPi = 1.57079632679489661923, kHalfPiRest = 6.123233995736766e-17;
    const double u = place * double(freq), k = __builtin_rint(u * kTwoOverPi), r = fma(-k, kHalfPiRest, fma(-k, kHalfPi, u)), r2 = r * r;
    const int quarter = int(k - 4.0 * __builtin_floor(k * 0.25));
    double a = 1.0 / 1307674368000.0, b = 1.0 / 20922789888000.0;   // -r^15 / 15!, r^16 / 16!
    a = fma(r2, -a, 1.0 / 6227020800.0);
    a = fma(r2, a, -1.0 / 39916800.0);
    a = fma(r2, a, 1.0 / 362880.0);
    a = fma(r2, a, -1.0 / 5040.0);
    a = fma(r2, a, 1.0 / 120.0);
    a = fma(r2, a, -1.0 / 6.0);
    a = fma(r * r2, a, r);
    b = fma(r2, b, -1.0 / 87178291200.0);
    b = fma(r2, b, 1.0 / 479001600.0);
    b = fma(r2, b, -1.0 / 3628800.0);
    b = fma(r2, b, 1.0 / 40320.0);
    b = fma(r2, b, -1.0 / 720.0);
    b = fma(r2, b, 1.0 / 24.0);
    b = fma(r2, b, -0.5);
    b = fma(r2, b, 1.0);
    const double s = quarter & 1 ? b : a, c = quarter & 1 ? a : b;
    return f64x2_t{(quarter + 1) & 2 ? -c : c, quarter & 2 ? -s : s};
}

// Which pair each of a thread's eight channels belongs to, and where the other channel of it is.  NEXT: pairs of neighbours (akb_rotary.pairs).
template <int D, bool NEXT> struct Pairs {
    int first, step;      // number of the first channel's pair; how many octets (lanes) further the partners are
    int partner;          // four times their lane
    bool any;
    uint32_t minus;       // sign bit where these channels are the first of their pairs, which take their partners times -sin (NEXT: every other one is)
    __device__ __forceinline__ Pairs(int rot, int oct, int lane)
    {
        const int half = rot / 16;   // octets
        const bool low = oct < half;
        any = oct * 8 < rot;
        step = !any || NEXT ? 0 : (low ? half : -half);
        partner = 4 * (lane + step);
        first = !any ? 0 : (NEXT ? oct * 4 : (low ? oct : oct - half) * 8);
        minus = low ? 0x80000000u : 0u;
    }
    // a partner's number with the sign that its sine has
    __device__ __forceinline__ float signed_for(int e, float v) const { return NEXT ? (e & 1 ? v : -v) : bits_float(float_bits(v) ^ minus); }
    __device__ __forceinline__ uint32_t other(uint32_t w) const { return uint32_t(__builtin_amdgcn_ds_bpermute(partner, int(w))); }
    __device__ __forceinline__ double other(double v) const
    {
        const u32x2_t w = __builtin_bit_cast(u32x2_t, v);
        const uint32_t lo = w.x, hi = w.y;
        return __builtin_bit_cast(double, u32x2_t{other(lo), other(hi)});
    }
    __device__ __forceinline__ u32x4_t others(const u32x4_t& x) const
    {
        u32x4_t p;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t w = x[k];
            p[k] = NEXT ? w >> 16 | w << 16 : other(w);
        }
        return p;
    }
};
// cos, sin of one token more
__device__ __forceinline__ f64x2_t turn_on(f64x2_t cs, f64x2_t on) { return f64x2_t{fma(cs[0], on[0], -cs[1] * on[1]), fma(cs[1], on[0], cs[0] * on[1])}; }
// What is made from x is made again behind this, not kept from turn to turn of a loop: the registers are few
template <class V> __device__ __forceinline__ void forget(V& x) { asm volatile("" : "+v"(x)); }

template <class T> __device__ __forceinline__ float channel(const u32x4_t& x, int e) { return e & 1 ? T::hi(x[e >> 1]) : T::lo(x[e >> 1]); }

// v of the lane that CTRL (a permutation of the lanes of 16) names
template <int CTRL> __device__ __forceinline__ float dpp(float v) { return bits_float(uint32_t(__builtin_amdgcn_update_dpp(0, int(float_bits(v)), CTRL, 0xF, 0xF, true))); }
template <int CTRL> __device__ __forceinline__ double dpp(double v)
{
    const u32x2_t w = __builtin_bit_cast(u32x2_t, v);
    const uint32_t lo = w.x, hi = w.y;
    return __builtin_bit_cast(double, u32x2_t{uint32_t(__builtin_amdgcn_update_dpp(0, int(lo), CTRL, 0xF, 0xF, true)), uint32_t(__builtin_amdgcn_update_dpp(0, int(hi), CTRL, 0xF, 0xF, true))});
}
// the sum over a row's D / 8 lanes, in each of them
template <int D, class V> __device__ __forceinline__ V row_sum(V v)
{
    v += dpp<0xB1>(v);    // neighbours
    v += dpp<0x4E>(v);    // pairs of them
    v += dpp<0x141>(v);   // fours: mirrored in eight lanes
    if (D == 128) v += dpp<0x128>(v);   // eights: turned by eight lanes
    return v;
}
// 1 / sqrt(mean of a row's squares + eps): in 64 bits, where squares of every finite number have room, ..
template <class T, int D> __device__ __forceinline__ double norm_scale(const u32x4_t& x, float eps)
{
    double sum = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const double a = channel<T>(x, e);
        sum = fma(a, a, sum);
    }
    const double m = fma(row_sum<D>(sum), 1.0 / D, double(eps));
    double y = __builtin_amdgcn_rsq(m);
    y = y * fma(-0.5 * m * y, y, 1.5);
    return y * fma(-0.5 * m * y, y, 1.5);
}
// .. and in 32, unless this row's have none there (which is the same in all of its lanes)
template <class T, int D> __device__ __forceinline__ float norm_scale32(const u32x4_t& x, float eps)
{
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fmaf(channel<T>(x, e), channel<T>(x, e), sum);
    sum = row_sum<D>(sum);
    if (!(sum > 0x1p-100f && sum < 0x1p120f)) return float(norm_scale<T, D>(x, eps));
    return __builtin_amdgcn_rsqf(fmaf(sum, 1.f / D, eps));
}

// As append_kernel (akb_store.hip), with K turned on its way in; and the query heads of the KV head, whose tokens' angles are the same.
// NT: with the non-temporal hint.
template <class T, int D, bool NEXT, bool NT>
__global__ __launch_bounds__(2 * D, NEXT ? 3 : 4) void append_rotated_kernel(TurnArgs a)
{
    constexpr int kHeads = 2;          // that are asked for at a time
    constexpr int kRow = 2 * D + 16;   // bytes of a turned key in LDS: shifted by four banks from token to token
    __shared__ PackLds<D> lds;
    __shared__ __align__(16) uint8_t rows_s[kTB * kRow];
    __shared__ f64x2_t on_s[D / 2];    // cos, sin of 16 tokens
    __shared__ u32x4_t norm_s[2][D / 8];   // the norms' weights, of queries and of keys
    const akb_cache& c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, b = blockIdx.y;
    const int Hkv = c.shape.Hkv, walks = a.blocks * Hkv, Ncap = c.shape.Ncap, n = a.n;
    const bool behind = int(blockIdx.x) >= walks, in_rows = behind && a.rows > 0;
    // (a head's blocks one behind the other: the heads of a block beside each other 162 us of 4 x 8192 tokens for 151)
    const int walk = behind ? blockIdx.x - walks : blockIdx.x, h = walk / a.blocks % Hkv, j = walk % a.blocks;
    const int len = seq_len(c, b), cnt = a.n_new ? min(max(a.n_new[b], 0), n) : n;
    if (cnt == 0) return;
    if (len + cnt > Ncap) {   // the sequence is left unchanged
        if (a.ticketed && blockIdx.x == 0 && tid == 0) atomicAdd(&c.flags[AKV_FLAG_OVERFLOW], 1);
        return;
    }
    if (tid < 2 * (D / 8)) {
        const uint16_t* norm = tid < D / 8 ? a.r.q_norm : a.r.k_norm;
        if (norm) norm_s[0][tid] = *reinterpret_cast<const u32x4_t*>(norm + tid % (D / 8) * 8);
    }
    __syncthreads();
    int ticket = -1;   // drawn once all waves of the workgroup have read the length, looked at when it leaves
    if (a.ticketed && tid == 0) ticket = atomicAdd(&c.flags[AKV_NFLAGS + b], 1);
    const bool few = a.rows > 0 && len % kTB + cnt < kTB;   // few: the rows' workgroups turn the keys and store the values, too
    const bool do_q = a.q_out && a.rows == 0 && behind == (a.apart != 0), do_kv = !behind && !few;
    const size_t bh = size_t(b) * Hkv + h;
    const int first = len / kTB, had = len % kTB, total = had + cnt;   // counted from the start of block `first`
    const double place0 = double(a.r.base ? a.r.base[b / (c.shape.B / a.r.n_base)] : 0) + double(first) * kTB;
    const BlockLane<D> at(tid);
    const int t0 = at.t0;
    const Pairs<D, NEXT> pairs(a.r.rot, at.oct, lane);
    auto fresh = [&](int t) { return t >= had && t < total; };   // token t counted from the start of block `first`
    auto get = [&](const uint16_t* p) -> u32x4_t { return NT ? __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p)) : *reinterpret_cast<const u32x4_t*>(p); };
    // cos, sin of a thread's pairs at a place (NEXT: its channels are four pairs; otherwise eight, of which its partner makes the other four)
    auto first_turns = [&](double place, f64x2_t (&cs)[8]) {
        f64x2_t made[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) made[e] = pairs.any ? cos_sin(place, a.r.inv_freq[pairs.first + e + (NEXT || pairs.minus ? 0 : 4)]) : f64x2_t{1.0, 0.0};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (NEXT) {
                cs[2 * e] = cs[2 * e + 1] = made[e];
            } else {
                const f64x2_t other = {pairs.other(made[e][0]), pairs.other(made[e][1])};
                cs[e] = pairs.minus ? made[e] : other;
                cs[4 + e] = pairs.minus ? other : made[e];
            }
        }
    };
    // eight channels of a key (octet `oct`)
    auto turn_key = [&](const u32x4_t& k, const f64x2_t (&cs)[8], int oct) {
        const u32x4_t w = norm_s[1][oct], wo = NEXT ? pairs.others(w) : norm_s[1][oct + pairs.step];   // the norm's weights, those of the partners
        const u32x4_t o = pairs.others(k);
        const double scale = a.r.k_norm ? norm_scale<T, D>(k, a.r.eps) : 1.0;
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            double u = channel<T>(k, e);
            if (a.r.k_norm) u *= double(channel<T>(w, e)) * scale;
            if (pairs.any) {
                double v = pairs.signed_for(e, channel<T>(o, e));
                if (a.r.k_norm) v *= double(channel<T>(wo, e)) * scale;
                u = fma(v, cs[e][1], u * cs[e][0]);
            }
            y[e] = float(u);
            if (e & 1) __builtin_amdgcn_sched_barrier(0);   // (all eight at a time do not fit the registers)
        }
        return u32x4_t{T::pack(y[0], y[1]), T::pack(y[2], y[3]), T::pack(y[4], y[5]), T::pack(y[6], y[7])};
    };
    // ... of queries: cosine times a channel's weight, sine times its partner's
    auto query_turns = [&](const f64x2_t (&cs)[8], int oct, float (&cw)[8], float (&sw)[8]) {
        const u32x4_t w = norm_s[0][oct], wo = NEXT ? pairs.others(w) : norm_s[0][oct + pairs.step];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            cw[e] = float(cs[e][0]) * (a.r.q_norm ? channel<T>(w, e) : 1.f);
            sw[e] = float(cs[e][1]) * pairs.signed_for(e, a.r.q_norm ? channel<T>(wo, e) : 1.f);
        }
    };
    auto turn_query_by = [&](const u32x4_t& q, const float (&cw)[8], const float (&sw)[8]) {
        const u32x4_t o = pairs.others(q);
        const float scale = a.r.q_norm ? norm_scale32<T, D>(q, a.r.eps) : 1.f;
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {   // the scale first: a channel times its weight may have no room in 32 bits (bfloat16)
            y[e] = channel<T>(q, e) * scale * cw[e];
            if (pairs.any) y[e] = fmaf(channel<T>(o, e) * scale, sw[e], y[e]);
        }
        return u32x4_t{T::pack(y[0], y[1]), T::pack(y[2], y[3]), T::pack(y[4], y[5]), T::pack(y[6], y[7])};
    };
    // The new tokens among the 64 from w0 on: keys to LDS (for a complete block) or to the tail; queries to q_out
    auto turn_rows = [&](int w0, bool keys, bool to_tail, bool queries) {
        const int G = c.shape.Hq / Hkv, part = behind ? walk / walks * kApart : 0, head0 = h * G + part, heads = behind ? min(kApart, G - part) : G;   // the query heads
        const int begin = max(had - w0, 0), end = min(total - w0, kTB) - 1;
        if (begin / 16 != end / 16) {   // (otherwise nothing is turned on)
            if (tid < a.r.rot / 2) on_s[tid] = cos_sin(16.0, a.r.inv_freq[tid]);
            __syncthreads();
        }
        // a wave's rows that are new lie one behind the other: the first, and its loads, here (the power series' constants would fill the loop's registers)
        int i = 0;
        while (i < 4 && !__any(fresh(w0 + 16 * i + at.grp))) ++i;
        if (i == 4) return;
        u32x4_t k, q[kHeads];
        auto fetch = [&](int t, int g0) {   // the query rows of some heads
#pragma unroll
            for (int g = 0; g < kHeads; ++g)
                q[g] = fresh(t) && g0 + g < heads ? get(a.x.q + b * a.x.q_seq + (t - had) * a.x.q_token + (head0 + g0 + g) * D + at.oct * 8) : u32x4_t{0, 0, 0, 0};
        };
        auto fetch_key = [&](int t) {
            if (keys) k = fresh(t) ? get(a.x.k + b * a.x.k_seq + (t - had) * a.x.k_token + h * D + at.oct * 8) : u32x4_t{0, 0, 0, 0};
        };
        fetch_key(w0 + 16 * i + at.grp);
        if (queries) fetch(w0 + 16 * i + at.grp, 0);
        f64x2_t cs[8];
        first_turns(place0 + double(w0 + 16 * i + at.grp), cs);
#pragma unroll 1
        for (;;) {
            const int t = w0 + 16 * i + at.grp;
            const bool mine = fresh(t);
            int pair0 = pairs.first, oct = at.oct;
            forget(pair0);
            forget(oct);
            if (keys) {
                const u32x4_t z = turn_key(k, cs, oct);
                if (!to_tail) *reinterpret_cast<u32x4_t*>(rows_s + (t - w0) * kRow + at.oct * 16) = z;
                else if (mine) *reinterpret_cast<u32x4_t*>(c.k_tail + (bh * kTB + (t - w0)) * D + at.oct * 8) = z;
            }
            if (queries) {
                float cw[8], sw[8];
                query_turns(cs, oct, cw, sw);
                for (int g0 = 0;;) {
#pragma unroll
                    for (int g = 0; g < kHeads; ++g) {
                        if (g0 + g >= heads) break;
                        const u32x4_t z = turn_query_by(q[g], cw, sw);
                        if (!mine) continue;
                        u32x4_t* out = reinterpret_cast<u32x4_t*>(a.q_out + ((size_t(b) * c.shape.Hq + head0 + g0 + g) * n + (t - had)) * D + at.oct * 8);
                        if (NT) __builtin_nontemporal_store(z, out);
                        else *out = z;
                    }
                    if ((g0 += kHeads) >= heads) break;
                    fetch(t, g0);
                }
            }
            if (++i == 4 || !__any(fresh(t + 16))) break;
            fetch_key(t + 16);
            if (queries) fetch(t + 16, 0);
            if (pairs.any)
#pragma unroll
                for (int e = 0; e < 8; ++e) cs[e] = turn_on(cs[e], on_s[pair0 + (NEXT ? e >> 1 : e)]);
        }
    };
    auto load_v = [&](int w0, u32x4_t (&to)[4]) {
        const uint16_t* p = a.x.v + b * a.x.v_seq + (w0 + t0 - had) * a.x.v_token + h * D + at.oct * 8;
#pragma unroll
        for (int r = 0; r < 4; ++r) to[r] = fresh(w0 + t0 + r) ? get(p + r * a.x.v_token) : u32x4_t{0, 0, 0, 0};
    };
    if (in_rows) {   // row by row: the query heads, the KV heads' keys and, where the tail takes them, values of each token
        const int heads = c.shape.Hq + 2 * Hkv, row = walk * 16 + at.grp, i = row / heads, s = row - i * heads;
        const bool is_q = s < c.shape.Hq, is_k = !is_q && s < c.shape.Hq + Hkv;
        if (i < cnt && (is_q ? a.q_out != nullptr : few)) {
            const int head = is_q ? s : (is_k ? s - c.shape.Hq : s - c.shape.Hq - Hkv);
            const u32x4_t v = get(is_q ? a.x.q + b * a.x.q_seq + i * a.x.q_token + head * D + at.oct * 8
                                       : (is_k ? a.x.k + b * a.x.k_seq + i * a.x.k_token : a.x.v + b * a.x.v_seq + i * a.x.v_token) + head * D + at.oct * 8);
            if (is_q || is_k) {
                f64x2_t cs[8];
                first_turns(place0 + double(had + i), cs);
                if (is_q) {
                    float cw[8], sw[8];
                    query_turns(cs, at.oct, cw, sw);
                    *reinterpret_cast<u32x4_t*>(a.q_out + ((size_t(b) * c.shape.Hq + head) * n + i) * D + at.oct * 8) = turn_query_by(v, cw, sw);
                } else {
                    *reinterpret_cast<u32x4_t*>(c.k_tail + ((size_t(b) * Hkv + head) * kTB + had + i) * D + at.oct * 8) = turn_key(v, cs, at.oct);
                }
            } else {
                uint16_t* to = c.v_tail + ((size_t(b) * Hkv + head) * D + at.oct * 8) * kTB + v_place(had + i);
#pragma unroll
                for (int e = 0; e < 8; ++e) to[e * kTB] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
                if (c.score && at.oct == 0) c.score[(size_t(b) * Hkv + head) * Ncap + len + i] = 0.f;
            }
        }
    }
    const bool some = !in_rows && (do_q || do_kv) && j * kTB < total, complete = (j + 1) * kTB <= total;
    // the incomplete block goes to the tail by the workgroup that has it, or, where the tail holds what the first block takes, by the workgroup of that
    const int last = total / kTB * kTB;
    const bool tail = total % kTB && (had > 0 ? j == 0 : j * kTB == last), tail_here = tail && j * kTB == last;
    u32x4_t x[4];
    if (some) turn_rows(j * kTB, do_kv && (complete || tail_here), tail_here, do_q);
    if (do_kv && complete) {
        __syncthreads();
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const bool is_v = side == 1;
            if (is_v) {
                load_v(j * kTB, x);
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r) x[r] = *reinterpret_cast<const u32x4_t*>(rows_s + (t0 + r) * kRow + at.oct * 16);
            }
            if (j == 0 && had > 0) {
                const bool old[4] = {t0 < had, t0 + 1 < had, t0 + 2 < had, t0 + 3 < had};
                const int token[4] = {t0, t0 + 1, t0 + 2, t0 + 3};
                load_tail<D, true>(c, bh, is_v, x, old, token);
            }
            if (is_v) __syncthreads();   // K's block has been packed
            pack_block<T, D, NT>(c, bh * (Ncap / kTB) + first + j, is_v, x, lds);
        }
    }
    if (do_kv && tail) {   // its new tokens go to the tail (what of the old ones is needed has been read)
        if (!tail_here) {
            __syncthreads();
            turn_rows(last, true, true, false);
        }
        bool store[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) store[r] = fresh(last + t0 + r);
        load_v(last, x);
        store_tail<D>(c, bh, true, x, store);
    }
    if (do_kv && c.score && tid < kTB) {   // the new tokens' scores
        const int t = j * kTB + tid;
        if (fresh(t)) c.score[bh * Ncap + first * kTB + t] = 0.f;
    }
    if (ticket == int(gridDim.x) - 1) {   // the last workgroup of the sequence (thread 0 of it)
        c.flags[AKV_NFLAGS + b] = 0;
        c.lens[b] = len + cnt;
    }
}

constexpr int kFewTokens = 8;
// How a call is shared out
struct RotatedPlan {
    int blocks, rows, apart;   // TurnArgs
    bool ticketed, streamed;
};
static RotatedPlan plan(const akb_shape& s, int n, bool queries)
{
    RotatedPlan p;
    p.blocks = (kTB - 1 + n + kTB - 1) / kTB;
    // Few tokens: row by row, 16 to a workgroup, which leaves little to any.  Otherwise / row by row, us, the copy that sets the lengths with them, 32 heads on 8 at D = 128 where not
    // said otherwise.  One token: 64 sequences 14.0 / 13.7, of 64 heads 20.7 / 13.3, 256 sequences 25.0 / 16.9.  Eight: 23.8 / 23.6, 25.5 / 25.1, 52.1 / 49.2, at D = 64 17.3 / 18.6.
    // Nine: 23.1 / 24.7, 26.7 / 28.4, 54.1 / 52.2, 17.9 / 18.8.  Twelve: 24.1 / 27.8, 27.9 / 31.6, 57.9 / 68.5, 21.1 / 21.2.  (Four sequences: 13.2 to 13.8 all of them.)
    p.rows = n <= kFewTokens ? (n * (s.Hq + 2 * s.Hkv) + 15) / 16 : 0;
    // Where they are few, workgroups of two waves (D = 64) and those of many query heads leave the query heads to others.  Beside / apart, us, by the workgroups that have KV heads.
    // D = 64, 200 tokens: groups of four, 500 28.1 / 22.0, 1020 31.8 / 28.6, 1200 35.6 / 30.2, 1600 36.3 / 36.4, 2400 49.2 / 54.8 (777 tokens: 1008 31.3 / 28.6, 1176 33.9 / 34.3); of
    // eight, 1020 42.2 / 36.5, 2400 66.8 / 72.4; of one, 900 24.7 / 24.8, 1020 25.9 / 26.8, 1600 29.2 / 33.9.  D = 128, 200 tokens: groups of eight, 240 37.3 / 30.6, 500 39.7 / 35.4,
    // 640 48.3 / 42.9, 800 54.4 / 53.6, 1200 66.3 / 72.5; of five, 120 29.5 / 23.4, 480 32.4 / 33.2, 640 34.3 / 36.6; of sixteen, 777 tokens, 504 82.0 / 69.4, 784 96.4 / 97.2.  Groups of
    // four at D = 128 stay beside: two sequences of eight KV heads 24.9 / 25.7, though 120 to 500 workgroups of four gain, 400 28.5 / 25.4, and lose again
    // from 640 on, 31.5 / 31.6, 800 33.2 / 38.0.
    const int G = s.Hq / s.Hkv;
    const long walks = long(p.blocks) * s.Hkv * s.B;
    p.apart = p.rows == 0 && queries && (s.D == 64 ? walks <= 1024 : (G > kApart && walks <= 512)) ? (G + kApart - 1) / kApart : 0;
    // The append's line.  Tickets / a launch behind, us: one block, 512 workgroups 14.1 / 16.9, 640 14.1 / 17.0, 1024 14.2 / 16.9 (32 sequences of 32 KV heads 17.8 / 16.8); two or more,
    // 288 31.0 / 31.6, 29.3 / 29.3, at D = 64 with query heads apart 24.0 / 20.4, 384 15.4 / 17.1 (five tokens), 31.4 / 32.1, 30.6 / 30.4, 23.2 / 19.8, 512 16.9 / 16.9, 32.7 / 32.4.
    p.ticketed = append_ticketed(s, n);
    // As in the append: tensors of more than half of the last-level cache are read and written with the non-temporal hint.  Plain / with it, us, 32 heads on 8 at D = 128; one set of
    // tensors used again and again, 96 MB 31.4 / 35.4, 128 36.9 / 41.6, 160 39.4 / 46.3, 256 73.4 / 74.4, 512 140 / 136; four sets in turn, which no cache holds, 48 26.3 / 28.9, 64
    // 32.9 / 31.9, 96 38.1 / 35.5, 128 44.4 / 42.0, 160 50.1 / 47.7, 512 141 / 138: by where the projection left them the line would be at 64 or at 256.
    p.streamed = (size_t(queries ? 2 * s.Hq : 0) + 2 * size_t(s.Hkv)) * s.B * n * s.D * 2 > (size_t(128) << 20);
    return p;
}
int rotated_path(const akb_shape& s, int n, bool queries, int32_t* how)
{
    const RotatedPlan p = plan(s, n, queries);
    if (how) {
        how[0] = p.streamed;
        how[1] = p.ticketed;
    }
    return p.rows ? 1 : (p.apart ? 3 : 2);
}
hipError_t launch_append_rotated(const akb_cache& c, const akb_tokens& x, const int32_t* n_new, int n, uint16_t* q_out, const akb_rotary& r, hipStream_t st)
{
    const RotatedPlan p = plan(c.shape, n, q_out != nullptr);
    const dim3 grid(p.blocks * c.shape.Hkv * (1 + p.apart) + p.rows, c.shape.B);
    const TurnArgs a{c, x, r, n_new, n, q_out, p.ticketed ? 1 : 0, p.blocks, p.apart, p.rows};
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(2 * c.shape.D), 0, st, a); };
    auto pick = [&](auto type, auto width) {
        using T = decltype(type);
        constexpr int D = decltype(width)::value;
        if (r.pairs) p.streamed ? launch(append_rotated_kernel<T, D, true, true>) : launch(append_rotated_kernel<T, D, true, false>);
        else p.streamed ? launch(append_rotated_kernel<T, D, false, true>) : launch(append_rotated_kernel<T, D, false, false>);
    };
    using D64 = std::integral_constant<int, 64>;
    using D128 = std::integral_constant<int, 128>;
    if (c.shape.dtype == AKB_FP16) c.shape.D == 64 ? pick(Fp16(), D64()) : pick(Fp16(), D128());
    else c.shape.D == 64 ? pick(Bf16(), D64()) : pick(Bf16(), D128());
    if (hipError_t e = hipGetLastError()) return e;
    return p.ticketed ? hipSuccess : launch_append_lens(c, n_new, n, st);
}

}  // namespace akb
