// Tokens from a model's projections into the block-scaled 8-bit cache: norms per head, rotary positions, the append (rules and layout: include/akb.h).
#include "akb_pack.h"

namespace akb {

struct TurnArgs {
    akb_cache c;
    akb_tokens x;
    akb_rotary r;
    const int32_t* n_new;
    int n;
    uint16_t* q_out;
    int ticketed;
};

// sin and cos of place x freq.  The angle is made and brought into +-pi/4 in 64 bits (a place of 10^6 leaves 32 bits no digits behind the point), then the sums
// of their power series, cut where the next term is below 2^-28.
__device__ __forceinline__ void sin_cos(double place, float freq, float& s, float& c)
{
    constexpr double kTwoOverPi = 0.63661977236758134308, kHalfPi = 1.57079632679489661923, kHalfPiRest = 6.123233995736766e-17;
    const double u = place * double(freq), k = __builtin_rint(u * kTwoOverPi);
    const float r = float(fma(-k, kHalfPiRest, fma(-k, kHalfPi, u))), r2 = r * r;
    const int quarter = int(k - 4.0 * __builtin_floor(k * 0.25));
    float a = fmaf(r2, 1.f / 362880.f, -1.f / 5040.f);
    a = fmaf(r2, a, 1.f / 120.f);
    a = fmaf(r2, a, -1.f / 6.f);
    a = fmaf(r * r2, a, r);
    float b = fmaf(r2, -1.f / 3628800.f, 1.f / 40320.f);
    b = fmaf(r2, b, -1.f / 720.f);
    b = fmaf(r2, b, 1.f / 24.f);
    b = fmaf(r2, b, -0.5f);
    b = fmaf(r2, b, 1.f);
    const float p = quarter & 1 ? b : a, q = quarter & 1 ? a : b;
    s = quarter & 2 ? -p : p;
    c = (quarter + 1) & 2 ? -q : q;
}

// What a thread's eight channels of four tokens are multiplied with: x_d c_d + x_partner s_d
template <int D> struct Turn {
    float c[4][8], s[4][8];
    int partner;   // the lane that has the partners, or this one
    bool any, pairs;
    __device__ __forceinline__ void init(const akb_rotary& r, int oct, int lane)
    {
        pairs = r.pairs != 0;
        const int half = r.rot / 16;   // octets
        any = oct * 8 < r.rot;
        partner = !any || pairs ? lane : (oct < half ? lane + half : lane - half);
    }
    // of the token at `place`
    __device__ __forceinline__ void angles(const akb_rotary& r, int oct, int i, double place)
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            c[i][e] = 1.f;
            s[i][e] = -0.f;   // (a channel that does not turn keeps its sign of zero)
        }
        if (!any) return;
        if (pairs) {
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                sin_cos(place, r.inv_freq[oct * 4 + e / 2], s[i][e + 1], c[i][e]);
                s[i][e] = -s[i][e + 1];
                c[i][e + 1] = c[i][e];
            }
        } else {
            const int half = r.rot / 16;
            const bool low = oct < half;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sin_cos(place, r.inv_freq[(low ? oct : oct - half) * 8 + e], s[i][e], c[i][e]);
                if (low) s[i][e] = -s[i][e];
            }
        }
    }
};

// 1 / sqrt(mean of squares + eps) of a head whose channels lie in D / 8 lanes, eight in each.  Summed in 64 bits, where squares of every finite number have room;
// the root in 32 bits of a number between 1 and 4.
template <class T, int D> __device__ __forceinline__ float norm_scale(const u32x4_t& x, float eps)
{
    double sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const double a = T::lo(x[i]), b = T::hi(x[i]);
        sum = fma(a, a, sum);
        sum = fma(b, b, sum);
    }
#pragma unroll
    for (int d = 1; d < D / 8; d *= 2) sum += __shfl_xor(sum, d);
    const double m = sum * (1.0 / D) + double(eps);
    const int e = (__builtin_amdgcn_frexp_exp(m) - 1) >> 1;   // m 4^-e: in 1 .. 4
    return ldexpf(1.f / sqrtf(float(ldexp(m, -2 * e))), -e);
}

// Eight channels of a token, normed where there is a weight (`w`: this thread's, and its partners'), turned
template <class T, int D> __device__ __forceinline__ u32x4_t turned(const u32x4_t& x, const Turn<D>& t, int i, bool normed, float eps, const float (&w)[8], const float (&wp)[8])
{
    const float scale = normed ? norm_scale<T, D>(x, eps) : 1.f;
    u32x4_t p = x;
    if (!t.pairs)
#pragma unroll
        for (int k = 0; k < 4; ++k) p[k] = __shfl(int(x[k]), t.partner);
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int f = t.pairs ? e ^ 1 : e;
        float a = e & 1 ? T::hi(x[e >> 1]) : T::lo(x[e >> 1]), b = f & 1 ? T::hi(p[f >> 1]) : T::lo(p[f >> 1]);
        if (normed) {
            a = a * scale * w[e];
            b = b * scale * wp[e];
        }
        y[e] = fmaf(t.any ? b : 0.f, t.s[i][e], a * t.c[i][e]);
    }
    return u32x4_t{T::pack(y[0], y[1]), T::pack(y[2], y[3]), T::pack(y[4], y[5]), T::pack(y[6], y[7])};
}

// As append_kernel (akb_store.hip), with K turned on its way in; and the query heads of the KV head, whose tokens' angles are the same.
template <class T, int D>
__global__ __launch_bounds__(2 * D) void append_rotated_kernel(TurnArgs a)
{
    __shared__ PackLds<D> lds;
    const akb_cache& c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, h = blockIdx.y, b = blockIdx.z, j = blockIdx.x;
    const int Hkv = c.shape.Hkv, Ncap = c.shape.Ncap, G = c.shape.Hq / Hkv, n = a.n;
    const int len = seq_len(c, b), cnt = a.n_new ? min(max(a.n_new[b], 0), n) : n;
    if (cnt == 0) return;
    if (len + cnt > Ncap) {   // the sequence is left unchanged
        if (a.ticketed && j == 0 && h == 0 && tid == 0) atomicAdd(&c.flags[AKV_FLAG_OVERFLOW], 1);
        return;
    }
    int ticket = -1;
    if (a.ticketed) {   // drawn once all waves of the workgroup have read the length, looked at when it leaves
        __syncthreads();
        if (tid == 0) ticket = atomicAdd(&c.flags[AKV_NFLAGS + b], 1);
    }
    const size_t bh = size_t(b) * Hkv + h;
    const int first = len / kTB, had = len % kTB, total = had + cnt;   // counted from the start of block `first`
    const double place0 = double(a.r.base ? a.r.base[b / (c.shape.B / a.r.n_base)] : 0) + double(first * kTB);
    const BlockLane<D> at(tid);
    const int t0 = at.t0;
    Turn<D> turn;
    turn.init(a.r, at.oct, lane);
    float w[8], wp[8];
    auto weights = [&](const uint16_t* norm) {
        if (!norm) return;
        const u32x4_t x = *reinterpret_cast<const u32x4_t*>(norm + at.oct * 8);
        u32x4_t p = x;
        if (!turn.pairs)
#pragma unroll
            for (int k = 0; k < 4; ++k) p[k] = __shfl(int(x[k]), turn.partner);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int f = turn.pairs ? e ^ 1 : e;
            w[e] = e & 1 ? T::hi(x[e >> 1]) : T::lo(x[e >> 1]);
            wp[e] = f & 1 ? T::hi(p[f >> 1]) : T::lo(p[f >> 1]);
        }
    };
    auto fresh = [&](int t) { return t >= had && t < total; };   // token t counted from the start of block `first`
    auto angles = [&](int w0) {
#pragma unroll
        for (int r = 0; r < 4; ++r) turn.angles(a.r, at.oct, r, place0 + double(w0 + t0 + r));
    };
    auto load = [&](const uint16_t* x, int64_t seq, int64_t token, int head, int w0, u32x4_t (&to)[4]) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int t = w0 + t0 + r;
            to[r] = fresh(t) ? *reinterpret_cast<const u32x4_t*>(x + b * seq + (t - had) * token + head * D + at.oct * 8) : u32x4_t{0, 0, 0, 0};
        }
    };
    auto load_k = [&](int w0, u32x4_t (&to)[4]) {   // (the angles are those of w0)
        load(a.x.k, a.x.k_seq, a.x.k_token, h, w0, to);
#pragma unroll
        for (int r = 0; r < 4; ++r) to[r] = turned<T, D>(to[r], turn, r, a.r.k_norm, a.r.eps, w, wp);
    };
    if (j * kTB < total) angles(j * kTB);
    weights(a.r.k_norm);
    const bool complete = (j + 1) * kTB <= total, tail = j == 0 && total % kTB;
    const int last = total / kTB * kTB;
    u32x4_t x[4];
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const bool is_v = side == 1;
        if (complete) {
            if (is_v) load(a.x.v, a.x.v_seq, a.x.v_token, h, j * kTB, x);
            else load_k(j * kTB, x);
            if (j == 0 && had > 0) {
                const bool old[4] = {t0 < had, t0 + 1 < had, t0 + 2 < had, t0 + 3 < had};
                const int token[4] = {t0, t0 + 1, t0 + 2, t0 + 3};
                load_tail<D, true>(c, bh, is_v, x, old, token);
            }
            if (is_v) __syncthreads();   // K's block has been packed
            pack_block<T, D, false>(c, bh * (Ncap / kTB) + first + j, is_v, x, lds);
        }
    }
    if (a.q_out && j * kTB < total) {
        weights(a.r.q_norm);
        for (int g = 0; g < G; ++g) {
            load(a.x.q, a.x.q_seq, a.x.q_token, h * G + g, j * kTB, x);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[r] = turned<T, D>(x[r], turn, r, a.r.q_norm, a.r.eps, w, wp);
                const int t = j * kTB + t0 + r;
                if (fresh(t)) *reinterpret_cast<u32x4_t*>(a.q_out + ((bh * G + g) * n + (t - had)) * D + at.oct * 8) = x[r];
            }
        }
    }
    if (tail) {   // the incomplete block: its new tokens go to the tail (what of the old ones is needed has been read)
        __syncthreads();
        bool store[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) store[r] = fresh(last + t0 + r);
        if (last) angles(last);
        weights(a.r.k_norm);
        load_k(last, x);
        store_tail<D>(c, bh, false, x, store);
        load(a.x.v, a.x.v_seq, a.x.v_token, h, last, x);
        store_tail<D>(c, bh, true, x, store);
    }
    if (c.score && tid < kTB) {   // the new tokens' scores
        const int t = j * kTB + tid;
        if (fresh(t)) c.score[bh * Ncap + first * kTB + t] = 0.f;
    }
    if (ticket == int(gridDim.x) * Hkv - 1) {   // the last workgroup of the sequence (thread 0 of it)
        c.flags[AKV_NFLAGS + b] = 0;
        c.lens[b] = len + cnt;
    }
}

hipError_t launch_append_rotated(const akb_cache& c, const akb_tokens& x, const int32_t* n_new, int n, uint16_t* q_out, const akb_rotary& r, hipStream_t st)
{
    const int blocks = (kTB - 1 + n + kTB - 1) / kTB;
    const dim3 grid(blocks, c.shape.Hkv, c.shape.B);
    const bool ticketed = append_ticketed(c.shape, n);
    const TurnArgs a{c, x, r, n_new, n, q_out, ticketed ? 1 : 0};
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(2 * c.shape.D), 0, st, a); };
    if (c.shape.dtype == AKB_FP16) c.shape.D == 64 ? launch(append_rotated_kernel<Fp16, 64>) : launch(append_rotated_kernel<Fp16, 128>);
    else c.shape.D == 64 ? launch(append_rotated_kernel<Bf16, 64>) : launch(append_rotated_kernel<Bf16, 128>);
    if (hipError_t e = hipGetLastError()) return e;
    return ticketed ? hipSuccess : launch_append_lens(c, n_new, n, st);
}

}  // namespace akb
