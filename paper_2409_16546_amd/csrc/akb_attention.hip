// Attention over the block-scaled 8-bit cache (rules and layout: include/akb.h).
//
// Rows: the query rows of one (sequence, KV head) are its n_q query tokens times its G query heads, row = token * G + head, so
// that one walk over K and V serves the whole group; 16 rows form a matrix tile.
// Both products are taken transposed, S^T = K Q^T and O^T = V^T P^T, so that a lane's column is a query row throughout: its
// four scores of a tile are four tokens of one row, which is what the second product takes as its operand (V's bytes lie in
// that order), and the running maximum, the sum and the rescaling of a row need no value of another row's lanes.
#include "akb_common.h"

namespace akb {

// In 16 bits the weights of fp16 caches would lose bits below 2^-14: they are taken relative to 2^-14 of the maximum (up to 2^14).
constexpr float kWeightBits = 14.f;
constexpr int kWaves = 4;

// what one row tile of one split of the tokens gives: O [16][D], then (maximum, sum) per row
template <int D> constexpr int part_floats() { return 16 * D + 32; }

struct AttentionPlan {
    int groups;   // row tiles of a (sequence, KV head)
    int splits;   // parts its blocks are cut into
    size_t parts, stats, total;   // offsets into the workspace
};
// (a call has more than one split only where there are fewer row tiles than 2 workgroups per unit, and then at most twice as many parts)
static AttentionPlan plan(const akb_shape& s, int n, int max_len, bool accumulate)
{
    AttentionPlan p;
    p.groups = (int)((long(n) * (s.Hq / s.Hkv) + 15) / 16);
    const long items = long(s.B) * s.Hkv * p.groups, blocks = (max_len + kTB - 1) / kTB;
    const long want = (2L * akv::compute_units() + items - 1) / items;
    p.splits = (int)std::max(1L, std::min(want, (blocks + kWaves - 1) / kWaves));
    p.parts = 0;
    p.stats = align256(size_t(4) * akv::compute_units() * (16 * s.D + 32) * sizeof(float));
    p.total = p.stats + (accumulate ? align256(size_t(items) * 32 * sizeof(float)) : 0);
    return p;
}
size_t attention_workspace(const akb_shape& s, int n, bool accumulate)
{
    return plan(s, n, s.Ncap, accumulate).total;
}

struct RowArgs {
    akb_cache c;
    const uint16_t* q;
    const int32_t* n_q;
    int n, groups, splits, out_dtype;
    void* out;
    float c2;
    float *parts, *stats;   // stats: (maximum, 1 / sum) per row, or NULL
};

// The tokens that rows see: row r (its query token r / G of m) the first `limit`
__device__ __forceinline__ int row_limit(int row, int G, int m, int len) { return row < m * G ? len - m + row / G + 1 : 0; }

// A block of K as the operand of S^T: lane (token t % 16, quarter g of 64 channels), [tile][64 channels]: 16 codes
template <int D> struct Codes {
    u32x4_t k[4][D / 64], v[D / 16];
    float ks, vs;
    __device__ __forceinline__ void load(const akb_cache& c, size_t block, int lane)
    {
        const size_t at = block * (kTB * D) + (lane & 15) * 64 + (lane >> 4) * 16;
        const uint8_t *kp = c.k8 + at, *vp = c.v8 + at;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < D / 64; ++i) k[t][i] = *reinterpret_cast<const u32x4_t*>(kp + t * (16 * D) + i * 1024);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) v[i] = *reinterpret_cast<const u32x4_t*>(vp + i * 1024);
        ks = pow2(c.exps[block * 2]);
        vs = pow2(c.exps[block * 2 + 1]);
    }
};

// Running state of a row tile in one wave: lane (row l % 16, g): channels 16 i + 4 g .. + 3 of O, the row's maximum, its share of the sum
template <class T, int D> struct RowState {
    u32x4_t q[D / 32];
    f32x4_t o[D / 16];
    float m, z;
    // channel order of the first product: step s of 32 channels, lane group g: 64 (s / 2) + 16 g + 8 (s % 2) .. + 7
    __device__ __forceinline__ void init(const uint16_t* qrow, int lane)
    {
        const int g = lane >> 4;
#pragma unroll
        for (int s = 0; s < D / 32; ++s) q[s] = qrow ? *reinterpret_cast<const u32x4_t*>(qrow + 64 * (s >> 1) + 16 * g + 8 * (s & 1)) : u32x4_t{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[i] = f32x4_t{0, 0, 0, 0};
        m = -__builtin_inff();
        z = 0.f;
    }
    // S^T of 64 tokens -> weights; p[u]: tokens 32 u + .. as the operand of the second product (its high parts, and what they lack)
    template <bool EXACT> __device__ __forceinline__ void weights(const f32x4_t (&s)[4], int first, int limit, bool masked, float c2, int lane, u32x4_t (&ph)[2], u32x4_t (&pl)[2])
    {
        float x[4][4];
        const int g = lane >> 4;
        float mx = -__builtin_inff();
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[t][r] = s[t][r] * c2;
                if (masked && first + 16 * t + 4 * g + r >= limit) x[t][r] = -__builtin_inff();
                mx = fmaxf(mx, x[t][r]);
            }
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float m_new = fmaxf(m, mx - kWeightBits);
        const float base = m_new == -__builtin_inff() ? 0.f : m_new;   // nothing seen yet: all weights are 2^-inf
        const float a = __builtin_amdgcn_exp2f(m - base);
        m = m_new;
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[t][r] = __builtin_amdgcn_exp2f(x[t][r] - base);
                sum += x[t][r];
            }
        z = fmaf(z, a, sum);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[i] *= a;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float p0 = x[2 * u + (k >> 1)][2 * (k & 1)], p1 = x[2 * u + (k >> 1)][2 * (k & 1) + 1];
                ph[u][k] = T::pack(p0, p1);
                if (EXACT) pl[u][k] = T::pack(p0 - T::lo(ph[u][k]), p1 - T::hi(ph[u][k]));
            }
    }
};

// One workgroup of four waves per (row tile, split): wave w takes every fourth block of the split, and the four states are put together
// through LDS.  EXACT: 32-bit results; the weights go into the second product as two 16-bit numbers each (their sum carries 16 bits or more
// where one carries 8 or 11, which is what a 16-bit result keeps).
template <class T, int D, bool EXACT>
__global__ __launch_bounds__(64 * kWaves) void rows_kernel(RowArgs a)
{
    __shared__ float o_s[kWaves][16][D + 4];
    __shared__ float m_s[kWaves][16], z_s[kWaves][16];
    const akb_cache& c = a.c;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int split = blockIdx.x % a.splits, group = blockIdx.x / a.splits, h = blockIdx.y, b = blockIdx.z;
    const int G = c.shape.Hq / c.shape.Hkv, n = a.n;
    const int len = seq_len(c, b), m = a.n_q ? min(max(a.n_q[b], 0), n) : n;
    const size_t bh = size_t(b) * c.shape.Hkv + h;
    const size_t item = bh * a.groups + group;
    const int row = group * 16 + (lane & 15);
    if (group * 16 >= m * G) return;   // no row of the tile is wanted
    const int last_row = min(group * 16 + 15, m * G - 1);
    const int keys = max(row_limit(last_row, G, m, len), 0), nb = (keys + kTB - 1) / kTB;
    const int all_see = row_limit(group * 16, G, m, len);        // tokens that every row of the tile sees
    const int limit = row_limit(row, G, m, len);
    const int lo = (int)(long(nb) * split / a.splits), hi = (int)(long(nb) * (split + 1) / a.splits);
    const int whole = min(hi, len / kTB);                         // blocks in 8 bits
    RowState<T, D> st;
    const int token = row / G, head = row % G;
    const size_t out_row = (bh * G + head) * n + token;
    st.init(row < m * G ? a.q + out_row * D : nullptr, lane);
    const size_t block0 = bh * (c.shape.Ncap / kTB);
    Codes<D> code;
    int blk = lo + wave;
    for (; blk < whole; blk += kWaves) {
        code.load(c, block0 + blk, lane);
        f32x4_t s[4] = {};
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < D / 64; ++i) {
                s[t] = T::mfma16(cvt8<T>(code.k[t][i][0], code.k[t][i][1], code.ks), st.q[2 * i], s[t]);
                s[t] = T::mfma16(cvt8<T>(code.k[t][i][2], code.k[t][i][3], code.ks), st.q[2 * i + 1], s[t]);
            }
        u32x4_t ph[2], pl[2];
        st.template weights<EXACT>(s, blk * kTB, limit, (blk + 1) * kTB > all_see, a.c2, lane, ph, pl);
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const u32x4_t v = cvt8<T>(code.v[i][2 * u], code.v[i][2 * u + 1], code.vs);
                st.o[i] = T::mfma16(v, ph[u], st.o[i]);
                if (EXACT) st.o[i] = T::mfma16(v, pl[u], st.o[i]);
            }
    }
    if (blk < hi) {   // the incomplete block, in 16 bits
        const uint16_t *kt = c.k_tail + bh * kTB * D, *vt = c.v_tail + bh * kTB * D;
        const int g = lane >> 4, left = len - blk * kTB;
        f32x4_t s[4] = {};
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int k = 0; k < D / 32; ++k)
                s[t] = T::mfma16(*reinterpret_cast<const u32x4_t*>(kt + (16 * t + (lane & 15)) * D + 64 * (k >> 1) + 16 * g + 8 * (k & 1)), st.q[k], s[t]);
        u32x4_t ph[2], pl[2];
        st.template weights<EXACT>(s, blk * kTB, min(limit, len), true, a.c2, lane, ph, pl);
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                u32x4_t v = *reinterpret_cast<const u32x4_t*>(vt + (16 * i + (lane & 15)) * kTB + 16 * g + 8 * u);
#pragma unroll
                for (int k = 0; k < 4; ++k) {   // what lies behind the length may be anything: zero, so that a weight of zero makes zero of it
                    const int t = 16 * (2 * u + (k >> 1)) + 4 * g + 2 * (k & 1);
                    v[k] = t + 1 < left ? v[k] : (t < left ? v[k] & 0xFFFFu : 0u);
                }
                st.o[i] = T::mfma16(v, ph[u], st.o[i]);
                if (EXACT) st.o[i] = T::mfma16(v, pl[u], st.o[i]);
            }
    }
    float z = st.z;
    z += __shfl_xor(z, 16);
    z += __shfl_xor(z, 32);
    if (lane < 16) {
        m_s[wave][lane] = st.m;
        z_s[wave][lane] = z;
    }
#pragma unroll
    for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4_t*>(&o_s[wave][lane & 15][16 * i + 4 * (lane >> 4)]) = st.o[i];
    __syncthreads();
    // four consecutive channels of one row per thread and turn
    for (int e = threadIdx.x; e < 16 * D / 4; e += 64 * kWaves) {
        const int r = e / (D / 4), d = e % (D / 4) * 4;
        float top = m_s[0][r];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, m_s[w][r]);
        const float base = top == -__builtin_inff() ? 0.f : top;
        f32x4_t o = {0, 0, 0, 0};
        float zz = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(m_s[w][r] - base);
            zz = fmaf(z_s[w][r], f, zz);
            o += *reinterpret_cast<const f32x4_t*>(&o_s[w][r][d]) * f;
        }
        if (a.splits > 1) {
            float* p = a.parts + (item * a.splits + split) * part_floats<D>();
            *reinterpret_cast<f32x4_t*>(p + r * D + d) = o;
            if (d == 0) {
                p[16 * D + 2 * r] = top;
                p[16 * D + 2 * r + 1] = zz;
            }
        } else if (group * 16 + r < m * G) {
            const float inv = zz > 0.f || zz != zz ? 1.f / zz : 0.f;
            o *= inv;
            const int rr = group * 16 + r;
            const size_t at = ((bh * G + rr % G) * n + rr / G) * D + d;
            if (a.out_dtype == 0) *reinterpret_cast<f32x4_t*>(static_cast<float*>(a.out) + at) = o;
            else *reinterpret_cast<u32x2_t*>(static_cast<uint16_t*>(a.out) + at) = u32x2_t{T::pack(o[0], o[1]), T::pack(o[2], o[3])};
            if (a.stats && d == 0) {
                a.stats[(item * 16 + r) * 2] = base;
                a.stats[(item * 16 + r) * 2 + 1] = inv;
            }
        }
    }
}

// The parts of a row tile put together: one workgroup per row tile.
template <class T, int D>
__global__ __launch_bounds__(256) void join_kernel(RowArgs a)
{
    const akb_cache& c = a.c;
    const int group = blockIdx.x, h = blockIdx.y, b = blockIdx.z, G = c.shape.Hq / c.shape.Hkv, n = a.n;
    const int m = a.n_q ? min(max(a.n_q[b], 0), n) : n;
    const size_t bh = size_t(b) * c.shape.Hkv + h, item = bh * a.groups + group;
    const float* parts = a.parts + item * a.splits * part_floats<D>();
    for (int e = threadIdx.x; e < 16 * D / 4; e += 256) {
        const int r = e / (D / 4), d = e % (D / 4) * 4, rr = group * 16 + r;
        if (rr >= m * G) continue;
        float top = -__builtin_inff();
        for (int s = 0; s < a.splits; ++s) top = fmaxf(top, parts[size_t(s) * part_floats<D>() + 16 * D + 2 * r]);
        const float base = top == -__builtin_inff() ? 0.f : top;
        f32x4_t o = {0, 0, 0, 0};
        float zz = 0.f;
        for (int s = 0; s < a.splits; ++s) {
            const float* p = parts + size_t(s) * part_floats<D>();
            const float f = __builtin_amdgcn_exp2f(p[16 * D + 2 * r] - base);
            zz = fmaf(p[16 * D + 2 * r + 1], f, zz);
            o += *reinterpret_cast<const f32x4_t*>(p + r * D + d) * f;
        }
        const float inv = zz > 0.f || zz != zz ? 1.f / zz : 0.f;
        o *= inv;
        const size_t at = ((bh * G + rr % G) * n + rr / G) * D + d;
        if (a.out_dtype == 0) *reinterpret_cast<f32x4_t*>(static_cast<float*>(a.out) + at) = o;
        else *reinterpret_cast<u32x2_t*>(static_cast<uint16_t*>(a.out) + at) = u32x2_t{T::pack(o[0], o[1]), T::pack(o[2], o[3])};
        if (a.stats && d == 0) {
            a.stats[(item * 16 + r) * 2] = base;
            a.stats[(item * 16 + r) * 2 + 1] = inv;
        }
    }
}

// score[t] += sum over the rows of exp2(x - maximum) / sum: the scores of a block of K once more, for all rows (the weights of a row are known
// only when its last token has been seen).  One workgroup per (block, KV head, sequence), wave w takes every fourth row tile.
template <class T, int D>
__global__ __launch_bounds__(64 * kWaves) void score_kernel(RowArgs a)
{
    __shared__ float sum_s[kWaves][kTB];
    const akb_cache& c = a.c;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4;
    const int h = blockIdx.y, b = blockIdx.z, G = c.shape.Hq / c.shape.Hkv, n = a.n;
    const int len = seq_len(c, b), m = a.n_q ? min(max(a.n_q[b], 0), n) : n;
    if (m == 0) return;
    const size_t bh = size_t(b) * c.shape.Hkv + h;
    for (int blk = blockIdx.x; blk * kTB < len; blk += gridDim.x) {
        u32x4_t k[4][D / 32];
        if (blk < len / kTB) {
            Codes<D> code;
            code.load(c, bh * (c.shape.Ncap / kTB) + blk, lane);
    #pragma unroll
            for (int t = 0; t < 4; ++t)
    #pragma unroll
                for (int i = 0; i < D / 64; ++i) {
                    k[t][2 * i] = cvt8<T>(code.k[t][i][0], code.k[t][i][1], code.ks);
                    k[t][2 * i + 1] = cvt8<T>(code.k[t][i][2], code.k[t][i][3], code.ks);
                }
        } else {
            const uint16_t* kt = c.k_tail + bh * kTB * D;
    #pragma unroll
            for (int t = 0; t < 4; ++t)
    #pragma unroll
                for (int i = 0; i < D / 32; ++i) k[t][i] = *reinterpret_cast<const u32x4_t*>(kt + (16 * t + (lane & 15)) * D + 64 * (i >> 1) + 16 * g + 8 * (i & 1));
        }
        f32x4_t acc[4] = {};
        const int tiles = (m * G + 15) / 16;
        for (int tile = wave; tile < tiles; tile += kWaves) {
            const int row = tile * 16 + (lane & 15);
            const int limit = min(row_limit(row, G, m, len), len);
            if (row_limit(min(tile * 16 + 15, m * G - 1), G, m, len) <= blk * kTB) continue;   // no row of the tile sees the block
            RowState<T, D> st;
            st.init(row < m * G ? a.q + ((bh * G + row % G) * n + row / G) * D : nullptr, lane);
            const float* p = a.stats + ((bh * a.groups + tile) * 16 + (lane & 15)) * 2;
            const float base = row < m * G ? p[0] : 0.f, inv = row < m * G ? p[1] : 0.f;
    #pragma unroll
            for (int t = 0; t < 4; ++t) {
                f32x4_t s = {0, 0, 0, 0};
    #pragma unroll
                for (int i = 0; i < D / 32; ++i) s = T::mfma16(k[t][i], st.q[i], s);
    #pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (blk * kTB + 16 * t + 4 * g + r < limit) acc[t][r] = fmaf(__builtin_amdgcn_exp2f(s[r] * a.c2 - base), inv, acc[t][r]);
            }
        }
    #pragma unroll
        for (int t = 0; t < 4; ++t)
    #pragma unroll
            for (int r = 0; r < 4; ++r) {
                float v = acc[t][r];
                v = akv::add_dpp<0xB1>(v);
                v = akv::add_dpp<0x4E>(v);
                v = akv::add_dpp<0x124>(v);
                v = akv::add_dpp<0x128>(v);
                if ((lane & 15) == 0) sum_s[wave][16 * t + 4 * g + r] = v;
            }
        __syncthreads();
        if (threadIdx.x < kTB && blk * kTB + int(threadIdx.x) < len) {
            float v = 0.f;
    #pragma unroll
            for (int w = 0; w < kWaves; ++w) v += sum_s[w][threadIdx.x];
            c.score[bh * c.shape.Ncap + blk * kTB + threadIdx.x] += v;
        }
        __syncthreads();   // sum_s is written again
    }
}

template <class T, int D> static hipError_t launch(const RowArgs& r, int max_len, hipStream_t st)
{
    const akb_shape& s = r.c.shape;
    const dim3 grid(r.groups * r.splits, s.Hkv, s.B);
    if (r.out_dtype == 0) hipLaunchKernelGGL((rows_kernel<T, D, true>), grid, dim3(64 * kWaves), 0, st, r);
    else hipLaunchKernelGGL((rows_kernel<T, D, false>), grid, dim3(64 * kWaves), 0, st, r);
    if (hipError_t e = hipGetLastError()) return e;
    if (r.splits > 1) {
        hipLaunchKernelGGL((join_kernel<T, D>), dim3(r.groups, s.Hkv, s.B), dim3(256), 0, st, r);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (r.stats) hipLaunchKernelGGL((score_kernel<T, D>), dim3((max_len + kTB - 1) / kTB, s.Hkv, s.B), dim3(64 * kWaves), 0, st, r);
    return hipGetLastError();
}

hipError_t launch_attention(const AttentionArgs& a, hipStream_t st)
{
    const AttentionPlan p = plan(a.c.shape, a.n, a.max_len, a.accumulate);
    RowArgs r{a.c, a.q, a.n_q, a.n, p.groups, p.splits, a.out_dtype, a.out, a.c2, reinterpret_cast<float*>(a.ws + p.parts),
              a.accumulate ? reinterpret_cast<float*>(a.ws + p.stats) : nullptr};
    if (a.c.shape.dtype == AKB_FP16) return a.c.shape.D == 64 ? launch<Fp16, 64>(r, a.max_len, st) : launch<Fp16, 128>(r, a.max_len, st);
    return a.c.shape.D == 64 ? launch<Bf16, 64>(r, a.max_len, st) : launch<Bf16, 128>(r, a.max_len, st);
}

}  // namespace akb
