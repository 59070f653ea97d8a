// Attention of many query rows over the block-scaled 8-bit cache (rules and layout: include/akb.h; rows and parts: akb_rows.h).
//
// With many rows the products are what takes time, and turning codes into 16-bit numbers the next: a wave that does it for its own rows alone (the rows kernel)
// spends more on that than on its softmax.  Here the four waves of a workgroup have 32 rows each and share every block: it is turned once, into LDS, in the order
// in which 32 x 32 x 16 matrix instructions take their operands (1 KB per operand, lane after lane), while the block before is multiplied.
// Per block and wave: 32 matrix instructions of 32 cycles for K and V together (with 32-bit results 48 in binary16, 64 in bfloat16), 32 reads of 1 KB from LDS, and the softmax of 64 x 32 scores,
// 32 per lane, beside the scores of the next block.  Two workgroups of 64 KB share a compute unit.
// A prompt of 8192 tokens, 32 query heads on 8, bfloat16: 541 us, 1016 TFLOP/s of the products that are wanted (a plain product of 8192 x 8192 matrices reaches 1207
// here); the clock is at 1.9 GHz then.
#include "akb_rows.h"

namespace akb {

constexpr int kWaveRows = kPromptRows / kWaves;

// lane l has row l % 32; of a tile of 32 tokens (channels) it has 8 i + 4 (l / 32) .. + 3, i = 0 .. 3, in order
template <int D> struct KLds { u32x4_t x[2][D / 16][64]; };   // [32 tokens][16 channels]: lane (token % 32, half): channels 8 half .. + 7
template <int D> struct VLds { u32x4_t x[D / 32][4][64]; };   // [32 channels][16 tokens]: lane (channel % 32, half): tokens 4 half .. + 3, 8 + 4 half .. + 3

// One side of a block on its way from memory to LDS: wave w has pieces w, w + 4, .. of 1 KB of codes (K's [tile][64 channels], V's [16 channels]), a lane 16 of them
template <class T, int D> struct Stage {
    static constexpr int kPieces = D / 64;   // per wave
    u32x4_t w[kPieces];
    int e;
    __device__ __forceinline__ void load(const uint8_t* plane, const int8_t* exps, size_t block, int wave, int lane)
    {
        const uint8_t* p = plane + block * (kTB * D) + wave * 1024 + (lane & 15) * 64 + (lane >> 4) * 16;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) w[i] = *reinterpret_cast<const u32x4_t*>(p + kWaves * i * 1024);
        e = exps[block * 2];
    }
    __device__ __forceinline__ void store(KLds<D>& to, int wave, int lane) const
    {
        const float s = pow2(e);
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int piece = wave + kWaves * i, token = piece / (D / 64) * 16 + (lane & 15), ch16 = piece % (D / 64) * 4 + (lane >> 4);
            to.x[token >> 5][ch16][token & 31] = cvt8<T>(w[i][0], w[i][1], s);
            to.x[token >> 5][ch16][32 + (token & 31)] = cvt8<T>(w[i][2], w[i][3], s);
        }
    }
    __device__ __forceinline__ void store(VLds<D>& to, int wave, int lane) const   // tokens 16 t + 4 g .. + 3 of a channel, t = 0 .. 3
    {
        const float s = pow2(e);
        const int g = lane >> 4;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int ch = (wave + kWaves * i) * 16 + (lane & 15);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                reinterpret_cast<u32x2_t*>(&to.x[ch >> 5][t][(ch & 31) + 32 * (g & 1)])[g >> 1] = u32x2_t{T::template cvt2<false>(w[i][t], s), T::template cvt2<true>(w[i][t], s)};
        }
    }
    // the incomplete block of `left` tokens, in 16 bits; what lies behind is zero
    __device__ __forceinline__ static void store_tail(const uint16_t* tail, int left, KLds<D>& to, int tid)
    {
        for (int e = tid; e < kTB * (D / 8); e += 64 * kWaves) {   // 8 channels of a token
            const int token = e % kTB, oct = e / kTB;
            to.x[token >> 5][oct >> 1][(token & 31) + 32 * (oct & 1)] = token < left ? *reinterpret_cast<const u32x4_t*>(tail + token * D + oct * 8) : u32x4_t{0, 0, 0, 0};
        }
    }
    __device__ __forceinline__ static void store_tail(const uint16_t* tail, int left, VLds<D>& to, int tid)
    {
        for (int e = tid; e < D * 16; e += 64 * kWaves) {          // tokens 16 t + 4 g .. + 3 of a channel
            const int ch = e % D, t = (e / D) & 3, g = e / D / 4, token = 16 * t + 4 * g;
            u32x2_t w = {0, 0};
            if (token < left) {
                w = *reinterpret_cast<const u32x2_t*>(tail + ch * kTB + 16 * g + 4 * t);
#pragma unroll
                for (int k = 0; k < 2; ++k) w[k] = token + 2 * k + 1 < left ? w[k] : (token + 2 * k < left ? w[k] & 0xFFFFu : 0u);
            }
            reinterpret_cast<u32x2_t*>(&to.x[ch >> 5][t][(ch & 31) + 32 * (g & 1)])[g >> 1] = w;
        }
    }
    // whether the incomplete block's V has large values (in this thread's share of it)
    __device__ __forceinline__ static bool large_tail(const uint16_t* tail, int left, int tid)
    {
        uint32_t large = 0;
#pragma unroll
        for (int p = tid; p < D * 8; p += 64 * kWaves) {           // tokens 32 (p % 2) + 4 g .. + 3 and 16 further of a channel, g = p / 2 % 4
            const u32x4_t w = *reinterpret_cast<const u32x4_t*>(tail + p * 8);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int token = 32 * (p & 1) + 16 * (e >> 1) + 4 * (p >> 1 & 3) + 2 * (e & 1);
                large |= large_values(w[e] & (token + 1 < left ? 0xFFFFFFFFu : (token < left ? 0xFFFFu : 0u)));
            }
        }
        return large & kLargeValues;
    }
};

template <class T, int D, bool EXACT>
__global__ __launch_bounds__(64 * kWaves, 2) void prompt_kernel(RowArgs a)
{
    __shared__ KLds<D> k_s[2];
    __shared__ VLds<D> v_s[2];
    __shared__ bool large_s[kWaves];
    const akb_cache& c = a.c;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    Cut cut;
    if (!cut.find<false>(a, 0)) return;
    const int splits = cut.splits, split = (cut.w - cut.first) % splits, walk = (cut.w - cut.first) / splits;
    const int group = a.groups - 1 - walk % a.groups;   // the rows that see most go first
    const int b = cut.b, G = c.shape.Hq / c.shape.Hkv, n = a.n;
    const size_t bh = size_t(b) * c.shape.Hkv + walk / a.groups;
    const int len = seq_len(c, b), m = a.n_q ? min(max(a.n_q[b], 0), n) : n;
    const int row0 = group * kPromptRows, rows = min(kPromptRows, m * G - row0);
    if (rows <= 0) return;
    const int nb = (max(row_limit(a, row0 + rows - 1, G, m, len), 0) + kTB - 1) / kTB;
    const int lo = (int)(long(nb) * split / splits), hi = (int)(long(nb) * (split + 1) / splits);
    const int first_row = row0 + wave * kWaveRows, row = first_row + (lane & 31);
    const int wave_rows = min(kWaveRows, row0 + rows - first_row);   // may be below 1: the wave only helps to turn blocks
    const int all_see = row_limit(a, first_row, G, m, len), most_see = wave_rows > 0 ? row_limit(a, first_row + wave_rows - 1, G, m, len) : 0;
    const int limit = row_limit(a, row, G, m, len);
    auto place = [&](int row) { return row_place(a, bh, G, row, D); };   // of a row in q and out
    u32x4_t q[D / 16];
#pragma unroll
    for (int i = 0; i < D / 16; ++i) q[i] = row < m * G ? *reinterpret_cast<const u32x4_t*>(a.q + place(row) + 16 * i + 8 * half) : u32x4_t{0, 0, 0, 0};
    f32x16_t o[D / 32];
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
    float top = -__builtin_inff(), z = 0.f;

    const size_t block0 = bh * (c.shape.Ncap / kTB);
    const int whole = len / kTB;   // blocks in 8 bits
    const uint16_t *k_tail = c.k_tail + bh * kTB * D, *v_tail = c.v_tail + bh * kTB * D;
    Stage<T, D> ks, vs;
    auto fetch_k = [&](int blk) { if (blk < min(hi, whole)) ks.load(c.k8, c.exps, block0 + blk, wave, lane); };
    auto fetch_v = [&](int blk) { if (blk < min(hi, whole)) vs.load(c.v8, c.exps + 1, block0 + blk, wave, lane); };
    auto put_k = [&](int blk, KLds<D>& to) {
        if (blk < min(hi, whole)) ks.store(to, wave, lane);
        else if (blk < hi) Stage<T, D>::store_tail(k_tail, len - blk * kTB, to, threadIdx.x);
    };
    auto put_v = [&](int blk, VLds<D>& to) {
        if (blk < min(hi, whole)) vs.store(to, wave, lane);
        else if (blk < hi) Stage<T, D>::store_tail(v_tail, len - blk * kTB, to, threadIdx.x);
    };
    // steps 2 j, 2 j + 1 of the first product of the block in `k`
    auto product = [&](f32x16_t (&s)[2], const KLds<D>& k, int j) {
#pragma unroll
        for (int i = j * (D / 64); i < (j + 1) * (D / 64); ++i)
#pragma unroll
            for (int t = 0; t < 2; ++t) s[t] = T::mfma32(k.x[t][i][lane], q[i], s[t]);
    };
    auto clear = [](f32x16_t (&s)[2]) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[t][r] = 0.f;
    };
    f32x16_t sa[2], sb[2];
    fetch_k(lo);
    fetch_v(lo);
    put_k(lo, k_s[0]);
    fetch_k(lo + 1);
    float unit = kWeightBits;
    if (T::kWide) {   // one unit for the walk: found out here, it costs the loop a scalar register (followed from block to block, 560 us of the prompt above for 541)
        bool some = hi > whole && Stage<T, D>::large_tail(v_tail, len - whole * kTB, threadIdx.x);
        for (int blk = lo + int(threadIdx.x); blk < min(hi, whole); blk += 64 * kWaves) some |= c.exps[(block0 + blk) * 2 + 1] >= kLargeExp;
        some = __any(some);
        if (lane == 0) large_s[wave] = some;
        lds_barrier();
        unit = weight_bits<T>(__builtin_amdgcn_readfirstlane(large_s[0] | large_s[1] | large_s[2] | large_s[3]));
    }
    put_v(lo, v_s[0]);
    put_k(lo + 1, k_s[1]);
    lds_barrier();
    clear(sa);
#pragma unroll
    for (int j = 0; j < 4; ++j) product(sa, k_s[0], j);
    // Block blk: its scores are in s; those of the next are made (`next`, from k_next) while these become weights, so that a wave's products and its softmax are
    // beside each other.  Behind that K of the block after the next goes to where K of this one was, V of the next to where V of the one before was.
    auto step = [&](int blk, f32x16_t (&s)[2], f32x16_t (&next)[2], KLds<D>& k_this, const KLds<D>& k_next, const VLds<D>& v, VLds<D>& v_next) {
        lds_barrier();   // the next K and this V are there, and nobody reads what is written below any more
        fetch_k(blk + 2);
        fetch_v(blk + 1);
        if (blk * kTB < most_see) {   // some row of the wave sees it
            if ((blk + 1) * kTB > all_see) {
                const int seen = limit - blk * kTB - 4 * half;   // counted from the lane's first token
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (32 * t + 8 * (r >> 2) + (r & 3) >= seen) s[t][r] = -__builtin_inff();
            }
            float mx = -__builtin_inff();
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[t][r]);
            mx = max_lane32(mx);
            const float now = fmaf(mx, a.c2, -unit);
            if (__any(now > top + kSlackBits)) {
                const float up = fmaxf(top, now), f = __builtin_amdgcn_exp2f(top - (up == -__builtin_inff() ? 0.f : up));
                z *= f;
#pragma unroll
                for (int i = 0; i < D / 32; ++i) o[i] *= f;
                top = up;
            }
            const float base = top == -__builtin_inff() ? 0.f : top;   // nothing seen yet: all weights are 2^-inf
            clear(next);
            u32x4_t ph[2], pl[2], pr[2];
#pragma unroll
            for (int t = 0; t < 5; ++t) {   // 16 tokens: weights of t, products of t - 1
                if (t < 4) {
                    product(next, k_next, t);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int r = 8 * (t & 1) + 2 * k;
                        const float p0 = __builtin_amdgcn_exp2f(fmaf(s[t >> 1][r], a.c2, -base)), p1 = __builtin_amdgcn_exp2f(fmaf(s[t >> 1][r + 1], a.c2, -base));
                        z += p0 + p1;
                        ph[t & 1][k] = T::pack(p0, p1);
                        if (!EXACT) continue;
                        const float l0 = p0 - T::lo(ph[t & 1][k]), l1 = p1 - T::hi(ph[t & 1][k]);
                        pl[t & 1][k] = T::pack(l0, l1);
                        if (T::kWide) pr[t & 1][k] = T::pack(l0 - T::lo(pl[t & 1][k]), l1 - T::hi(pl[t & 1][k]));
                    }
                }
                if (t > 0) {
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) {
                        const u32x4_t x = v.x[i][t - 1][lane];
                        o[i] = T::mfma32(x, ph[(t - 1) & 1], o[i]);
                        if (EXACT) o[i] = T::mfma32(x, pl[(t - 1) & 1], o[i]);
                        if (EXACT && T::kWide) o[i] = T::mfma32(x, pr[(t - 1) & 1], o[i]);
                    }
                }
                // the order that the compiler keeps of its own accord has the products in a row; with two products per weight it has too few registers to choose
                if (EXACT) {
                    __builtin_amdgcn_sched_barrier(0);
                } else {
                    __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);       // reads from LDS
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);   // vector instructions
                        __builtin_amdgcn_sched_group_barrier(0x400, 1, 0);   // an exponential
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);   // a matrix instruction
                    }
                }
            }
        }
        put_k(blk + 2, k_this);
        put_v(blk + 1, v_next);
    };
    for (int blk = lo; blk < hi; blk += 2) {   // (in pairs: which half of LDS is which is known to the compiler)
        step(blk, sa, sb, k_s[0], k_s[1], v_s[0], v_s[1]);
        if (blk + 1 < hi) step(blk + 1, sb, sa, k_s[1], k_s[0], v_s[1], v_s[0]);
    }
    if (wave_rows <= 0 || (lane & 31) >= wave_rows) return;
    z = akv::add_lane32(z);
    const int r = row - row0;
    Joined j;
    j.top = top;
    j.z = z;
    float* part = a.parts + size_t(cut.w - split) * part_floats(min(n * G, kPromptRows), D) + size_t(split) * part_floats(rows, D);
    if (splits > 1 && half == 0) {
        part[2 * r] = top;
        part[2 * r + 1] = z;
    }
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int d = 32 * i + 8 * k + 4 * half;
            j.o = f32x4_t{o[i][4 * k], o[i][4 * k + 1], o[i][4 * k + 2], o[i][4 * k + 3]};
            if (splits == 1) j.template finish<T>(a, bh * n * G, row, place(row), d);
            else *reinterpret_cast<f32x4_t*>(part + part_head(rows) + r * D + d) = j.o;
        }
}

template <class T, int D> static void launch(const RowArgs& r, int grid, hipStream_t st)
{
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(akv::xcd_grid(grid)), dim3(64 * kWaves), 0, st, r); };
    r.out_dtype == 0 ? go(prompt_kernel<T, D, true>) : go(prompt_kernel<T, D, false>);
}
hipError_t launch_prompt(const RowArgs& r, int grid, hipStream_t st)
{
    if (r.c.shape.dtype == AKB_FP16) r.c.shape.D == 64 ? launch<Fp16, 64>(r, grid, st) : launch<Fp16, 128>(r, grid, st);
    else r.c.shape.D == 64 ? launch<Bf16, 64>(r, grid, st) : launch<Bf16, 128>(r, grid, st);
    return hipGetLastError();
}

}  // namespace akb
