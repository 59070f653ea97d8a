// Eviction from the block-scaled 8-bit cache by accumulated attention weight (rules and layout: include/akb.h).
#include "akb_pack.h"

namespace akb {

constexpr int kSelThreads = 1024;
constexpr int kBins = 2048;
constexpr int kCopies = 4;   // of the counts: many scores are alike, and counts of one value in one place are taken one after the other
constexpr int kPer = 8;      // neighbouring scores per thread and turn
constexpr int kTurns = 4;    // turns whose scores are asked for together

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

// The scores of the first n tokens in turns of kPer neighbouring ones per thread, kTurns turns asked for together (a workgroup is alone with its head, and
// a trip to memory per turn is what it would wait for): f(turn's first token of this thread, its keys), every thread takes every turn
template <class F> __device__ __forceinline__ void for_scores(const float* score, int n, F f)
{
    for (int base = 0; base < n; base += kTurns * kPer * kSelThreads) {
        f32x4_t v[kTurns][kPer / 4];
#pragma unroll
        for (int k = 0; k < kTurns; ++k)
#pragma unroll
            for (int i = 0; i < kPer / 4; ++i) {   // rows are whole blocks long: a piece that begins below n can be read
                const int t = base + (k * kSelThreads + int(threadIdx.x)) * kPer + 4 * i;
                v[k][i] = t < n ? *reinterpret_cast<const f32x4_t*>(score + t) : f32x4_t{0, 0, 0, 0};
            }
#pragma unroll
        for (int k = 0; k < kTurns; ++k) {
            if (base + k * kSelThreads * kPer >= n) break;
            uint32_t key[kPer];
#pragma unroll
            for (int i = 0; i < kPer; ++i) key[i] = order_key(v[k][i >> 2][i & 3]);
            f(base + (k * kSelThreads + int(threadIdx.x)) * kPer, key);
        }
    }
}

// Which tokens of a (sequence, KV head) stay: one workgroup each.  The place among the sorted scores is found 11, 11 and 10 bits at a
// time (counts of each value of the bits among the scores that agree in the bits above), then one pass writes the kept tokens' places in
// their order: those above the threshold, of those at it the first.
__global__ __launch_bounds__(kSelThreads) void select_kernel(akb_cache c, akb_cache d, int keep, int recent, int32_t* __restrict__ kept)
{
    __shared__ int hist[kCopies * kBins];
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
            for (int i = tid; i < kCopies * kBins; i += kSelThreads) hist[i] = 0;
            __syncthreads();
            int* mine = hist + (tid % kCopies) * kBins;
            for_scores(score, pool, [&](int t0, const uint32_t (&key)[kPer]) {
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (t0 + i < pool && (pass == 0 || (key[i] >> (shift + bits)) == prefix)) atomicAdd(&mine[(key[i] >> shift) & ((1u << bits) - 1)], 1);
            });
            __syncthreads();
            // from the largest value down: thread i has values 2 i, 2 i + 1 counted from the top
            const int top = kBins - 1 - 2 * tid;
            int h0 = 0, h1 = 0;
#pragma unroll
            for (int k = 0; k < kCopies; ++k) {
                h0 += hist[k * kBins + top];
                h1 += hist[k * kBins + top - 1];
            }
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
    int32_t* out = kept + bh * keep;
    if (count - sure >= pool) {           // all stay
        for (int t = tid; t < count; t += kSelThreads) out[t] = t;
    } else {
        // written so far, and tokens at the threshold passed so far; a thread has kPer neighbouring tokens and counts those above the threshold
        // (low half of the word that is summed up over the workgroup) and those at it (high half)
        int above = 0, ties = 0;
        for_scores(score, count > sure ? pool : 0, [&](int t0, const uint32_t (&key)[kPer]) {
            int mine = 0;
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (t0 + i < pool) mine += key[i] > prefix ? 1 : (key[i] == prefix ? 1 << 16 : 0);
            int all;
            const int upto = block_scan(mine, wave_s, &all) - mine;
            int a = above + (upto & 0xFFFF), e = ties + (upto >> 16);
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                if (t0 + i >= pool) continue;
                if (key[i] > prefix || (key[i] == prefix && e < need)) out[a + min(e, need)] = t0 + i;
                a += key[i] > prefix ? 1 : 0;
                e += key[i] == prefix ? 1 : 0;
            }
            above += all & 0xFFFF;
            ties += all >> 16;
        });
        for (int i = tid; i < sure; i += kSelThreads) out[count - sure + i] = len - sure + i;
    }
    for (int i = count + tid; i < keep; i += kSelThreads) out[i] = -1;
    if (h == 0 && tid == 0) d.lens[b] = count;
}

// The same for few heads with long rows, where one workgroup per head would leave most of the device idle: a workgroup per 8192 scores, and a launch per step, since
// every step needs the counts of all of a head's workgroups.  Steps 0 to 2 count 11, 11 and 10 bits (integers: their order does not matter), 3 counts the tokens
// above the threshold and at it per workgroup, 4 writes the places.
constexpr int kChunk = kSelThreads * kPer;
struct SelectWs {
    int32_t* hist;    // [3][pairs][kBins]
    int32_t* state;   // [3][pairs][2]: bits of the threshold so far, tokens still needed
    int32_t* counts;  // [pairs][chunks][2]
};
template <int STEP>
__global__ __launch_bounds__(kSelThreads) void select_step_kernel(akb_cache c, akb_cache d, int keep, int recent, int32_t* __restrict__ kept, SelectWs ws)
{
    __shared__ int hist_s[STEP < 3 ? kCopies * kBins : 1];
    __shared__ int wave_s[kSelThreads / 64];
    __shared__ int found_s[2];
    const int chunk = blockIdx.x, h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
    const size_t pairs = size_t(c.shape.B) * c.shape.Hkv, bh = size_t(b) * c.shape.Hkv + h;
    const int len = seq_len(c, b), count = min(len, keep), sure = min(recent, count), pool = len - sure;
    const int want = count - sure;
    const bool choose = want > 0 && want < pool;
    int32_t* out = kept + bh * keep;
    if (STEP == 4 && chunk == 0) {
        for (int i = tid; i < sure; i += kSelThreads) out[want + i] = len - sure + i;
        for (int i = count + tid; i < keep; i += kSelThreads) out[i] = -1;
        if (h == 0 && tid == 0) d.lens[b] = count;
    }
    if (chunk * kChunk >= pool || want <= 0) return;
    const int t0 = chunk * kChunk + tid * kPer;
    if (!choose) {   // all stay
        if (STEP == 4)
            for (int i = 0; i < kPer; ++i)
                if (t0 + i < pool) out[t0 + i] = t0 + i;
        return;
    }
    uint32_t key[kPer];
    {
        const float* score = c.score + bh * c.shape.Ncap;
        f32x4_t v[kPer / 4];
#pragma unroll
        for (int i = 0; i < kPer / 4; ++i) v[i] = t0 + 4 * i < pool ? *reinterpret_cast<const f32x4_t*>(score + t0 + 4 * i) : f32x4_t{0, 0, 0, 0};   // rows are whole blocks long
#pragma unroll
        for (int i = 0; i < kPer; ++i) key[i] = order_key(v[i >> 2][i & 3]);
    }
    uint32_t prefix = 0;
    int need = want;
    if (STEP > 0) {   // what the step before has counted: the value of its bits that the threshold has
        const int at = min(STEP, 3) - 1, bits = at == 2 ? 10 : 11;
        const int32_t* state = ws.state + (size_t(at) * pairs + bh) * 2;
        if (STEP == 4) {
            prefix = state[0];
            need = state[1];
        } else {
            if (at > 0) {
                prefix = state[-2 * int(pairs)];
                need = state[1 - 2 * int(pairs)];
            }
            const int32_t* hist = ws.hist + (size_t(at) * pairs + bh) * kBins;
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
            if (chunk == 0 && tid == 0) {
                int32_t* mine = ws.state + (size_t(at) * pairs + bh) * 2;
                mine[0] = int32_t(prefix);
                mine[1] = need;
            }
        }
    }
    if constexpr (STEP < 3) {
        const int shift = STEP == 0 ? 21 : (STEP == 1 ? 10 : 0), bits = STEP == 2 ? 10 : 11;
        for (int i = tid; i < kCopies * kBins; i += kSelThreads) hist_s[i] = 0;
        __syncthreads();
        int* mine = hist_s + (tid % kCopies) * kBins;
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (t0 + i < pool && (STEP == 0 || (key[i] >> (shift + bits)) == prefix)) atomicAdd(&mine[(key[i] >> shift) & ((1u << bits) - 1)], 1);
        __syncthreads();
        int32_t* hist = ws.hist + (size_t(STEP) * pairs + bh) * kBins;
        for (int i = tid; i < kBins; i += kSelThreads) {
            int sum = 0;
#pragma unroll
            for (int k = 0; k < kCopies; ++k) sum += hist_s[k * kBins + i];
            if (sum) atomicAdd(hist + i, sum);
        }
    } else {
        int mine = 0;   // above the threshold in the low half, at it in the high half
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (t0 + i < pool) mine += key[i] > prefix ? 1 : (key[i] == prefix ? 1 << 16 : 0);
        int all;
        const int upto = block_scan(mine, wave_s, &all) - mine;
        int32_t* counts = ws.counts + bh * gridDim.x * 2;
        if constexpr (STEP == 3) {
            if (tid == 0) {
                counts[2 * chunk] = all & 0xFFFF;
                counts[2 * chunk + 1] = all >> 16;
            }
        } else {
            int above = 0, ties = 0;   // of the chunks before
            for (int i = 0; i < chunk; ++i) {
                above += counts[2 * i];
                ties += counts[2 * i + 1];
            }
            int a = above + (upto & 0xFFFF), e = ties + (upto >> 16);
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                if (t0 + i >= pool) continue;
                if (key[i] > prefix || (key[i] == prefix && e < need)) out[a + min(e, need)] = t0 + i;
                a += key[i] > prefix ? 1 : 0;
                e += key[i] == prefix ? 1 : 0;
            }
        }
    }
}

// A block of the destination: one workgroup of 2 D threads per (block, side, KV head, sequence), as in the append.  K: a token's codes are runs of 64
// bytes, read where they lie.  V: a token is one byte in each channel's 64 (byte loads, a wave's touching 64 lines each, took four times as long), so the source
// blocks that hold a kept token are read whole, one after the other, into LDS (rows padded to 17 dwords, so that a token's bytes lie in different banks), and
// the kept tokens' bytes go token-major to where the threads take them from.  Bound by memory: V is read whole unless no token of a block stays, and
// of K 128 bytes for each run of 64: 268 + 134 + 33 (scores) MB in and 138 out for 8 x 32 heads 8192 -> 2048 tokens, 99 us.
template <class T, int D>
__global__ __launch_bounds__(2 * D) void gather_kernel(akb_cache c, akb_cache d, int keep, const int32_t* __restrict__ kept)
{
    constexpr int kStride = PackLds<D>::kStride, kRow = D + 8;   // bytes of a token's row: shifted by two dwords from token to token
    __shared__ PackLds<D> lds;   // the source block in its place, before the block is packed
    __shared__ __align__(16) uint8_t rows_s[kTB * kRow];
    __shared__ int from_s[kTB];
    __shared__ float scale_s[kTB];
    const int tid = threadIdx.x, lane = tid & 63, h = blockIdx.y, b = blockIdx.z, blk = blockIdx.x >> 1;
    const bool is_v = blockIdx.x & 1;
    const size_t bh = size_t(b) * c.shape.Hkv + h, block0 = bh * (c.shape.Ncap / kTB);
    const int len = seq_len(c, b), count = min(len, keep), whole = len / kTB;
    if (blk * kTB >= count) return;
    if (tid < kTB) {
        const int i = blk * kTB + tid, t = i < count ? kept[bh * keep + i] : -1;
        from_s[tid] = t;
        scale_s[tid] = t >= 0 && t / kTB < whole ? pow2(c.exps[(block0 + t / kTB) * 2 + (is_v ? 1 : 0)]) : 0.f;
        if (!is_v && d.score && t >= 0) d.score[bh * d.shape.Ncap + i] = c.score[bh * c.shape.Ncap + t];
    }
    __syncthreads();
    const BlockLane<D> at(tid);
    u32x4_t x[4] = {};
    int token[4];
    bool in_tail[4], stays[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int t = from_s[at.t0 + r];
        stays[r] = t >= 0;
        in_tail[r] = stays[r] && t / kTB >= whole;
        token[r] = t;
    }
    if (!is_v) {
        u32x2_t w[4] = {};
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (stays[r] && !in_tail[r]) w[r] = *reinterpret_cast<const u32x2_t*>(c.k8 + (block0 + token[r] / kTB) * (kTB * D) + k_place<D>(token[r] % kTB, at.oct * 8));
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = cvt8<T>(w[r][0], w[r][1], scale_s[at.t0 + r]);
    } else {
        // lane i of every wave: source block of token i; `starts`: the first token of each source block
        const int t = from_s[lane], src = t >= 0 && t / kTB < whole ? t / kTB : -1;
        const int place = v_place(max(t, 0) % kTB), before = __shfl_up(src, 1);
        const int half = __builtin_amdgcn_readfirstlane(tid / D);   // which of two neighbouring tokens the wave moves
        uint64_t starts = __ballot(src >= 0 && (lane == 0 || before != src));
        const int used = __popcll(__ballot(src >= 0));   // tokens of whole blocks: the first ones, as the places ascend
        u32x4_t piece[2];
        auto fetch = [&](int first) {
            const uint8_t* p = c.v8 + (block0 + __builtin_amdgcn_readlane(src, first)) * (kTB * D) + tid * 16;
            piece[0] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
            piece[1] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p + 2 * D * 16));
        };
        if (starts) fetch(0);
        while (starts) {
            const int first = __builtin_ctzll(starts);
            starts &= starts - 1;
            const int end = starts ? __builtin_ctzll(starts) : used;
            lds_barrier();   // the block before has been read
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) lds.codes[((tid + k * 2 * D) >> 2) * kStride + (tid & 3) * 4 + i] = piece[k][i];
            if (starts) fetch(end);
            lds_barrier();
            const uint8_t* raw = reinterpret_cast<const uint8_t*>(lds.codes) + (tid % D) * (4 * kStride);
            for (int i = first + half; i < end; i += 8) {   // four of the wave's tokens at a time
                uint8_t code[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) code[k] = raw[__builtin_amdgcn_readlane(place, min(i + 2 * k, end - 1))];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (i + 2 * k < end) rows_s[(i + 2 * k) * kRow + tid % D] = code[k];
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (stays[r] && !in_tail[r]) {
                const u32x2_t w = *reinterpret_cast<const u32x2_t*>(rows_s + (at.t0 + r) * kRow + at.oct * 8);
                x[r] = cvt8<T>(w[0], w[1], scale_s[at.t0 + r]);
            }
    }
    if (in_tail[0] || in_tail[1] || in_tail[2] || in_tail[3]) {
        int slot[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) slot[r] = token[r] % kTB;
        load_tail<D, false>(c, bh, is_v, x, in_tail, slot);
    }
    // codes stored with the hint: 8 x 32 heads 8192 -> 2048 tokens 126 / 110 us, and with the step that follows 138.6 / 136.8; fewer alike
    if ((blk + 1) * kTB <= count) pack_block<T, D, true>(d, bh * (d.shape.Ncap / kTB) + blk, is_v, x, lds);
    else store_tail<D>(d, bh, is_v, x, stays);
}

// Workgroups per head where the heads are few and their rows long.  One workgroup per head / a launch per step, us: 8 heads 131001 -> 16384
// tokens 124.6 / 75.8 with the gather, 32 of 65536 -> 4096 125 / 110, 8 of 32768 38.1 / 37.3; 32 of 16384 41.8 / 48.8, 128 of 40000 171 / 182, 256 of 32768 270 / 299.
static int chunks_of(const akb_shape& s)
{
    const int chunks = (s.Ncap + kChunk - 1) / kChunk;
    return long(s.B) * s.Hkv <= 64 && chunks > 4 ? chunks : 1;
}
static size_t kept_bytes(const akb_shape& s, int keep) { return align256(size_t(s.B) * s.Hkv * size_t(keep) * sizeof(int32_t)); }
size_t evict_workspace(const akb_shape& s, int keep)
{
    const int chunks = chunks_of(s);
    return kept_bytes(s, keep) + (chunks > 1 ? align256(size_t(s.B) * s.Hkv * (3 * (kBins + 2) + 2 * size_t(chunks)) * sizeof(int32_t)) : 0);
}

hipError_t launch_evict(const akb_cache& src, const akb_cache& dst, int keep, int recent, int32_t* kept, char* ws, hipStream_t st)
{
    const akb_shape& s = src.shape;
    const int chunks = chunks_of(s);
    if (!kept) kept = reinterpret_cast<int32_t*>(ws);
    if (chunks == 1) {
        hipLaunchKernelGGL(select_kernel, dim3(s.Hkv, s.B), dim3(kSelThreads), 0, st, src, dst, keep, recent, kept);
    } else {
        const size_t pairs = size_t(s.B) * s.Hkv;
        SelectWs w;
        w.hist = reinterpret_cast<int32_t*>(ws + kept_bytes(s, keep));
        w.state = w.hist + 3 * pairs * kBins;
        w.counts = w.state + 3 * pairs * 2;
        if (hipError_t e = akv::launch_zero(w.hist, 3 * pairs * kBins * sizeof(int32_t), st)) return e;
        auto step = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(chunks, s.Hkv, s.B), dim3(kSelThreads), 0, st, src, dst, keep, recent, kept, w); };
        step(select_step_kernel<0>);
        step(select_step_kernel<1>);
        step(select_step_kernel<2>);
        step(select_step_kernel<3>);
        step(select_step_kernel<4>);
    }
    if (hipError_t e = hipGetLastError()) return e;
    const int blocks = (std::min(keep, s.Ncap) + kTB - 1) / kTB;
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(2 * blocks, s.Hkv, s.B), dim3(2 * s.D), 0, st, src, dst, keep, kept); };
    if (s.dtype == AKB_FP16) s.D == 64 ? launch(gather_kernel<Fp16, 64>) : launch(gather_kernel<Fp16, 128>);
    else s.D == 64 ? launch(gather_kernel<Bf16, 64>) : launch(gather_kernel<Bf16, 128>);
    return hipGetLastError();
}

}  // namespace akb
