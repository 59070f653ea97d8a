// Attention of many query rows over the block-scaled 8-bit cache (rules and layout: include/akb.h; rows and parts: akb_rows.h).
//
// With many rows the products are what takes time, and turning codes into 16-bit numbers the next: a wave that does it for its own rows alone (the rows kernel)
// spends more on that than on its softmax.  Here the four waves of a workgroup have 32 rows each and share every block: it is turned once, into LDS, in the order
// in which 32 x 32 x 16 matrix instructions take their operands (1 KB per operand, lane after lane), while the block before is multiplied.
// Per block and wave: 32 matrix instructions of 32 cycles for K and V together (with 32-bit results 48 in binary16, 64 in bfloat16), 32 reads of 1 KB from LDS, and the softmax of 64 x 32 scores,
// 32 per lane, beside the scores of the next block.  Two workgroups of 64 KB share a compute unit.
// A prompt of 8192 tokens, 32 query heads on 8, bfloat16: 541 us, 1016 TFLOP/s of the products that are wanted (a plain product of 8192 x 8192 matrices reaches 1207
// here); the clock is at 1.9 GHz then.
#include "akb_prompt_walk.h"

namespace akb {

// Args: RowArgs, or SharedArgs, where a walk goes over the blocks of the prefix and then over the sequence's own (akb_rows.h): which of them a block is one of is the same for
// the whole workgroup.
template <class T, int D, bool EXACT, class Args>
__global__ __launch_bounds__(64 * kWaves, 2) void prompt_kernel(Args a)
{
    constexpr bool kShared = std::is_same<Args, SharedArgs>::value;
    __shared__ PromptLds<D> lds;
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
    const int shared = [&] { if constexpr (kShared) return seq_len(a.prefix, b / a.per); else return 0; }();   // tokens of the prefix
    const int shared_blocks = (shared + kTB - 1) / kTB, gap = shared_blocks * kTB - shared;
    // the tokens that a row sees, as a place
    auto limit_of = [&](int row) {
        const int own = row_limit(a, row, G, m, len);
        return kShared && row < m * G ? shared + own + (own > 0 ? gap : 0) : own;
    };
    const int nb = (max(limit_of(row0 + rows - 1), 0) + kTB - 1) / kTB;
    const int lo = (int)(long(nb) * split / splits), hi = (int)(long(nb) * (split + 1) / splits);
    const int first_row = row0 + wave * kWaveRows, row = first_row + (lane & 31);
    const int wave_rows = min(kWaveRows, row0 + rows - first_row);   // may be below 1: the wave only helps to turn blocks
    const int all_see = limit_of(first_row), most_see = wave_rows > 0 ? limit_of(first_row + wave_rows - 1) : 0;
    const int limit = limit_of(row);
    auto place = [&](int row) { return row_place(a, bh, G, row, D); };   // of a row in q and out
    u32x4_t q[D / 16];
#pragma unroll
    for (int i = 0; i < D / 16; ++i) q[i] = row < m * G ? *reinterpret_cast<const u32x4_t*>(a.q + place(row) + 16 * i + 8 * half) : u32x4_t{0, 0, 0, 0};
    f32x16_t o[D / 32];
    float top, z;
    const OneSequence<D> own(c, bh, len);
    if constexpr (kShared) {
        const PrefixThenOwn<D> at(OneSequence<D>(a.prefix, size_t(b / a.per) * c.shape.Hkv + bh % c.shape.Hkv, shared), own);
        walk_prompt<T, D, EXACT>(lds, at, lo, hi, q, limit, all_see, most_see, a.c2, wave, lane, o, top, z);
    } else {
        walk_prompt<T, D, EXACT>(lds, own, lo, hi, q, limit, all_see, most_see, a.c2, wave, lane, o, top, z);
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

template <class T, int D, class Args> static hipError_t launch(const Args& r, int grid, hipStream_t st)
{
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(akv::xcd_grid(grid)), dim3(64 * kWaves), 0, st, r); };
    r.out_dtype == 0 ? go(prompt_kernel<T, D, true, Args>) : go(prompt_kernel<T, D, false, Args>);
    return hipGetLastError();
}
template <class Args> static hipError_t launch_typed(const Args& r, int grid, hipStream_t st)
{
    if (r.c.shape.dtype == AKB_FP16) return r.c.shape.D == 64 ? launch<Fp16, 64>(r, grid, st) : launch<Fp16, 128>(r, grid, st);
    return r.c.shape.D == 64 ? launch<Bf16, 64>(r, grid, st) : launch<Bf16, 128>(r, grid, st);
}
hipError_t launch_prompt(const RowArgs& r, int grid, hipStream_t st) { return launch_typed(r, grid, st); }
hipError_t launch_prompt_shared(const SharedArgs& r, int grid, hipStream_t st) { return launch_typed(r, grid, st); }

}  // namespace akb
