// What the attention kernels of the block-scaled 8-bit cache share: their arguments, how the walks over the blocks are cut, how parts of a row are put together.
//
// Rows: the query rows of one (sequence, KV head) are its n_q query tokens times its G query heads, row = token * G + head, so
// that one walk over K and V serves the whole group; 16 rows form a matrix tile.
// Both products are taken transposed, S^T = K Q^T and O^T = V^T P^T, so that a lane's column is a query row throughout: its
// four scores of a tile are four tokens of one row, which is what the second product takes as its operand (V's bytes lie in
// that order), and the running maximum, the sum and the rescaling of a row need no value of another row's lanes.
#pragma once

#include "akb_common.h"

namespace akb {

// In 16 bits the weights of fp16 caches lose bits below 2^-14, and end at 2^16.  They are taken relative to 2^-7 of a maximum that is moved only when a score
// lies 2^8 above it (then up to 2^15): O and the sum are multiplied anew in few blocks instead of in every other one.
constexpr float kWeightBits = 7.f, kSlackBits = 8.f;
// bfloat16 values reach as far as binary32 does: a token of weight 2^7 and value 2^121 would be beyond O.  The tokens of blocks whose values pass 2^71, and of tails whose
// values pass 2^65 (in the prompt kernel: of parts of a walk that hold such a one), have weights relative to 2^31 of their maximum: 2^22 of them, 2^(8 - 31) each, sum
// up to half of the largest value, and the others, 2^15 each, up to 2^109.  Only they: at this unit values below 2^-95 would lose bits, and the exponentials'
// arguments carry 2^-20 where the others' carry 2^-22.
constexpr float kSmallWeightBits = -31.f;
constexpr int kLargeExp = 64;       // least exponent of a block whose values pass 2^71 (448 2^63)
constexpr int kWaves = 4;           // of a workgroup
constexpr int kPromptRows = 128;    // of a row group of the prompt kernel
// What one split of a row group leaves for the workgroup that joins them: per row (maximum, sum), padded to 16 bytes, then O [row][D]
__host__ __device__ constexpr int part_head(int rows) { return (2 * rows + 3) / 4 * 4; }
__host__ __device__ constexpr int part_floats(int rows, int D) { return part_head(rows) + rows * D; }

constexpr int kMostCut = 256;   // sequences whose lengths every workgroup looks through

struct RowArgs {
    akb_cache c;
    const uint16_t* q;
    const int32_t* n_q;
    int n, groups, splits, slots, out_dtype;
    void* out;
    float c2;
    uint32_t inv_g;     // ceil(2^32 / G), or 0 where G is 1 (row_token)
    int32_t* tickets;   // [sequence, KV head, row group]: splits that have arrived, zero between calls; NULL: join_kernel follows
    float *parts, *logits, *stats;   // logits: q . k of the one row group, [sequence, KV head][block][tile][row][16]; stats: (maximum, 1 / sum) per row; or NULL
};

// Sequences that go on from shared ones: sequence b from sequence b / per of `prefix`.  In a walk over both the prefix's blocks come first: token t of a sequence's own stands at
// place 64 ceil(P / 64) + t, and the places between P and there are nobody's.
struct SharedArgs : RowArgs {
    akb_cache prefix;
    int per;
};

#if defined(__HIPCC__)
// the unit of the weights
template <class T> __device__ __forceinline__ float weight_bits(bool large) { return T::kWide && large ? kSmallWeightBits : kWeightBits; }
// bits 14 and 30 of what this gives: the two numbers are 2^65 or more (their exponents begin with two ones)
__device__ __forceinline__ uint32_t large_values(uint32_t w) { return w & (w << 1); }
constexpr uint32_t kLargeValues = 0x40004000u;

// the query token of a row, row / G: exact below 2^28 rows (there are at most 2^22 tokens of 16 rows)
__device__ __forceinline__ int row_token(const RowArgs& a, int row) { return a.inv_g ? int(__umulhi(uint32_t(row), a.inv_g)) : row; }
// the place of a row in q and out, [sequence][query head][n][D]; first: the pair's, of which G n rows follow
__device__ __forceinline__ size_t row_place(const RowArgs& a, size_t pair, int G, int row, int D)
{
    const int token = row_token(a, row);
    return ((pair * G + (row - token * G)) * a.n + token) * D;
}
// The tokens that rows see: row r (its query token of m) the first `limit`
__device__ __forceinline__ int row_limit(const RowArgs& a, int row, int G, int m, int len) { return row < m * G ? len - m + row_token(a, row) + 1 : 0; }

// How the walks of a call are cut: the same in every wave that asks.  Lane l has sequences l, l + 64, ..
struct Cut {
    unsigned w;        // this workgroup's number among those that have work
    int b, splits;     // its sequence, the parts of its walks
    unsigned first;    // the sequence's first workgroup
    // Workgroups are dealt to the XCDs in turn.  All row groups and parts of a (sequence, KV head) go to one XCD, whose L2 they share, every eighth pair to the same;
    // where the pairs are no multiple of the XCDs the work is dealt as it comes.  With one stretch of the pairs per XCD, long sequences, or a prompt's late rows,
    // fall to few XCDs.  Stretch / dealt, us: 16 x 8 pairs 300 query tokens, ragged 126.7 / 97.5; a prompt of 8192 tokens on 2 pairs with scores 746 / 588; 4 x 8 ragged
    // prompts of 4096 244 / 197; 8 x 32 ragged pairs of 4300 tokens 40.4 / 35.0; 16 x 32 of 8192 161.0 / 158.1, ragged 118 / 114; but 2 x 32 chunks of 777 onto
    // 20000 290 / 320, and 12 pairs' prompts 244 / 264.
    __device__ __forceinline__ bool deal(unsigned pairs, unsigned per_pair)
    {
        w = blockIdx.x;
        if (pairs % akv::kXcds == 0) {
            const unsigned x = blockIdx.x % akv::kXcds, i = blockIdx.x / akv::kXcds;
            w = (x + akv::kXcds * (i / per_pair)) * per_pair + i % per_pair;
        }
        return blockIdx.x < pairs * per_pair;
    }
    // ... of parts of equal length an XCD has one stretch: false where none is left
    __device__ __forceinline__ bool stretch(unsigned n)
    {
        const unsigned per = (n + akv::kXcds - 1) / akv::kXcds, x = blockIdx.x % akv::kXcds, i = blockIdx.x / akv::kXcds;
        w = x * per + i;
        return i < per && w < n;
    }
    // OF: of sequence `of`; otherwise of this workgroup; false where there is no work for it
    template <bool OF> __device__ __forceinline__ bool find(const RowArgs& a, int of)
    {
        const int B = a.c.shape.B, walks = a.c.shape.Hkv * a.groups, lane = threadIdx.x & 63;   // walks: per sequence
        splits = a.splits;
        if (splits) {
            if (!OF && !deal(unsigned(B) * a.c.shape.Hkv, unsigned(a.groups) * splits)) return false;
            b = OF ? of : int(w / unsigned(walks * splits));
            first = unsigned(b) * walks * splits;
            return true;
        }
        constexpr int kTurns = kMostCut / 64;
        int nb[kTurns];   // blocks of sequence 64 i + lane
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            const int s = 64 * i + lane;
            nb[i] = s < B && (!a.n_q || a.n_q[s] > 0) ? (seq_len(a.c, s) + kTB - 1) / kTB : 0;
        }
        unsigned total = 0;   // fewer than 2^25: at most 128 walks of 65536 blocks (and at least one part per walk in the `slots`)
#pragma unroll
        for (int i = 0; i < kTurns; ++i)
            if (64 * i < B) total += akv::wave_read(akv::wave_scan_add(nb[i]), 63);
        // the sum of all ceil(blocks / q) is below total / q + walks, so it fits the slots
        const unsigned most = a.slots - B * walks, q = max(unsigned(kWaves), (total * walks + most - 1) / most);
        auto parts = [&](int i) { return 64 * i + lane < B ? max(int((nb[i] + q - 1) / q), 1) : 0; };
        unsigned n = 0, before = 0;
#pragma unroll
        for (int i = 0; i < kTurns; ++i)
            if (64 * i < B) n += akv::wave_read(akv::wave_scan_add(parts(i)), 63);
        if (!OF && !stretch(n * walks)) return false;
        b = B;
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            if (64 * i >= B || b < B) continue;
            const int mine = parts(i), upto = akv::wave_scan_add(mine);
            const bool here = 64 * i + lane < B && (OF ? 64 * i + lane == of : (before + unsigned(upto)) * walks > w);
            if (const uint64_t past = __ballot(here)) {
                const int l = __builtin_ctzll(past);
                b = 64 * i + l;
                splits = akv::wave_read(mine, l);
                first = (before + unsigned(akv::wave_read(upto, l)) - splits) * walks;
            }
            before += akv::wave_read(upto, 63);
        }
        return true;
    }
};

template <class T> __device__ __forceinline__ void store_row(void* out, int out_dtype, size_t at, f32x4_t o)
{
    if (out_dtype == 0) *reinterpret_cast<f32x4_t*>(static_cast<float*>(out) + at) = o;
    else *reinterpret_cast<u32x2_t*>(static_cast<uint16_t*>(out) + at) = u32x2_t{T::pack(o[0], o[1]), T::pack(o[2], o[3])};
}

// Four channels of a row, put together from parts
struct Joined {
    float top = -__builtin_inff(), z = 0.f;
    f32x4_t o = {0, 0, 0, 0};
    __device__ __forceinline__ void add(float m1, float z1, f32x4_t o1)
    {
        const float up = fmaxf(top, m1), base = up == -__builtin_inff() ? 0.f : up;
        const float f = __builtin_amdgcn_exp2f(top - base), g = __builtin_amdgcn_exp2f(m1 - base);
        z = fmaf(z, f, z1 * g);
        o = o * f + o1 * g;
        top = up;
    }
    __device__ __forceinline__ void put(float (&p)[6]) const
    {
        p[0] = top;
        p[1] = z;
#pragma unroll
        for (int i = 0; i < 4; ++i) p[2 + i] = o[i];
    }
    __device__ __forceinline__ void add(const float (&p)[6]) { add(p[0], p[1], f32x4_t{p[2], p[3], p[4], p[5]}); }
    // the row's channels d .. d + 3 at `at` of out, and its statistics
    template <class T> __device__ __forceinline__ void finish(const RowArgs& a, size_t first_row, int row, size_t at, int d) const
    {
        const float inv = z == 0.f ? 0.f : 1.f / z;   // zero: the row sees nothing
        store_row<T>(a.out, a.out_dtype, at + d, o * inv);
        if (a.stats && d == 0) {
            float* p = a.stats + (first_row + row) * 2;
            p[0] = top == -__builtin_inff() ? 0.f : top;
            p[1] = inv;
        }
    }
};

#endif

hipError_t launch_prompt(const RowArgs& r, int grid, hipStream_t st);   // row groups of kPromptRows
hipError_t launch_prompt_shared(const SharedArgs& r, int grid, hipStream_t st);
hipError_t launch_join(const RowArgs& r, int group_rows, hipStream_t st);   // the parts of every walk put together by a launch
// Parts of each of `items` walks over `blocks` blocks, of which `slots` run at a time
long parts_of(long items, long blocks, long slots);

}  // namespace akb
