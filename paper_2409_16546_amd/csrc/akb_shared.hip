// Attention of sequences that go on from shared ones (rules and layout: include/akb.h; rows and parts: akb_rows.h).
//
// Few rows per sequence: the rows of all sequences of a prefix are the rows of one walk over it (a step of 64 sequences with four heads per KV head: 256 rows that read a
// prefix once instead of 64 times four), each sequence's own tokens are a walk of their own, and a launch behind puts a row's parts of both together.  Both kinds of
// walk are workgroups of one launch, those over prefixes first.
// Many rows per sequence (chunks behind a document): one walk over the prefix's blocks and the own ones, by the prompt kernel.  Its products are what takes time, and
// they do not get fewer by sharing.
#include "akb_prompt_walk.h"
#include "akb_rows_walk.h"

namespace akb {

// One kind of walk: over prefixes (the rows of `per` sequences) or over the sequences' own tokens (per = 1)
struct Side {
    akb_cache c;
    int per, groups, splits;
    float* parts;   // [pair][row group][split]
};
struct StepArgs {
    Side side[2];       // prefix, own
    unsigned items;     // workgroups of side 0
    const uint16_t* q;
    const int32_t* n_q;
    int n, G, out_dtype;
    void* out;
    float c2;
    int solo;           // an own walk is a wave's alone
};
// rows of a row group of TILES tiles (8: the prompt walk)
constexpr int tile_rows(int tiles) { return 16 * tiles; }

// A row of a side: sequence of the batch, query token, head of the group
struct StepRow {
    int b, token, head;
    __device__ __forceinline__ StepRow(const StepArgs& a, const Side& s, int first_b, int row)
    {
        const int per_seq = a.n * a.G, j = s.per == 1 ? 0 : row / per_seq, r = row - j * per_seq;
        b = first_b + j;
        token = r / a.G;
        head = r - token * a.G;
    }
};
__device__ __forceinline__ int queries(const StepArgs& a, int b) { return a.n_q ? min(max(a.n_q[b], 0), a.n) : a.n; }

// SOLO: by this wave alone, which meets no other
template <class T, int D, bool EXACT, int TILES, bool PREFIX, bool SOLO>
__device__ __forceinline__ void step_walk(const StepArgs& a, unsigned item, char* lds)
{
    const Side& s = a.side[PREFIX ? 0 : 1];
    const akb_cache& c = s.c;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned per_pair = s.groups * s.splits, pair = item / per_pair, in_pair = item - pair * per_pair;
    const int split = in_pair / s.groups, group = in_pair - split * s.groups;   // (the row groups of a part beside each other: they read the same blocks)
    const int p = pair / c.shape.Hkv, h = pair - p * c.shape.Hkv, first_b = p * s.per;
    const int len = seq_len(c, p), row0 = group * tile_rows(TILES), all_rows = s.per * a.n * a.G;
    const akb_cache& own = a.side[1].c;
    int keys = len;
    if (!PREFIX) {   // (of one sequence: the row groups behind its last row have nothing to do)
        const int m = queries(a, first_b);
        if (row0 >= m * a.G) return;
        const StepRow last(a, s, first_b, min(row0 + tile_rows(TILES), m * a.G) - 1);
        keys = max(len - m + last.token + 1, 0);
    }
    const int nb = (keys + kTB - 1) / kTB, lo = (int)(long(nb) * split / s.splits), hi = (int)(long(nb) * (split + 1) / s.splits);
    // where a row's query lies (NULL: nobody's, behind its sequence's n_q: it is multiplied with its tile all the same), and the tokens that it sees
    auto row_of = [&](int row, int& limit) -> const uint16_t* {
        limit = len;   // (a row that nobody wants: no mask on its account)
        if (row >= all_rows) return nullptr;
        const StepRow r(a, s, first_b, row);
        const int m = queries(a, r.b);
        if (r.token >= m) return nullptr;
        limit = PREFIX ? len + min(0, seq_len(own, r.b) - m + r.token + 1) : len - m + r.token + 1;
        return a.q + ((size_t(r.b) * c.shape.Hkv * a.G + h * a.G + r.head) * a.n + r.token) * D;
    };
    float* part = s.parts + (size_t(pair * s.groups + group) * s.splits + split) * part_floats(tile_rows(TILES), D);
    if constexpr (TILES <= 2) {
        float(*o_s)[kTileRows][D + 4] = reinterpret_cast<float(*)[kTileRows][D + 4]>(lds);
        float(*m_s)[kTileRows] = reinterpret_cast<float(*)[kTileRows]>(lds + sizeof(float) * kWaves * kTileRows * (D + 4));
        float(*z_s)[kTileRows] = m_s + kWaves;
        RowState<T, D> st[TILES];
        // (0 as soon as rows differ: all blocks of own walks of several query tokens are asked about then.  Until the least of the limits no block need be; 16 x 64 heads of 5 and 12
        // query tokens over 3001 own ones 32.6 / 32.0 and 39.4 / 39.4 us, 64 x 32 of 20 over 500 behind 2000 85.9 / 85.2)
        int all_see = len;
#pragma unroll
        for (int k = 0; k < TILES; ++k) {
            int limit;
            const uint16_t* q = row_of(row0 + 16 * k + (lane & 15), limit);
            st[k].init(q, limit, lane);
            if (__any(limit < len)) all_see = 0;
        }
        walk_rows<T, D, EXACT, TILES, false, SOLO ? 1 : kWaves>(c, pair, st, lo, hi, len, all_see, a.c2, lane, SOLO ? 0 : wave, nullptr, 0);
        const int rows = min(tile_rows(TILES), all_rows - row0);
        if (SOLO) {
#pragma unroll
            for (int k = 0; k < TILES; ++k) {
                const int r = 16 * k + (lane & 15);
                const float z = akv::add_lane32(akv::add_lane16(st[k].z));
                if (r >= rows) continue;
                if (lane < 16) {
                    part[2 * r] = st[k].m;
                    part[2 * r + 1] = z;
                }
#pragma unroll
                for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4_t*>(part + part_head(tile_rows(TILES)) + r * D + 16 * i + 4 * (lane >> 4)) = st[k].o[i];
            }
            return;
        }
#pragma unroll
        for (int k = 0; k < TILES; ++k) {
            if (16 * k >= rows) break;
            if (k) __syncthreads();   // the tile before has been put together
            const float z = akv::add_lane32(akv::add_lane16(st[k].z));
            if (lane < 16) {
                m_s[wave][lane] = st[k].m;
                z_s[wave][lane] = z;
            }
#pragma unroll
            for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4_t*>(&o_s[wave][lane & 15][16 * i + 4 * (lane >> 4)]) = st[k].o[i];
            __syncthreads();
            for (int e = threadIdx.x; e < min(16, rows - 16 * k) * (D / 4); e += 64 * kWaves) {   // four channels of a row
                const int r = e / (D / 4), d = e % (D / 4) * 4;
                Joined j;
                j.top = m_s[0][r];
#pragma unroll
                for (int w = 1; w < kWaves; ++w) j.top = fmaxf(j.top, m_s[w][r]);
                const float base = j.top == -__builtin_inff() ? 0.f : j.top;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    const float f = __builtin_amdgcn_exp2f(m_s[w][r] - base);
                    j.z = fmaf(z_s[w][r], f, j.z);
                    j.o += *reinterpret_cast<const f32x4_t*>(&o_s[w][r][d]) * f;
                }
                *reinterpret_cast<f32x4_t*>(part + part_head(tile_rows(TILES)) + (16 * k + r) * D + d) = j.o;
                if (d == 0) {
                    part[2 * (16 * k + r)] = j.top;
                    part[2 * (16 * k + r) + 1] = j.z;
                }
            }
        }
    } else {
        const int half = lane >> 5, r = wave * kWaveRows + (lane & 31);
        int limit;
        const uint16_t* row = row_of(row0 + r, limit);
        u32x4_t q[D / 16];
#pragma unroll
        for (int i = 0; i < D / 16; ++i) q[i] = row ? *reinterpret_cast<const u32x4_t*>(row + 16 * i + 8 * half) : u32x4_t{0, 0, 0, 0};
        const int all_see = __any(limit < len) ? 0 : len, most_see = row0 + wave * kWaveRows < all_rows ? len : 0;
        f32x16_t o[D / 32];
        float top, z;
        walk_prompt<T, D, EXACT>(*reinterpret_cast<PromptLds<D>*>(lds), OneSequence<D>(c, pair, len), lo, hi, q, limit, all_see, most_see, a.c2, wave, lane, o, top, z);
        if (row0 + r >= all_rows) return;
        z = akv::add_lane32(z);
        if (half == 0) {
            part[2 * r] = top;
            part[2 * r + 1] = z;
        }
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                *reinterpret_cast<f32x4_t*>(part + part_head(tile_rows(TILES)) + r * D + 32 * i + 8 * k + 4 * half) = f32x4_t{o[i][4 * k], o[i][4 * k + 1], o[i][4 * k + 2], o[i][4 * k + 3]};
    }
}

template <class T, int D, bool EXACT, int PREFIX_TILES, int OWN_TILES>
__global__ __launch_bounds__(64 * kWaves, 2) void step_kernel(StepArgs a)
{
    constexpr size_t kRowsLds = sizeof(float) * kWaves * kTileRows * (D + 4 + 2), kLds = PREFIX_TILES > 2 ? std::max(sizeof(PromptLds<D>), kRowsLds) : kRowsLds;
    __shared__ __align__(16) char lds[kLds];
    // the walks of a (sequence, KV head) of the prefix on one XCD, whose L2 they share, where the pairs are a multiple of the XCDs
    unsigned w = blockIdx.x;
    if (w < a.items) {
        const unsigned pairs = a.side[0].c.shape.B * a.side[0].c.shape.Hkv, per_pair = a.side[0].groups * a.side[0].splits;
        if (pairs % akv::kXcds == 0) {
            const unsigned x = w % akv::kXcds, i = w / akv::kXcds;
            w = (x + akv::kXcds * (i / per_pair)) * per_pair + i % per_pair;
        }
        step_walk<T, D, EXACT, PREFIX_TILES, true, false>(a, w, lds);
    } else if (a.solo) {
        const unsigned item = (w - a.items) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (item < unsigned(a.side[1].c.shape.B) * a.side[1].c.shape.Hkv * a.side[1].groups) step_walk<T, D, EXACT, OWN_TILES, false, true>(a, item, lds);
    } else {
        step_walk<T, D, EXACT, OWN_TILES, false, false>(a, w - a.items, lds);
    }
}

// A row's parts of both sides put together: a thread has four channels of a row in every `SLICES`-th part, a workgroup kRows rows of a (sequence, KV head) per turn.
template <class T, int D, int SLICES>
__global__ __launch_bounds__(256) void step_join_kernel(StepArgs a, int prefix_rows, int own_rows, unsigned turns, unsigned per_pair)
{
    constexpr int kRun = D / 4, kRows = 256 / (kRun * SLICES);
    __shared__ float x_s[256][6];
    const int tid = threadIdx.x, per_seq = a.n * a.G;
    const int Hkv = a.side[1].c.shape.Hkv;
    for (unsigned turn = blockIdx.x; turn < turns; turn += gridDim.x) {
        const unsigned pair = turn / per_pair, first = (turn - pair * per_pair) * kRows;
        const int b = pair / Hkv, h = pair - b * Hkv, m = queries(a, b);
        if (int(first) >= m * a.G) continue;
        const int row = first + tid / (kRun * SLICES), slice = tid / kRun % SLICES, d = tid % kRun * 4;
        Joined j;
        if (row < m * a.G) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const Side& s = a.side[i];
                const int tile = i == 0 ? prefix_rows : own_rows, p = b / s.per, at = row + (b - p * s.per) * per_seq, group = at / tile, r = at - group * tile;
                const float* parts = s.parts + size_t((size_t(p) * Hkv + h) * s.groups + group) * s.splits * part_floats(tile, D);
#pragma unroll 4
                for (int k = slice; k < s.splits; k += SLICES) {
                    const float* x = parts + size_t(k) * part_floats(tile, D);
                    j.add(x[2 * r], x[2 * r + 1], *reinterpret_cast<const f32x4_t*>(x + part_head(tile) + r * D + d));
                }
            }
        }
        if (SLICES > 1) {
            j.put(x_s[tid]);
            __syncthreads();
            if (slice == 0)
                for (int s = 1; s < SLICES; ++s) j.add(x_s[tid + s * kRun]);
            __syncthreads();   // (the next turn writes there)
        }
        if (row >= m * a.G || slice) continue;
        const int token = row / a.G, head = row - token * a.G;
        const float inv = j.z == 0.f ? 0.f : 1.f / j.z;   // zero: the row sees nothing
        store_row<T>(a.out, a.out_dtype, ((size_t(pair) * a.G + head) * a.n + token) * D + d, j.o * inv);
    }
}

// How a call is cut.
struct SharedPlan {
    bool one_walk;              // prefix and own blocks by one walk
    bool solo;                  // an own walk is a wave's alone
    int tiles[2], groups[2], splits[2];
    size_t parts[2], total;     // offsets into the workspace, its size
};
// Parts of each of `walks` walks: one workgroup or more per unit, two at most, and of those the numbers at which the unit with the most has the least
static long cut_into(long walks, long blocks, long units)
{
    long best = (units + walks - 1) / walks;
    for (long s = best + 1; walks * s <= 2 * units; ++s)
        if ((walks * s + units - 1) / units * best < (walks * best + units - 1) / units * s) best = s;
    return std::max(1L, std::min(best, blocks / kWaves));
}
// Rows of a sequence from which on one walk goes over both.  Walks of their own / one walk, us, at 64, 96, 128, 136 and 256 rows: 16 sequences of 500 tokens behind 8192, 32 heads on 8,
// 36.8 / 53.4, 52.3 / 57.4, 65.8 / 65.7, 70.5 / 92.5, 122.9 / 105.0; 16 of 3001 behind 13000, 64 on 8, 67.2 / 100.6, 102.9 / 107.3, 132.1 / 123.4, 141.5 / 196.6, 266.8 / 222.7;
// eight of eight behind 2000 73.3 / 75.5, 96.2 / 79.6, 126.7 / 88.6, 138.8 / 147.8, 238.1 / 159.6; two of four behind 20000 45.7 / 67.0, 65.3 / 73.1, 76.0 / 83.9, 112.3 / 118.4,
// 129.5 / 133.9.  The one walk fills each sequence's rows up to a multiple of 128, the others a prefix's rows to a multiple of 128 and a sequence's to one of 32.
constexpr int kOneWalkRows = 96;
// Whether a prefix's rows are the prompt walks', which turn a block once for 128 rows: where row walks, of 32 rows each, would be more than run at a time and do not all fall
// into one tile.  Row walk / prompt walk, us: 256 rows over 32768 tokens 56 / 66, 512 over 16384 45.5 / 57.8, 640 over 13000 59.1 / 58.6, 1024 over 4096 40.0 / 44.8 (256 row
// walks); but 816 over 163 34.2 / 27.8 (624), 1600 over 1000 57.0 / 48.6 (800), 100 over 2000 136.9 / 123.9 (1280), and 64 over 2000 171.6 / 181 (1280).
static bool prompt_walks(long pairs, long rows, long slots) { return rows > 96 && pairs * ((rows + 31) / 32) > slots; }
static SharedPlan plan(const akb_shape& f, const akb_shape& s, int n, int max_len, int prefix_max_len)
{
    SharedPlan p = {};
    const int per = s.B / f.B;
    const long slots = 2L * akv::compute_units(), seq_rows = long(n) * (s.Hq / s.Hkv);
    const long blocks[2] = {(prefix_max_len + kTB - 1) / kTB, (max_len + kTB - 1) / kTB}, pairs[2] = {long(f.B) * s.Hkv, long(s.B) * s.Hkv}, rows[2] = {per * seq_rows, seq_rows};
    p.one_walk = seq_rows >= kOneWalkRows;
    size_t at = align256(attention_tickets());
    if (p.one_walk) {
        p.groups[1] = int((seq_rows + kPromptRows - 1) / kPromptRows);
        p.splits[1] = int(parts_of(pairs[1] * p.groups[1], blocks[0] + blocks[1], slots));
        p.parts[1] = at;
        p.total = at + align256(size_t(2 * slots) * part_floats((int)std::min(seq_rows, long(kPromptRows)), s.D) * sizeof(float));
        return p;
    }
    // Parts: both kinds make one workgroup per compute unit where that shares the work out evenly, and no part is shorter than a block per wave: two prefix walks on a unit
    // take from each other most of what they gain, and own walks fill the second place.  Both kinds to fill both places / one each, us: 16 x 64 heads 13000 + 3001 tokens 80
    // / 59, 4 x 32 heads 32768 + 100 21.3 / 19.1, 8 x 8 heads 8192 + 2000 17.8 / 15.5, 8 prefixes of 8 x 32 heads 8192 + 500 43 / 38, 64 x 32 heads 32768 + 1000 63.7 / 56.3.
    // 160 row walks over 13000 tokens, in two / three: 54 / 46.5; 192 prompt walks, whole / in two: 89 / 80.5.  Own walks of five blocks, in two / whole: 13.7 / 12.0.
    const long units = slots / 2;
    for (int i = 0; i < 2; ++i) {
        const bool prompt = i == 0 && prompt_walks(pairs[i], rows[i], slots);
        p.tiles[i] = prompt ? kPromptRows / 16 : (i == 1 && rows[i] <= 16 ? 1 : 2);
        p.groups[i] = int((rows[i] + tile_rows(p.tiles[i]) - 1) / tile_rows(p.tiles[i]));
        const long walks = pairs[i] * p.groups[i];
        p.splits[i] = int(cut_into(walks, blocks[i], units));
        p.parts[i] = at;
        at += align256(size_t(walks) * p.splits[i] * part_floats(tile_rows(p.tiles[i]), s.D) * sizeof(float));
    }
    // Own walks of few blocks that are more than run at a time, one to a wave: 256 x 32 heads 4096 + 200 tokens 48.5 / 44, 120 x 64 heads of D = 64 2753 + 5 34 / 30 us; but
    // 16 x 32 heads 8192 + 250 16.2 / 19.5
    p.solo = long(pairs[1]) * p.groups[1] > slots && blocks[1] <= 4;
    p.total = at;
    return p;
}
// For calls of up to n query tokens: no kind of call needs more than this, whatever its number of tokens up to n and its bounds of the lengths.  Parts of walks that are
// cut are fewer than 2 slots; a walk that is not cut has its rows, filled up to a row group.
size_t shared_workspace(const akb_shape& f, const akb_shape& s, int n)
{
    const size_t slots = 2 * size_t(akv::compute_units()), G = s.Hq / s.Hkv, rows_all = size_t(std::max(n, 1)) * G, seq_rows = std::min(rows_all, size_t(kOneWalkRows));
    const size_t front = align256(attention_tickets()), pairs[2] = {size_t(f.B) * s.Hkv, size_t(s.B) * s.Hkv}, rows[2] = {size_t(s.B / f.B) * seq_rows, seq_rows};
    size_t step = front;
    for (int i = 0; i < 2; ++i) {
        const int tile = i == 0 && prompt_walks(long(pairs[i]), long(rows[i]), long(slots)) ? kPromptRows : 32;
        step += align256(std::max(2 * slots, pairs[i] * ((rows[i] + tile - 1) / tile)) * part_floats(tile, s.D) * sizeof(float));
    }
    const size_t one = rows_all >= size_t(kOneWalkRows) ? front + align256(2 * slots * part_floats(kPromptRows, s.D) * sizeof(float)) : 0;
    return std::max(step, one);
}
int shared_path(const akb_shape& f, const akb_shape& s, int n, int max_len, int prefix_max_len, int32_t* parts)
{
    const SharedPlan p = plan(f, s, n, max_len, prefix_max_len);
    if (parts)
        for (int i = 0; i < 2; ++i) parts[i] = p.splits[p.one_walk ? 1 : i];
    return p.one_walk ? 3 : (p.tiles[0] > 2 ? 2 : 1);
}

template <class T, int D> static hipError_t launch(const StepArgs& a, const SharedPlan& p, unsigned items, hipStream_t st)
{
    auto go = [&](auto f32, auto b16) {
        if (a.out_dtype == 0) hipLaunchKernelGGL(f32, dim3(items), dim3(64 * kWaves), 0, st, a);
        else hipLaunchKernelGGL(b16, dim3(items), dim3(64 * kWaves), 0, st, a);
    };
    if (p.tiles[0] == 2 && p.tiles[1] == 1) go(step_kernel<T, D, true, 2, 1>, step_kernel<T, D, false, 2, 1>);
    else if (p.tiles[0] == 2) go(step_kernel<T, D, true, 2, 2>, step_kernel<T, D, false, 2, 2>);
    else if (p.tiles[1] == 1) go(step_kernel<T, D, true, 8, 1>, step_kernel<T, D, false, 8, 1>);
    else go(step_kernel<T, D, true, 8, 2>, step_kernel<T, D, false, 8, 2>);
    if (hipError_t e = hipGetLastError()) return e;
    auto join = [&](auto kernel, int rows) {
        const unsigned per_pair = (a.n * a.G + rows - 1) / rows, turns = per_pair * a.side[1].c.shape.B * a.side[1].c.shape.Hkv;
        hipLaunchKernelGGL(kernel, dim3(std::min(turns, 1u << 20)), dim3(256), 0, st, a, tile_rows(p.tiles[0]), tile_rows(p.tiles[1]), turns, per_pair);
    };
    // A row's parts one after the other / by eight threads, us: 1 + 1 of them 50.2 / 73.0, 3 + 1 58.4 / 64.8, 4 + 1 38.5 / 41.3, 56.2 / 57.4 and 11.1 / 11.2, 8 + 2 23.0 /
    // 23.0, 16 + 1 18.7 / 18.3, 16 + 2 22.6 / 21.3, 32 + 2 22.5 / 19.5, 117 + 1 23.7 / 13.6.
    if (p.splits[0] + p.splits[1] <= 8) join(step_join_kernel<T, D, 1>, 1024 / D);
    else join(step_join_kernel<T, D, 8>, 128 / D);
    return hipGetLastError();
}

hipError_t launch_shared(const akb_cache& prefix, int prefix_max_len, const AttentionArgs& a, hipStream_t st)
{
    const akb_shape& s = a.c.shape;
    const SharedPlan p = plan(prefix.shape, s, a.n, a.max_len, prefix_max_len);
    const int G = s.Hq / s.Hkv, per = s.B / prefix.shape.B;
    if (p.one_walk) {
        const int grid = s.B * s.Hkv * p.groups[1] * p.splits[1];
        SharedArgs r;
        static_cast<RowArgs&>(r) = RowArgs{a.c, a.q, a.n_q, a.n, p.groups[1], p.splits[1], grid, a.out_dtype, a.out, a.c2, uint32_t(G > 1 ? ((uint64_t(1) << 32) + G - 1) / G : 0), nullptr,
                                           reinterpret_cast<float*>(a.ws + p.parts[1]), nullptr, nullptr};
        r.prefix = prefix;
        r.per = per;
        if (hipError_t e = launch_prompt_shared(r, grid, st)) return e;
        return p.splits[1] > 1 ? launch_join(r, kPromptRows, st) : hipSuccess;
    }
    auto side = [&](int i, const akb_cache& c, int per) { return Side{c, per, p.groups[i], p.splits[i], reinterpret_cast<float*>(a.ws + p.parts[i])}; };
    StepArgs r{{side(0, prefix, per), side(1, a.c, 1)}, 0, a.q, a.n_q, a.n, G, a.out_dtype, a.out, a.c2, p.solo ? 1 : 0};
    r.items = unsigned(prefix.shape.B) * s.Hkv * p.groups[0] * p.splits[0];
    const unsigned own = unsigned(s.B) * s.Hkv * p.groups[1] * p.splits[1], items = r.items + (p.solo ? (own + kWaves - 1) / kWaves : own);
    if (items >= 1u << 24) return hipErrorInvalidConfiguration;   // (a launch has fewer than 2^32 threads)
    if (s.dtype == AKB_FP16) return s.D == 64 ? launch<Fp16, 64>(r, p, items, st) : launch<Fp16, 128>(r, p, items, st);
    return s.D == 64 ? launch<Bf16, 64>(r, p, items, st) : launch<Bf16, 128>(r, p, items, st);
}

}  // namespace akb
