// Attention over the block-scaled 8-bit cache for few query rows, the score, and which kernels a call takes (rules and layout: include/akb.h; rows and
// parts: akb_rows.h; many rows: akb_prompt.hip).
//
// Few rows are bound by the codes: 2 D bytes per token and KV head, read once for all rows of a group.  A code becomes a number in one conversion of two (exact:
// the block's power of two is the conversion's scale) and goes from there to the matrix instruction; one walk keeps 16 KB per wave in flight.  16 sequences x 32 heads,
// 8192 tokens: 156 us, 6.9 TB/s, where a plain read of memory reaches 7.0.  Small calls are bound by their chain: launch, lengths, one block per wave, the
// waves' states through LDS, the parts through memory (32 heads, 1024 tokens: 7.6 us).
#include "akb_rows_walk.h"

namespace akb {

// How the walks over the blocks (one per row group) are shared out.  `slots` workgroups run at a time, two per compute unit (three or four per unit measured
// behind: their fixed costs, parts to write and join, outweigh what more loads in flight give; 8 x 8 pairs of 4096 tokens 15.6 / 18.3 / 19.4 us).  Where there
// are fewer walks than that, each is cut into parts.  The host knows a bound of the lengths only.  Calls of several long sequences with few walks are cut
// by the device, which looks through the lengths: parts of about equal length, all in one round (4 sequences of 32768 to 131072 tokens, 8 heads each: 139 ->
// 123 us).  Elsewhere every walk is cut into the same number of parts: a short call would wait for the lengths (8.0 -> 9.9 us), and with many walks the
// parts that are not full cost what they even out (16 x 32 pairs of 2048 to 8192 tokens 131 -> 145 us).
struct AttentionPlan {
    int tiles;      // row tiles of a row group: 1, 2 (rows kernel), 8 (prompt kernel)
    int groups;     // row groups of a (sequence, KV head)
    int splits;     // parts of a walk, or 0: cut by the device
    int grid;       // workgroups at most
    bool ticketed;  // the last workgroup of a row group joins its parts; otherwise a launch does
    bool streamed;  // codes are read with the non-temporal hint
    int shares;     // parts the rows are cut into for the score
    size_t tickets, parts, logits, stats, total;   // offsets into the workspace
};
// Parts of each of `items` walks: none where they fill the slots, or where a wave has two blocks at most (32 heads, 500 tokens 8.4 / 7.2 us; 1024 tokens in four parts,
// two, one 7.5 / 9.0 / 9.2); at most 2 slots parts in all, which is what the workspace has room for.
long parts_of(long items, long blocks, long slots)
{
    return items >= slots || blocks <= 2 * kWaves ? 1 : std::max(1L, std::min({(slots + items - 1) / items, (blocks + kWaves - 1) / kWaves, 2 * slots / items}));
}
static AttentionPlan plan(const akb_shape& s, int n, int max_len, bool accumulate)
{
    AttentionPlan p;
    const long slots = 2L * akv::compute_units(), rows = long(n) * (s.Hq / s.Hkv), pairs = long(s.B) * s.Hkv, blocks = (max_len + kTB - 1) / kTB;
    auto items_of = [&](int tiles) { return pairs * ((rows + 16 * tiles - 1) / (16 * tiles)); };
    // The prompt kernel from 65 rows on, where its parts are 12 blocks or longer (it fills a pipeline, and its parts have 128 rows to write and join).  Rows / prompt
    // kernel, us: 32 pairs of 5000 tokens 256 rows 38.8 / 42.6, 1024 rows 111 / 103; 32 of 5000, 100 rows 25.2 / 29.0; 64 of 3000, 160 rows 41.6 / 40.2; 8 of
    // 20000, 2048 rows 206 / 182; 8 of 100000, 64 rows 57 / 70; 24 of 13000, 40 rows 25.6 / 39.5; a prompt of 8192 tokens, 8 pairs of 32768 rows 730 / 558.
    constexpr int kPromptTiles = kPromptRows / 16;
    const long prompt_items = items_of(kPromptTiles);
    p.tiles = rows <= 16 ? 1 : (rows > 64 && blocks >= 12 * parts_of(prompt_items, blocks, slots) ? kPromptTiles : 2);
    const long items = items_of(p.tiles), splits = parts_of(items, blocks, slots);
    p.groups = (int)(items / pairs);
    p.splits = s.B > 1 && s.B <= kMostCut && items * 4 <= slots && blocks >= 8 * kWaves * splits ? 0 : (int)splits;
    p.grid = (int)(p.splits ? items * p.splits : slots);
    // Joined by the last workgroup where that has little to read (a launch less), by a launch of its own where it has much: rows x parts per row group 4 7.4 /
    // 11.0 us, 48 11.6 / 14.4, 64 40.5 / 45.1; 128 23.2 / 20.9, 350 29.7 / 25.9, 512 27.9 / 19.3 (last workgroup / launch).
    p.ticketed = p.tiles <= 2 && std::min(rows, 16L * p.tiles) * splits <= 64;
    // (calls of fewer query tokens fit into what is laid out for more: at most `2 slots` parts of up to 128 rows, and as many tickets)
    p.tickets = 0;
    p.parts = align256(size_t(2 * slots) * sizeof(int32_t));
    p.logits = p.parts + align256(size_t(2 * slots) * part_floats((int)std::min(rows, long(kPromptRows)), s.D) * sizeof(float));
    // Codes that are read once and are more than half of the last-level cache pass it by.  Plain / with the hint, us: 1.07 GB of 512 pairs 196 / 178, 268 MB of 256 54.0 / 47.2, 0.67 GB of
    // 32 long ones 121 / 106; below, what a call finds there of the call before counts: 134 MB 26.0 / 26.4, 67 MB 15.6 / 15.9, two row groups of 50 MB 25.4 / 27.3.
    p.streamed = p.tiles == 1 && size_t(pairs) * max_len * s.D * 2 > (size_t(128) << 20);
    // the score of many rows: two rounds of workgroups, at most eight shares of 256 rows or more
    const long quads = pairs * ((blocks + kWaves - 1) / kWaves);
    p.shares = (int)std::max(1L, std::min({(2 * slots + quads - 1) / quads, 8L, rows / 256}));
    p.stats = p.logits + (accumulate ? align256(size_t(pairs) * std::min(rows, 16L) * s.Ncap * sizeof(float)) : 0);
    p.total = p.stats + (accumulate ? align256(size_t(pairs) * rows * 2 * sizeof(float)) : 0);
    return p;
}
size_t attention_workspace(const akb_shape& s, int n, bool accumulate) { return plan(s, std::max(n, 1), s.Ncap, accumulate).total; }
int attention_path(const akb_shape& s, int n, int max_len, int32_t* parts)
{
    const AttentionPlan p = plan(s, n, max_len, false);
    if (parts) *parts = p.splits;
    return p.tiles <= 2 ? p.tiles : 3;
}
int attention_join(const akb_shape& s, int n, int max_len)
{
    const AttentionPlan p = plan(s, n, max_len, false);
    return p.splits == 1 ? 1 : (p.ticketed ? 2 : 3);
}
size_t attention_tickets() { return size_t(4) * akv::compute_units() * sizeof(int32_t); }

// One workgroup of four waves per (row group of RT row tiles, split): wave w takes every fourth block of the split, and the four states are put together
// through LDS.  Where a row group has several splits, the last of its workgroups to arrive joins them (the parts go through memory with device scope, as
// the partial results of the 16-bit cache's V kernel do).  EXACT: 32-bit results; the weights go into the second product as two binary16 numbers each (their
// sum carries 22 bits) or three bfloat16 numbers (24; with two, 16 bits, results of few or unlike weights were up to 4.6 times as far off as 32-bit arithmetic is).  The
// third costs single tokens 1 to 5 %, drafts 9 % (8 x 8 pairs of 3000 tokens, 40 rows: 21.8 / 23.6 us), prompts 24 % (8192 tokens: 737 / 914 us).
template <class T, int D, bool EXACT, int RT, bool NT>
__global__ __launch_bounds__(64 * kWaves, 2) void rows_kernel(RowArgs a)
{
    __shared__ float o_s[kWaves][kTileRows][D + 4];
    __shared__ float m_s[kWaves][kTileRows], z_s[kWaves][kTileRows];
    __shared__ int last_s;
    constexpr int kRows = kTileRows * RT;
    const akb_cache& c = a.c;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Cut cut;
    if (!cut.find<false>(a, 0)) return;
    const unsigned w = cut.w;
    const int splits = cut.splits, split = (w - cut.first) % splits, walk = (w - cut.first) / splits;
    const int group = a.groups - 1 - walk % a.groups;   // the rows that see most go first
    const int b = cut.b, G = c.shape.Hq / c.shape.Hkv, n = a.n;
    const size_t pair = size_t(b) * c.shape.Hkv + walk / a.groups;
    const int len = seq_len(c, b), m = a.n_q ? min(max(a.n_q[b], 0), n) : n;
    const size_t bh = pair, item = bh * a.groups + group;
    const int row0 = group * kRows, rows = min(kRows, m * G - row0);
    if (rows <= 0) return;   // no row of the group is wanted (in any split)
    const int keys = max(row_limit(a, row0 + rows - 1, G, m, len), 0), nb = (keys + kTB - 1) / kTB;
    const int all_see = row_limit(a, row0, G, m, len);               // tokens that every row sees
    const int lo = (int)(long(nb) * split / splits), hi = (int)(long(nb) * (split + 1) / splits);
    auto place = [&](int row) { return row_place(a, bh, G, row, D); };   // of a row in q and out
    RowState<T, D> st[RT];
#pragma unroll
    for (int k = 0; k < RT; ++k) {
        const int row = row0 + 16 * k + (lane & 15);
        st[k].init(row < m * G ? a.q + place(row) : nullptr, row_limit(a, row, G, m, len), lane);
    }
    float* logits = RT == 1 && a.logits ? a.logits + bh * min(a.n * G, 16) * c.shape.Ncap : nullptr;
    walk_rows<T, D, EXACT, RT, NT, kWaves>(c, bh, st, lo, hi, len, all_see, a.c2, lane, wave, logits, rows);
    const int part = part_floats(rows, D);
    const __amdgpu_buffer_rsrc_t parts = akv::make_rsrc(a.parts + size_t(w - split) * part_floats(min(n * G, kRows), D), uint32_t(splits) * part * 4u);
#pragma unroll
    for (int k = 0; k < RT; ++k) {
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
        // four consecutive channels of one row per thread and turn
        for (int e = threadIdx.x; e < min(16, rows - 16 * k) * (D / 4); e += 64 * kWaves) {
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
            if (splits == 1) {
                j.template finish<T>(a, bh * n * G, row0 + 16 * k + r, place(row0 + 16 * k + r), d);
                continue;
            }
            const uint32_t at = uint32_t(split) * part;
            akv::buf_store_b128_agent(__builtin_bit_cast(u32x4_t, j.o), parts, (at + part_head(rows) + (16 * k + r) * D + d) * 4);
            if (d == 0) {
                __builtin_amdgcn_raw_buffer_store_b32(float_bits(j.top), parts, (at + 2 * (16 * k + r)) * 4, 0, akv::kAuxSc1);
                __builtin_amdgcn_raw_buffer_store_b32(float_bits(j.z), parts, (at + 2 * (16 * k + r) + 1) * 4, 0, akv::kAuxSc1);
            }
        }
    }
    if (splits == 1 || !a.tickets) return;
    akv::stores_done();
    __syncthreads();
    if (threadIdx.x == 0) {
        const int t = akv::take_ticket(a.tickets + item);
        last_s = t == splits - 1;
        if (last_s) akv::store_agent(a.tickets + item, 0);
    }
    __syncthreads();
    if (!last_s) return;
    // the parts joined: a thread has kPer runs of four channels of a row, all splits; where there are few rows, one run in every `slices`-th split, and
    // the slices meet in LDS
    constexpr int kPer = kRows * (D / 4) / (64 * kWaves);
    const int work_items = rows * (D / 4), slices = 64 * kWaves / work_items;
    const int step = max(slices, 1), slice = slices > 1 ? int(threadIdx.x) / work_items : 0, e0 = slices > 1 ? int(threadIdx.x) % work_items : int(threadIdx.x);
    Joined j[kPer];
    if (slice < step)
#pragma unroll 4
        for (int s = slice; s < splits; s += step) {
            const uint32_t at = uint32_t(s) * part;
            u32x2_t mz[kPer];
            u32x4_t x[kPer];
#pragma unroll
            for (int i = 0; i < kPer; ++i) {   // (beyond the rows: beyond the buffer, which gives zeros, or another split's numbers; not used)
                const int e = e0 + 64 * kWaves * i;
                mz[i] = __builtin_amdgcn_raw_buffer_load_b64(parts, (at + 2 * (e / (D / 4))) * 4, 0, akv::kAuxSc1);
                x[i] = akv::buf_load_b128_agent(parts, (at + part_head(rows) + e * 4) * 4);
            }
#pragma unroll
            for (int i = 0; i < kPer; ++i) j[i].add(bits_float(mz[i].x), bits_float(mz[i].y), __builtin_bit_cast(f32x4_t, x[i]));
        }
    if (slices > 1) {
        float(*mine)[6] = reinterpret_cast<float(*)[6]>(&o_s[0][0][0]);
        j[0].put(mine[threadIdx.x]);
        __syncthreads();
        if (int(threadIdx.x) < work_items)
            for (int s = 1; s < slices; ++s) j[0].add(mine[threadIdx.x + s * work_items]);
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int e = int(threadIdx.x) + 64 * kWaves * i, r = e / (D / 4);
        if (e < work_items) j[i].template finish<T>(a, bh * n * G, row0 + r, place(row0 + r), e % (D / 4) * 4);
    }
}

// score[t] += sum over the rows of exp2(x - maximum) / sum, from the x that the rows kernel has left: calls of one row group, whose x are fewer bytes than
// K's codes or not many more.  A thread has four tokens.
__global__ __launch_bounds__(256) void score_logits_kernel(RowArgs a)
{
    const akb_cache& c = a.c;
    const int h = blockIdx.y, b = blockIdx.z, G = c.shape.Hq / c.shape.Hkv;
    const int len = seq_len(c, b), m = a.n_q ? min(max(a.n_q[b], 0), a.n) : a.n, rows = m * G;
    const size_t bh = size_t(b) * c.shape.Hkv + h;
    const float* stats = a.stats + bh * a.n * G * 2;
    for (int t = (blockIdx.x * 256 + threadIdx.x) * 4; t < len; t += gridDim.x * 1024) {
        const float* x = a.logits + bh * min(a.n * G, 16) * c.shape.Ncap + size_t(t / 16) * 16 * rows + t % 16;
        f32x4_t* p = reinterpret_cast<f32x4_t*>(c.score + bh * c.shape.Ncap + t);
        f32x4_t acc = *p;
#pragma unroll 4
        for (int r = 0; r < rows; ++r) {
            const f32x4_t v = *reinterpret_cast<const f32x4_t*>(x + r * 16);
            const float base = stats[2 * r], inv = stats[2 * r + 1];
            const int limit = row_limit(a, r, G, m, len);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (t + i < limit) acc[i] = fmaf(__builtin_amdgcn_exp2f(fmaf(v[i], a.c2, -base)), inv, acc[i]);
        }
        *p = acc;   // (the last of the four may lie behind the length: as they were)
    }
}

// The parts joined by a launch of their own: a thread has four channels of a row in every `SLICES`-th split, a workgroup of 256 threads as many rows as that
// leaves (many parts: one row at D = 128, two at 64; few: eight or sixteen).
template <class T, int D, int SLICES>
__global__ __launch_bounds__(256) void join_kernel(RowArgs a, int group_rows)
{
    constexpr int kRun = D / 4, kRows = 256 / (kRun * SLICES);
    __shared__ float x_s[256][6];
    const akb_cache& c = a.c;
    const int G = c.shape.Hq / c.shape.Hkv, n = a.n, tid = threadIdx.x;
    const unsigned pair = blockIdx.y;
    const int b = pair / c.shape.Hkv;
    const int m = a.n_q ? min(max(a.n_q[b], 0), n) : n;
    if (int(blockIdx.x) * kRows >= m * G) return;
    Cut cut;
    cut.find<true>(a, b);
    const int splits = cut.splits;
    if (splits == 1) return;   // its rows are there already
    const int row = blockIdx.x * kRows + tid / (kRun * SLICES), slice = tid / kRun % SLICES, d = tid % kRun * 4;
    const int group = row / group_rows, r = row % group_rows, rows = min(group_rows, m * G - group * group_rows), part = part_floats(rows, D);
    Joined j;
    if (row < m * G) {
        const unsigned walk = (pair % c.shape.Hkv) * a.groups + a.groups - 1 - group;   // as the kernels of the parts count them
        const float* parts = a.parts + (size_t(cut.first) + size_t(walk) * splits) * part_floats(min(n * G, group_rows), D);
#pragma unroll 8
        for (int s = slice; s < splits; s += SLICES) {
            const float* p = parts + size_t(s) * part;
            j.add(p[2 * r], p[2 * r + 1], *reinterpret_cast<const f32x4_t*>(p + part_head(rows) + r * D + d));
        }
    }
    if (SLICES > 1) {
        j.put(x_s[tid]);
        __syncthreads();
        if (slice) return;
        for (int s = 1; s < SLICES; ++s) j.add(x_s[tid + s * kRun]);
    }
    if (row < m * G) j.template finish<T>(a, size_t(pair) * n * G, row, row_place(a, pair, G, row, D), d);
}

// score[t] += sum over the rows of exp2(x - maximum) / sum: the scores of a block of K once more, for all rows (the weights of a row are known
// only when its last token has been seen).  A wave keeps a block's 16-bit numbers in its registers as the operand of 32 x 32 x 16 matrix instructions; the
// query rows come 64 at a time through LDS for the four waves (four blocks) of a workgroup, asked for a turn ahead (read by every wave for itself they cost
// more than the products: 252 us of a chunk of 777 tokens onto 20000, 2 x 32 heads).  Bound by the matrix instructions (32 of 32 cycles per turn) and
// the 64 weights per lane.  The sum over a lane's rows stays in its registers; lanes meet once, at the end.  Few blocks: the rows are cut into `shares`, whose sums
// score_join_kernel adds up in their order.
constexpr int kScoreRows = 64;
template <class T, int D>
__global__ __launch_bounds__(64 * kWaves, 2) void score_kernel(RowArgs a, int shares, float* __restrict__ sums)
{
    constexpr int kSteps = D / 16, kOct = D / 8, kPieces = kScoreRows * kOct / (64 * kWaves);
    // [32 rows][16 channels]: lane (row % 32, half): channels 8 half .. + 7.  The place of a lane's 16 bytes is turned by the channel octet, so that a row's
    // octets, which neighbouring threads write, lie in different banks.
    __shared__ u32x4_t q_s[2][2][kSteps][64];
    __shared__ f32x2_t stats_s[2][kScoreRows];
    const akb_cache& c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), low = lane & 31, half = lane >> 5;
    const int share = blockIdx.x % shares, h = blockIdx.y, b = blockIdx.z, G = c.shape.Hq / c.shape.Hkv, n = a.n;
    const int len = seq_len(c, b), m = a.n_q ? min(max(a.n_q[b], 0), n) : n;
    const size_t bh = size_t(b) * c.shape.Hkv + h;
    auto slot = [](int s, int oct) { return (s & 48) | ((s ^ oct) & 15); };
    for (int blk0 = blockIdx.x / shares * kWaves; blk0 * kTB < len && m > 0; blk0 += gridDim.x / shares * kWaves) {
        const int blk = blk0 + wave;
        const bool mine = blk * kTB < len;
        // K: lane (token % 32, half): channels 16 i + 8 half .. + 7
        u32x4_t k[2][kSteps];
        if (mine && blk < len / kTB) {
            const size_t block = bh * (c.shape.Ncap / kTB) + blk;
            const float s = pow2(c.exps[block * 2]);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    const u32x2_t w = *reinterpret_cast<const u32x2_t*>(c.k8 + block * (kTB * D) + k_place<D>(32 * t + low, 16 * i + 8 * half));
                    k[t][i] = cvt8<T>(w[0], w[1], s);
                }
        } else if (mine) {
            const uint16_t* kt = c.k_tail + bh * kTB * D;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < kSteps; ++i) k[t][i] = *reinterpret_cast<const u32x4_t*>(kt + (32 * t + low) * D + 16 * i + 8 * half);
        }
        f32x16_t acc[2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[t][r] = 0.f;
        const int turns = (m * G + kScoreRows - 1) / kScoreRows, begin = max(0, (blk0 * kTB - (len - m)) * G) / kScoreRows;   // from the first row that sees the first block
        const int lo = begin + int(long(turns - begin) * share / shares), hi = begin + int(long(turns - begin) * (share + 1) / shares);
        u32x4_t piece[kPieces];
        f32x2_t stat;
        auto fetch = [&](int turn) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int e = tid + 64 * kWaves * i, row = min(turn * kScoreRows + e / kOct, m * G - 1);
                piece[i] = *reinterpret_cast<const u32x4_t*>(a.q + row_place(a, bh, G, row, D) + e % kOct * 8);
            }
            if (tid < kScoreRows) {
                const int row = turn * kScoreRows + tid;
                stat = row < m * G ? *reinterpret_cast<const f32x2_t*>(a.stats + (bh * n * G + row) * 2) : f32x2_t{__builtin_inff(), 0.f};   // a row behind the last weighs 2^-inf
            }
        };
        auto put = [&](int to) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int e = tid + 64 * kWaves * i, row = e / kOct, oct = e % kOct;
                q_s[to][row >> 5][oct >> 1][slot((row & 31) + 32 * (oct & 1), oct)] = piece[i];
            }
            if (tid < kScoreRows) stats_s[to][tid] = stat;
        };
        if (lo < hi) {
            fetch(lo);
            put(0);
        }
        for (int turn = lo; turn < hi; ++turn) {
            const int at = (turn - lo) & 1;
            lds_barrier();
            if (turn + 1 < hi) fetch(turn + 1);
            if (mine) {
#pragma unroll 1   // (both at a time do not fit the registers)
                for (int j = 0; j < 2; ++j) {
                    f32x16_t s[2];
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int r = 0; r < 16; ++r) s[t][r] = 0.f;
#pragma unroll
                    for (int i = 0; i < kSteps; ++i) {
                        const u32x4_t q = q_s[at][j][i][slot(lane, 2 * i + half)];
#pragma unroll
                        for (int t = 0; t < 2; ++t) s[t] = T::mfma32(k[t][i], q, s[t]);
                    }
                    const f32x2_t stat = stats_s[at][32 * j + low];
                    const int row0 = turn * kScoreRows + 32 * j;
                    if ((blk + 1) * kTB > row_limit(a, row0, G, m, len)) {
                        const int seen = min(row_limit(a, row0 + low, G, m, len), len) - blk * kTB - 4 * half;   // counted from the lane's first token
#pragma unroll
                        for (int t = 0; t < 2; ++t)
#pragma unroll
                            for (int r = 0; r < 16; ++r)
                                if (32 * t + 8 * (r >> 2) + (r & 3) >= seen) s[t][r] = -__builtin_inff();
                    }
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[t][r] = fmaf(__builtin_amdgcn_exp2f(fmaf(s[t][r], a.c2, -stat.x)), stat.y, acc[t][r]);
                }
            }
            if (turn + 1 < hi) put(1 - at);
        }
        // over the 32 rows of a half of the lanes; lane `low` < 16 then stores the token of its number
        float* out = sums ? sums + (size_t(share) * c.shape.B * c.shape.Hkv + bh) * c.shape.Ncap : c.score + bh * c.shape.Ncap;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float sum = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                float v = acc[t][r];
                v = akv::add_dpp<0xB1>(v);
                v = akv::add_dpp<0x4E>(v);
                v = akv::add_dpp<0x124>(v);
                v = akv::add_dpp<0x128>(v);
                v = akv::add_lane16(v);
                sum = low == r ? v : sum;
            }
            const int token = blk * kTB + 32 * t + 8 * (low >> 2) + 4 * half + (low & 3);
            if (low < 16 && token < len) out[token] = sums ? sum : out[token] + sum;
        }
        lds_barrier();   // the rows are written again
    }
}

__global__ __launch_bounds__(256) void score_join_kernel(RowArgs a, int shares, const float* __restrict__ sums)
{
    const akb_cache& c = a.c;
    const int len = seq_len(c, blockIdx.z);
    if (a.n_q && a.n_q[blockIdx.z] <= 0) return;
    const size_t bh = size_t(blockIdx.z) * c.shape.Hkv + blockIdx.y, all = size_t(c.shape.B) * c.shape.Hkv;
    for (int t = blockIdx.x * 256 + threadIdx.x; t < len; t += gridDim.x * 256) {
        float v = c.score[bh * c.shape.Ncap + t];
        for (int s = 0; s < shares; ++s) v += sums[(s * all + bh) * c.shape.Ncap + t];
        c.score[bh * c.shape.Ncap + t] = v;
    }
}

template <class T, int D> static hipError_t join(const RowArgs& r, int group_rows, hipStream_t st)
{
    const akb_shape& s = r.c.shape;
    const int rows_all = r.n * (s.Hq / s.Hkv);
    auto go = [&](auto kernel, int rows) { hipLaunchKernelGGL(kernel, dim3((rows_all + rows - 1) / rows, s.B * s.Hkv), dim3(256), 0, st, r, group_rows); };
    if (r.splits && r.splits <= 4) go(join_kernel<T, D, 1>, 1024 / D);
    else go(join_kernel<T, D, 8>, 128 / D);
    return hipGetLastError();
}
hipError_t launch_join(const RowArgs& r, int group_rows, hipStream_t st)
{
    if (r.c.shape.dtype == AKB_FP16) return r.c.shape.D == 64 ? join<Fp16, 64>(r, group_rows, st) : join<Fp16, 128>(r, group_rows, st);
    return r.c.shape.D == 64 ? join<Bf16, 64>(r, group_rows, st) : join<Bf16, 128>(r, group_rows, st);
}

template <class T, int D> static hipError_t launch(const RowArgs& r, const AttentionPlan& p, float* sums, int max_len, hipStream_t st)
{
    const akb_shape& s = r.c.shape;
    const int tiles = p.tiles, grid = p.grid;
    auto rows = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(akv::xcd_grid(grid)), dim3(64 * kWaves), 0, st, r); };
    if (tiles > 2) {
        if (hipError_t e = launch_prompt(r, grid, st)) return e;
    } else if (tiles == 2) {
        r.out_dtype == 0 ? rows(rows_kernel<T, D, true, 2, false>) : rows(rows_kernel<T, D, false, 2, false>);
    } else if (p.streamed) {
        r.out_dtype == 0 ? rows(rows_kernel<T, D, true, 1, true>) : rows(rows_kernel<T, D, false, 1, true>);
    } else {
        r.out_dtype == 0 ? rows(rows_kernel<T, D, true, 1, false>) : rows(rows_kernel<T, D, false, 1, false>);
    }
    if (hipError_t e = hipGetLastError()) return e;
    if (r.splits != 1 && !r.tickets)
        if (hipError_t e = join<T, D>(r, 16 * tiles, st)) return e;
    const int blocks = (max_len + kTB - 1) / kTB;
    if (r.logits) hipLaunchKernelGGL(score_logits_kernel, dim3((blocks + 15) / 16, s.Hkv, s.B), dim3(256), 0, st, r);
    else if (r.stats) {
        const int quads = (blocks + kWaves - 1) / kWaves;
        hipLaunchKernelGGL((score_kernel<T, D>), dim3(quads * p.shares, s.Hkv, s.B), dim3(64 * kWaves), 0, st, r, p.shares, p.shares > 1 ? sums : nullptr);
        if (hipError_t e = hipGetLastError()) return e;
        if (p.shares > 1) hipLaunchKernelGGL(score_join_kernel, dim3((blocks + 3) / 4, s.Hkv, s.B), dim3(256), 0, st, r, p.shares, sums);
    }
    return hipGetLastError();
}

hipError_t launch_attention(const AttentionArgs& a, hipStream_t st)
{
    const AttentionPlan p = plan(a.c.shape, a.n, a.max_len, a.accumulate);
    const int G = a.c.shape.Hq / a.c.shape.Hkv;
    RowArgs r{a.c, a.q, a.n_q, a.n, p.groups, p.splits, p.grid, a.out_dtype, a.out, a.c2, uint32_t(G > 1 ? ((uint64_t(1) << 32) + G - 1) / G : 0), p.ticketed ? reinterpret_cast<int32_t*>(a.ws + p.tickets) : nullptr,
              reinterpret_cast<float*>(a.ws + p.parts), a.accumulate && p.tiles == 1 ? reinterpret_cast<float*>(a.ws + p.logits) : nullptr,
              a.accumulate ? reinterpret_cast<float*>(a.ws + p.stats) : nullptr};
    float* sums = reinterpret_cast<float*>(a.ws + p.logits);   // (a call has logits or sums)
    if (a.c.shape.dtype == AKB_FP16) return a.c.shape.D == 64 ? launch<Fp16, 64>(r, p, sums, a.max_len, st) : launch<Fp16, 128>(r, p, sums, a.max_len, st);
    return a.c.shape.D == 64 ? launch<Bf16, 64>(r, p, sums, a.max_len, st) : launch<Bf16, 128>(r, p, sums, a.max_len, st);
}

}  // namespace akb
