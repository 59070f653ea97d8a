/*
 * akb.h -- C ABI of the block-scaled 8-bit KV cache for MI355X (gfx950); part of the same library as akv.h.
 *
 * What it computes: a KV cache of a fixed size of 8 bits per element, for contexts that do not fit the 16 bits of
 * akv.h's cache or whose steps are bound by its bytes; attention over it for one query token per sequence (a decode
 * step), for a few (a draft that is checked) or for many (a prompt, a chunk of one); and eviction, which brings every
 * (sequence, KV head) down to a budget of tokens by the attention weight that each token has received.
 *
 *   store     Tokens lie in blocks of 64.  A complete block of one (sequence, KV head) holds e4m3 numbers (sign, 4 bits
 *             of exponent, 3 of mantissa) and one power of two per side (K, V): x is stored as the number c nearest to
 *             x 2^-e (ties to even), e the least integer with max|x| <= 448 2^e, at least -100, and stands for c 2^e.
 *             (Where c 2^e would be beyond the 16-bit type, which takes a maximum within 1/16 of the type's largest
 *             number, the next smaller c is taken.)  c 2^e is a number of the 16-bit type: no step of the path rounds
 *             it again.  Powers of two, because a block can then be rebuilt from others (eviction) without its numbers
 *             being rounded anew, save those below 2^(e - 6), the smallest normal number of the new block, which keep
 *             fewer than four bits (none below 2^(e - 10)), and tokens of the tail that come to lie in a complete block,
 *             which are rounded for the first time.
 *             The tokens of the last, incomplete block are held in 16 bits (the tail) until the block is complete.  So
 *             every block is rounded once, from its own tokens, and the bytes do not depend on how the appends were cut.
 *   attend    Query token i of the n_q[b] of sequence b stands at place lens[b] - n_q[b] + i and sees the stored tokens
 *             up to and including its own place:
 *             x_t = scale (q . k_t);  p = softmax(x) over the tokens it sees;  out = sum_t p_t v_t.
 *             The query tokens are stored before they attend (akb_append first).  Scores, maxima, sums, and the weights
 *             as they are summed up are held in binary32, which q . k has to lie in.  For the product with v a weight is
 *             rounded to the 16-bit type where out has 16 bits, and is the sum of two or three such numbers where out is
 *             float32 (22 bits in binary16, 24 in bfloat16).  In binary16 a weight is no finer than 2^-32 of the row's largest.
 *             Finite v give finite results; values of 2^65 and more (bfloat16) cost the weights beside them some bits: their
 *             exponents carry 2^-20 instead of 2^-22, and values 2^160 below them may count as zero.
 *   score     Optionally score[b][h][t] += sum of p_t over the call's query tokens and the query heads of KV head h.
 *   evict     Of each (sequence, KV head) the `recent` last tokens stay, and of the others those with the largest score
 *             (ties: the earlier token), `keep` in all, in their order.
 *
 * Conventions: those of akv.h (device pointers owned by the caller unless named "host", nothing is allocated or
 * synchronised, work is enqueued on the caller's stream, akv_status / akv_last_error(), 16-byte alignment of every
 * device array, lens, flags, n_new and n_q 4 bytes).  Every call enqueues kernels only and can be captured into a HIP graph.
 * Inputs of tokens that are stored must be finite; an infinity or a NaN is stored as a NaN in 8 bits and reaches every
 * query row of its head whose tile holds it.  What lies behind a sequence's length, behind n_new[b] rows of k_new and v_new
 * or behind n_q[b] rows of q may be anything.
 */
#ifndef AKB_H
#define AKB_H

#include "akv.h"

#ifdef __cplusplus
extern "C" {
#endif

#define AKB_TB 64        /* tokens per block                       */
#define AKB_MAX_G 16     /* query heads per KV head                */
#define AKB_FP16 0       /* akb_shape.dtype: IEEE binary16         */
#define AKB_BF16 1       /* akb_shape.dtype: bfloat16              */

/* Hq query heads share Hkv KV heads in groups of G = Hq/Hkv <= 16 consecutive ones (any whole number); D is 64 or 128;
 * Ncap a multiple of 64. */
typedef struct akb_shape {
    int32_t B, Hq, Hkv, D, Ncap;
    int32_t dtype; /* of k_new, v_new, q, the tails and 16-bit results: AKB_FP16 or AKB_BF16 */
} akb_shape;

/*
 * The cache (NB = Ncap / 64; token t of a block: tile t / 16, group (t / 4) % 4, t % 4 in the group):
 *   k8     [B][Hkv][NB][4][D/64][16][64] uint8   K: tile of 16 tokens, 64 channels, token, channel
 *   v8     [B][Hkv][NB][D][64]           uint8   V: channel-major; token t at place 16 ((t/4) % 4) + 4 (t/16) + t % 4
 *   exps   [B][Hkv][NB][2]               int8    e of the block's K, of its V
 *   k_tail [B][Hkv][64][D]               16 bits the incomplete block's K, token-major
 *   v_tail [B][Hkv][D][64]               16 bits ... its V, in the order of v8
 *   score  [B][Hkv][Ncap]                float   accumulated attention weight, or NULL where it is not wanted
 *   lens   [B]                           int32   tokens stored; the caller may set a sequence's length to 0
 *   flags  [AKV_NFLAGS + B]              int32   as in akv.h: flags[AKV_FLAG_OVERFLOW] counts refused appends
 * (The orders are those in which the matrix units take their operands: a wave reads whole KiB, and a value goes from its
 * byte to a matrix instruction without changing lanes.)
 */
typedef struct akb_cache {
    akb_shape shape;
    uint8_t *k8, *v8;
    int8_t *exps;
    uint16_t *k_tail, *v_tail;
    float *score;
    int32_t *lens;
    int32_t *flags;
} akb_cache;

/* Byte sizes of the caller-owned buffers for a shape. */
typedef struct akb_sizes {
    size_t k8, v8, exps, k_tail, v_tail, score, lens, flags;
} akb_sizes;

akv_status akb_layout_sizes(const akb_shape *shape, akb_sizes *out);

/* Empty the cache: zero lens and flags, and score where there is one.  The planes need no clearing: nothing behind a
 * sequence's length is ever read. */
akv_status akb_cache_reset(const akb_cache *cache, void *stream);

/*
 * Append tokens.  k_new, v_new: device [B][Hkv][n][D] of the shape's type.  n_new: device int32 [B] with the number of
 * leading rows (0..n) to take for each sequence, or NULL for all n.  A sequence whose new length would exceed Ncap is left
 * unchanged and flags[AKV_FLAG_OVERFLOW] is incremented.  The new tokens' scores are set to 0.  Calls on one cache must be
 * ordered on one stream.
 */
akv_status akb_append(const akb_cache *cache, const uint16_t *k_new, const uint16_t *v_new, const int32_t *n_new, int32_t n, void *stream);

typedef struct akb_params {
    float scale;        /* softmax scale; <= 0 means 1/sqrt(D)                                              */
    int32_t out_dtype;  /* 0: out is float32; 1: out has the shape's 16-bit type                            */
    int32_t accumulate; /* nonzero: add the weights to cache->score                                         */
    int32_t max_len;    /* host-known bound of lens[] that the launch is laid out for; 0 means Ncap.  It is
                           a hint: longer sequences are attended whole all the same                         */
} akb_params;

/* Bytes of scratch akb_attention needs for calls of up to n query tokens, and akb_evict for its `keep`
 * (host computation; 0 on a bad shape). */
size_t akb_attention_workspace(const akb_shape *shape, int32_t n, int32_t accumulate);
size_t akb_evict_workspace(const akb_shape *shape, int32_t keep);

/* Prepare a workspace: zero its control words (arrival counters at its front, which every call leaves at zero again and evictions do not touch).
 * Once on every workspace before its first use, and again if anything else wrote to it; a single small fill kernel. */
akv_status akb_workspace_init(void *workspace, size_t workspace_bytes, void *stream);

/*
 * Attention of n query tokens per sequence.  q: device [B][Hq][n][D] of the shape's type.  n_q: device int32 [B] with the
 * number of leading query tokens (0..n) of each sequence, or NULL for n.  out: device [B][Hq][n][D] of params->out_dtype;
 * B * Hkv * ceil(n Hq/Hkv / 16) < 2^24.  Rows i >= n_q[b] are left as they were; a query token that sees nothing yields zeros.  workspace: device scratch, 256-B
 * aligned, prepared by akb_workspace_init; calls that overlap need distinct ones, and it holds nothing between calls.
 * Calls that accumulate into one cache's score must be ordered on one stream.  params may be
 * NULL (float32 out, no accumulation).  The same call gives the same bits.
 */
akv_status akb_attention(const akb_cache *cache, const uint16_t *q, const int32_t *n_q, int32_t n, void *out, const akb_params *params,
                         void *workspace, size_t workspace_bytes, void *stream);

/* Which kernels akb_attention takes for n query tokens: 1 = row groups of 16 rows, 2 = of 32, 3 = of 128 (many rows); max_len as in akb_params.  parts: NULL, or
 * a host pointer that receives the parts each walk over the blocks is cut into (0: the device cuts by the lengths).  Host computation; 0 on a bad shape.  For
 * callers that attribute time to kernels. */
int32_t akb_attention_path(const akb_shape *shape, int32_t n, int32_t max_len, int32_t *parts);

/* How the parts of that call are put together: 1 = every walk is one part, 2 = by the last workgroup of a row group, 3 = by a launch behind.  Host computation; 0
 * on a bad shape. */
int32_t akb_attention_join(const akb_shape *shape, int32_t n, int32_t max_len);

/*
 * Evict: src's tokens (their values as they are read, their scores) go to dst, at most `keep` of each (sequence, KV head):
 * the min(recent, kept) last ones and, of the others, those of the largest score.  A NaN counts as the largest.  dst has src's
 * B, Hkv, D and dtype, Ncap >= keep, and shares no memory with src; what it held is replaced, lens[b] becomes
 * min(lens[b], keep).  src needs a score; dst->score may be NULL.  kept: NULL, or device int32 [B][Hkv][keep] that
 * receives the kept tokens' places in src, ascending, -1 behind the last.  src is not written.
 * workspace: as for akb_attention, of akb_evict_workspace(src's shape, keep) bytes or more.
 */
akv_status akb_evict(const akb_cache *src, const akb_cache *dst, int32_t keep, int32_t recent, int32_t *kept, void *workspace, size_t workspace_bytes,
                     void *stream);

/* The values as they are read: device [B][Hkv][Ncap][D] of the shape's type, zeros behind a sequence's length.  Either output may be NULL. */
akv_status akb_unpack(const akb_cache *cache, uint16_t *k_out, uint16_t *v_out, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* AKB_H */
