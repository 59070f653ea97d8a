// C ABI of the block-scaled 8-bit cache (declared in include/akb.h): argument checks, launches.
#include <cmath>

#include "akb_common.h"

namespace {

constexpr auto fail = &akv::fail_msg;

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

bool shape_ok(const akb_shape& s)
{
    return s.B > 0 && s.B <= 65535 && s.Hq > 0 && s.Hkv > 0 && s.Hkv <= 65535 && (s.D == 64 || s.D == 128) && s.Hq % s.Hkv == 0 &&
           s.Hq / s.Hkv <= AKB_MAX_G && s.Ncap > 0 && s.Ncap % AKB_TB == 0 && s.Ncap <= (1 << 22) && (s.dtype == AKB_FP16 || s.dtype == AKB_BF16) &&
           size_t(s.B) * s.Hq * size_t(s.Ncap) < (size_t(1) << 40);
}
akv_status bad_shape(const akb_shape& s)
{
    return fail(AKV_EINVAL, "bad shape: B=%d Hq=%d Hkv=%d D=%d Ncap=%d dtype=%d (need D 64 or 128, Hq/Hkv whole and <= 16, Ncap %% 64 == 0, dtype 0 or 1)", s.B,
                s.Hq, s.Hkv, s.D, s.Ncap, s.dtype);
}

akv_status check_cache(const akb_cache* c)
{
    if (!c) return fail(AKV_EINVAL, "cache is NULL");
    if (!shape_ok(c->shape)) return bad_shape(c->shape);
    if (!c->k8 || !c->v8 || !c->exps || !c->k_tail || !c->v_tail || !c->lens || !c->flags)
        return fail(AKV_EINVAL, "cache has a NULL plane / exps / tail / lens / flags pointer");
    if (!aligned(c->k8, 16) || !aligned(c->v8, 16) || !aligned(c->exps, 16) || !aligned(c->k_tail, 16) || !aligned(c->v_tail, 16) || !aligned(c->score, 16) ||
        !aligned(c->lens, 4) || !aligned(c->flags, 4))
        return fail(AKV_EINVAL, "cache planes, exps, tails and score must be 16-byte aligned, lens and flags 4-byte aligned");
    return AKV_OK;
}

akv_status check_workspace(const void* ws, size_t given, size_t needed)
{
    if (!ws || given < needed) return fail(AKV_EWORKSPACE, "workspace of %zu bytes given, %zu needed", ws ? given : size_t(0), needed);
    if (!aligned(ws, 256)) return fail(AKV_EWORKSPACE, "workspace is not 256-byte aligned");
    return AKV_OK;
}

akv_status hip_result(hipError_t e, const char* what) { return e == hipSuccess ? AKV_OK : fail(AKV_EHIP, "%s: %s", what, hipGetErrorString(e)); }

void sizes_of(const akb_shape& s, akb_sizes* out)
{
    const size_t pairs = size_t(s.B) * s.Hkv, e = pairs * size_t(s.Ncap) * s.D;
    out->k8 = e;
    out->v8 = e;
    out->exps = pairs * (s.Ncap / AKB_TB) * 2;
    out->k_tail = out->v_tail = pairs * AKB_TB * s.D * 2;
    out->score = pairs * size_t(s.Ncap) * sizeof(float);
    out->lens = size_t(s.B) * sizeof(int32_t);
    out->flags = (AKV_NFLAGS + size_t(s.B)) * sizeof(int32_t);
}

// sequences of shape s that go on from those of f
bool shares_ok(const akb_shape& f, const akb_shape& s) { return s.B % f.B == 0 && s.Hq == f.Hq && s.Hkv == f.Hkv && s.D == f.D && s.dtype == f.dtype; }

bool overlap(const void* p, size_t n, const void* q, size_t m)
{
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    return p && q && n && m && a < b + m && b < a + n;
}

// a sequence's blocks that an append of n projected tokens can touch, by KV head: its workgroups have fewer than 2^32 threads
bool rotated_blocks_ok(const akb_shape& s, int n) { return (size_t(n) + 126) / AKB_TB * s.Hkv < size_t(1) << 23; }

// whether src and dst share memory (scores where dst's is written)
bool share_memory(const akb_cache& src, const akb_cache& dst)
{
    akb_sizes a, b;
    sizes_of(src.shape, &a);
    sizes_of(dst.shape, &b);
    const struct { const void *p; size_t n; } from[] = {{src.k8, a.k8}, {src.v8, a.v8}, {src.exps, a.exps}, {src.k_tail, a.k_tail}, {src.v_tail, a.v_tail}, {src.score, src.score ? a.score : 0}, {src.lens, a.lens}},
                 to[] = {{dst.k8, b.k8}, {dst.v8, b.v8}, {dst.exps, b.exps}, {dst.k_tail, b.k_tail}, {dst.v_tail, b.v_tail}, {dst.score, dst.score ? b.score : 0}, {dst.lens, b.lens}};
    for (const auto& x : from)
        for (const auto& y : to)
            if (overlap(x.p, x.n, y.p, y.n)) return true;
    return false;
}

// what attention's arguments have to be, whichever caches they are for
akv_status check_attention(const akb_shape& s, const akb_params& p, const uint16_t* q, const int32_t* n_q, int32_t n, const void* out)
{
    if (n < 0 || n > s.Ncap) return fail(AKV_EINVAL, "n = %d out of range 0..Ncap", n);
    const size_t tiles = size_t(s.B) * s.Hkv * ((size_t(n) * (s.Hq / s.Hkv) + 15) / 16);
    if (tiles >= (size_t(1) << 24)) return fail(AKV_EINVAL, "%zu tiles of 16 query rows: 2^24 or more", tiles);
    if (p.out_dtype != 0 && p.out_dtype != 1) return fail(AKV_EINVAL, "out_dtype = %d is neither 0 (f32) nor 1 (the cache's 16-bit type)", p.out_dtype);
    if (p.max_len < 0 || p.max_len > s.Ncap) return fail(AKV_EINVAL, "max_len = %d out of range 0..Ncap", p.max_len);
    if (!std::isfinite(p.scale)) return fail(AKV_EINVAL, "scale is not finite");
    if (n == 0) return AKV_OK;
    if (!q || !out) return fail(AKV_EINVAL, "q / out is NULL");
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(n_q, 4)) return fail(AKV_EINVAL, "q and out must be 16-byte aligned, n_q 4-byte aligned");
    return AKV_OK;
}
float scale_bits(const akb_params& p, int D)
{
    const double scale = p.scale > 0.f ? (double)p.scale : 1.0 / std::sqrt((double)D);
    return (float)(scale * 1.4426950408889634);
}

}  // namespace

extern "C" {

akv_status akb_layout_sizes(const akb_shape* shape, akb_sizes* out)
{
    if (!shape || !out) return fail(AKV_EINVAL, "NULL argument");
    if (!shape_ok(*shape)) return bad_shape(*shape);
    sizes_of(*shape, out);
    return AKV_OK;
}

akv_status akb_cache_reset(const akb_cache* cache, void* stream)
{
    if (akv_status st = check_cache(cache)) return st;
    akb_sizes sz;
    sizes_of(cache->shape, &sz);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (akv_status st = hip_result(akv::launch_zero(cache->lens, sz.lens, s), "zero launch")) return st;
    if (akv_status st = hip_result(akv::launch_zero(cache->flags, sz.flags, s), "zero launch")) return st;
    return cache->score ? hip_result(akv::launch_zero(cache->score, sz.score, s), "zero launch") : AKV_OK;
}

akv_status akb_append(const akb_cache* cache, const uint16_t* k_new, const uint16_t* v_new, const int32_t* n_new, int32_t n, void* stream)
{
    if (akv_status st = check_cache(cache)) return st;
    if (n < 0 || n > cache->shape.Ncap) return fail(AKV_EINVAL, "n = %d out of range 0..Ncap", n);
    if (n == 0) return AKV_OK;
    if (!k_new || !v_new) return fail(AKV_EINVAL, "k_new / v_new is NULL");
    if (!aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(n_new, 4)) return fail(AKV_EINVAL, "k_new / v_new must be 16-byte aligned, n_new 4-byte aligned");
    return hip_result(akb::launch_append(*cache, k_new, v_new, n_new, n, static_cast<hipStream_t>(stream)), "append launch");
}

size_t akb_attention_workspace(const akb_shape* shape, int32_t n, int32_t accumulate)
{
    if (!shape || !shape_ok(*shape) || n < 0 || n > shape->Ncap) {
        fail(AKV_EINVAL, "bad shape, or n out of range 0..Ncap");
        return 0;
    }
    return akb::attention_workspace(*shape, n, accumulate != 0);
}

akv_status akb_workspace_init(void* workspace, size_t workspace_bytes, void* stream)
{
    if (akv_status st = check_workspace(workspace, workspace_bytes, akb::attention_tickets())) return st;
    return hip_result(akv::launch_zero(workspace, akb::attention_tickets(), static_cast<hipStream_t>(stream)), "zero launch");
}

akv_status akb_attention(const akb_cache* cache, const uint16_t* q, const int32_t* n_q, int32_t n, void* out, const akb_params* params, void* workspace,
                         size_t workspace_bytes, void* stream)
{
    if (akv_status st = check_cache(cache)) return st;
    const akb_shape& s = cache->shape;
    akb_params p = {};
    if (params) p = *params;
    if (p.accumulate && !cache->score) return fail(AKV_EINVAL, "accumulate is set and the cache has no score");
    if (akv_status st = check_attention(s, p, q, n_q, n, out)) return st;
    if (n == 0) return AKV_OK;
    if (akv_status st = check_workspace(workspace, workspace_bytes, akb::attention_workspace(s, n, p.accumulate != 0))) return st;
    const akb::AttentionArgs a{*cache, q, n_q, n, out, p.out_dtype, p.accumulate != 0, p.max_len > 0 ? p.max_len : s.Ncap,
                               scale_bits(p, s.D), static_cast<char*>(workspace)};
    return hip_result(akb::launch_attention(a, static_cast<hipStream_t>(stream)), "attention launch");
}

int32_t akb_attention_path(const akb_shape* shape, int32_t n, int32_t max_len, int32_t* parts)
{
    if (!shape || !shape_ok(*shape) || n < 1 || n > shape->Ncap || max_len < 0 || max_len > shape->Ncap) return 0;
    return akb::attention_path(*shape, n, max_len > 0 ? max_len : shape->Ncap, parts);
}

int32_t akb_attention_join(const akb_shape* shape, int32_t n, int32_t max_len)
{
    if (!shape || !shape_ok(*shape) || n < 1 || n > shape->Ncap || max_len < 0 || max_len > shape->Ncap) return 0;
    return akb::attention_join(*shape, n, max_len > 0 ? max_len : shape->Ncap);
}

size_t akb_evict_workspace(const akb_shape* shape, int32_t keep)
{
    if (!shape || !shape_ok(*shape) || keep < 1) {
        fail(AKV_EINVAL, "bad shape, or keep below 1");
        return 0;
    }
    return akv::align256(akb::attention_tickets()) + akb::evict_workspace(*shape, keep);
}

akv_status akb_evict(const akb_cache* src, const akb_cache* dst, int32_t keep, int32_t recent, int32_t* kept, void* workspace, size_t workspace_bytes, void* stream)
{
    if (akv_status st = check_cache(src)) return st;
    if (akv_status st = check_cache(dst)) return st;
    const akb_shape &s = src->shape, &d = dst->shape;
    if (s.B != d.B || s.Hkv != d.Hkv || s.D != d.D || s.dtype != d.dtype)
        return fail(AKV_EINVAL, "src and dst differ: B %d/%d, Hkv %d/%d, D %d/%d, dtype %d/%d", s.B, d.B, s.Hkv, d.Hkv, s.D, d.D, s.dtype, d.dtype);
    if (!src->score) return fail(AKV_EINVAL, "src has no score");
    if (keep < 1 || keep > d.Ncap) return fail(AKV_EINVAL, "keep = %d out of range 1..dst Ncap", keep);
    if (recent < 0 || recent > keep) return fail(AKV_EINVAL, "recent = %d out of range 0..keep", recent);
    if (share_memory(*src, *dst)) return fail(AKV_EINVAL, "src and dst share memory");
    if (!aligned(kept, 4)) return fail(AKV_EINVAL, "kept must be 4-byte aligned");
    if (akv_status st = check_workspace(workspace, workspace_bytes, akb_evict_workspace(&s, keep))) return st;
    char* ws = static_cast<char*>(workspace) + akv::align256(akb::attention_tickets());   // (what lies in front is attention's between calls)
    return hip_result(akb::launch_evict(*src, *dst, keep, recent, kept, ws, static_cast<hipStream_t>(stream)), "evict launch");
}

size_t akb_attention_shared_workspace(const akb_shape* prefix, const akb_shape* shape, int32_t n)
{
    if (!prefix || !shape || !shape_ok(*prefix) || !shape_ok(*shape) || n < 0 || n > shape->Ncap || !shares_ok(*prefix, *shape)) {
        fail(AKV_EINVAL, "bad shapes, shapes of caches that do not go together, or n out of range 0..Ncap");
        return 0;
    }
    return akb::shared_workspace(*prefix, *shape, n);
}

akv_status akb_attention_shared(const akb_cache* prefix, const akb_cache* cache, const uint16_t* q, const int32_t* n_q, int32_t n, void* out,
                                const akb_params* params, int32_t prefix_max_len, void* workspace, size_t workspace_bytes, void* stream)
{
    if (akv_status st = check_cache(prefix)) return st;
    if (akv_status st = check_cache(cache)) return st;
    const akb_shape &f = prefix->shape, &s = cache->shape;
    if (!shares_ok(f, s))
        return fail(AKV_EINVAL, "prefix and cache do not go together: B %d/%d (the first divides the second), Hq %d/%d, Hkv %d/%d, D %d/%d, dtype %d/%d", f.B, s.B, f.Hq, s.Hq, f.Hkv,
                    s.Hkv, f.D, s.D, f.dtype, s.dtype);
    akb_params p = {};
    if (params) p = *params;
    if (p.accumulate) return fail(AKV_EINVAL, "accumulate is set: a shared prefix has no scores of one sequence");
    if (prefix_max_len < 0 || prefix_max_len > f.Ncap) return fail(AKV_EINVAL, "prefix_max_len = %d out of range 0..the prefix's Ncap", prefix_max_len);
    if (akv_status st = check_attention(s, p, q, n_q, n, out)) return st;
    if (n == 0) return AKV_OK;
    if (akv_status st = check_workspace(workspace, workspace_bytes, akb::shared_workspace(f, s, n))) return st;
    const akb::AttentionArgs a{*cache, q, n_q, n, out, p.out_dtype, 0, p.max_len > 0 ? p.max_len : s.Ncap, scale_bits(p, s.D), static_cast<char*>(workspace)};
    return hip_result(akb::launch_shared(*prefix, prefix_max_len > 0 ? prefix_max_len : f.Ncap, a, static_cast<hipStream_t>(stream)), "shared attention launch");
}

int32_t akb_attention_shared_path(const akb_shape* prefix, const akb_shape* shape, int32_t n, int32_t max_len, int32_t prefix_max_len, int32_t* parts)
{
    if (!prefix || !shape || !shape_ok(*prefix) || !shape_ok(*shape) || !shares_ok(*prefix, *shape) || n < 1 || n > shape->Ncap || max_len < 0 || max_len > shape->Ncap ||
        prefix_max_len < 0 || prefix_max_len > prefix->Ncap)
        return 0;
    return akb::shared_path(*prefix, *shape, n, max_len > 0 ? max_len : shape->Ncap, prefix_max_len > 0 ? prefix_max_len : prefix->Ncap, parts);
}

akv_status akb_append_rotated(const akb_cache* cache, const akb_tokens* tokens, const int32_t* n_new, int32_t n, uint16_t* q_out, const akb_rotary* rotary,
                              void* stream)
{
    if (akv_status st = check_cache(cache)) return st;
    if (!tokens || !rotary) return fail(AKV_EINVAL, "tokens / rotary is NULL");
    const akb_shape& s = cache->shape;
    const akb_tokens& x = *tokens;
    const akb_rotary& r = *rotary;
    if (n < 0 || n > s.Ncap) return fail(AKV_EINVAL, "n = %d out of range 0..Ncap", n);
    if (r.rot < 0 || r.rot > s.D || r.rot % 16 != 0) return fail(AKV_EINVAL, "rot = %d is no multiple of 16 in 0..D", r.rot);
    if (r.rot > 0 && !r.inv_freq) return fail(AKV_EINVAL, "inv_freq is NULL");
    if (r.base && (r.n_base < 1 || s.B % r.n_base != 0)) return fail(AKV_EINVAL, "n_base = %d does not divide B = %d", r.n_base, s.B);
    if (overlap(r.base, size_t(r.n_base) * sizeof(int32_t), cache->lens, size_t(s.B) * sizeof(int32_t))) return fail(AKV_EINVAL, "base shares memory with the lens that the call moves");
    if ((r.q_norm || r.k_norm) && !(std::isfinite(r.eps) && r.eps >= 0.f)) return fail(AKV_EINVAL, "eps is negative or not finite");
    if (!rotated_blocks_ok(s, n)) return fail(AKV_EINVAL, "%d tokens of %d KV heads: 2^23 blocks or more of a sequence", n, s.Hkv);
    if (n == 0) return AKV_OK;
    if (!x.k || !x.v) return fail(AKV_EINVAL, "k / v is NULL");
    if (!x.q != !q_out) return fail(AKV_EINVAL, "one of q and q_out is NULL, the other is not");
    if (!aligned(x.q, 16) || !aligned(x.k, 16) || !aligned(x.v, 16) || !aligned(q_out, 16) || !aligned(r.q_norm, 16) || !aligned(r.k_norm, 16) || !aligned(r.inv_freq, 4) ||
        !aligned(r.base, 4) || !aligned(n_new, 4))
        return fail(AKV_EINVAL, "tokens, q_out and norms must be 16-byte aligned, inv_freq, base and n_new 4-byte aligned");
    for (const int64_t stride : {x.q_seq, x.q_token, x.k_seq, x.k_token, x.v_seq, x.v_token})
        if (stride % 8 != 0 || stride < 0) return fail(AKV_EINVAL, "strides must be multiples of 8 elements, not negative");
    const struct { const uint16_t* p; int64_t seq, token; int heads; } in[] = {{x.q, x.q_seq, x.q_token, s.Hq}, {x.k, x.k_seq, x.k_token, s.Hkv}, {x.v, x.v_seq, x.v_token, s.Hkv}};
    for (const auto& i : in)
        if (q_out && i.p < q_out + size_t(s.B) * s.Hq * n * s.D && q_out < i.p + i.seq * (s.B - 1) + i.token * (n - 1) + int64_t(i.heads) * s.D)
            return fail(AKV_EINVAL, "q_out shares memory with the tokens");
    return hip_result(akb::launch_append_rotated(*cache, x, n_new, n, q_out, r, static_cast<hipStream_t>(stream)), "append launch");
}

int32_t akb_append_rotated_path(const akb_shape* shape, int32_t n, int32_t queries, int32_t* how)
{
    if (!shape || !shape_ok(*shape) || n < 1 || n > shape->Ncap || !rotated_blocks_ok(*shape, n)) return 0;
    return akb::rotated_path(*shape, n, queries != 0, how);
}

akv_status akb_fork(const akb_cache* src, const akb_cache* dst, const int32_t* parents, const int32_t* upto, void* stream)
{
    if (akv_status st = check_cache(src)) return st;
    if (akv_status st = check_cache(dst)) return st;
    const akb_shape &s = src->shape, &d = dst->shape;
    if (s.Hkv != d.Hkv || s.D != d.D || s.dtype != d.dtype) return fail(AKV_EINVAL, "src and dst differ: Hkv %d/%d, D %d/%d, dtype %d/%d", s.Hkv, d.Hkv, s.D, d.D, s.dtype, d.dtype);
    if (!parents && s.B != d.B) return fail(AKV_EINVAL, "parents is NULL and src and dst differ: B %d/%d", s.B, d.B);
    if (!aligned(parents, 4) || !aligned(upto, 4)) return fail(AKV_EINVAL, "parents and upto must be 4-byte aligned");
    if (share_memory(*src, *dst)) return fail(AKV_EINVAL, "src and dst share memory");
    if (overlap(parents, size_t(d.B) * sizeof(int32_t), dst->lens, size_t(d.B) * sizeof(int32_t))) return fail(AKV_EINVAL, "parents shares memory with dst's lens");
    return hip_result(akb::launch_fork(*src, *dst, parents, upto, static_cast<hipStream_t>(stream)), "fork launch");
}

akv_status akb_truncate(const akb_cache* cache, const int32_t* keep, void* stream)
{
    if (akv_status st = check_cache(cache)) return st;
    if (!keep) return fail(AKV_EINVAL, "keep is NULL");
    if (!aligned(keep, 4)) return fail(AKV_EINVAL, "keep must be 4-byte aligned");
    return hip_result(akb::launch_truncate(*cache, keep, static_cast<hipStream_t>(stream)), "truncate launch");
}

akv_status akb_unpack(const akb_cache* cache, uint16_t* k_out, uint16_t* v_out, void* stream)
{
    if (akv_status st = check_cache(cache)) return st;
    if (!k_out && !v_out) return AKV_OK;
    if (!aligned(k_out, 16) || !aligned(v_out, 16)) return fail(AKV_EINVAL, "k_out / v_out must be 16-byte aligned");
    return hip_result(akb::launch_unpack(*cache, k_out, v_out, static_cast<hipStream_t>(stream)), "unpack launch");
}

}  // extern "C"
