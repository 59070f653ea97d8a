// Attention of sequences that go on from shared ones (rules and layout: include/akb.h; rows and parts: akb_rows.h).
#include "akb_rows.h"

namespace akb {

// One walk per (sequence, KV head, row group of 128) over the prefix and the sequence's own blocks, cut where the walks are few.
struct SharedPlan {
    int groups, splits;
    size_t parts, total;   // offset into the workspace, its size
};
static SharedPlan plan(const akb_shape& f, const akb_shape& s, int n, int max_len, int prefix_max_len)
{
    SharedPlan p;
    const long slots = 2L * akv::compute_units(), rows = long(n) * (s.Hq / s.Hkv), pairs = long(s.B) * s.Hkv;
    const long blocks = (prefix_max_len + kTB - 1) / kTB + (max_len + kTB - 1) / kTB;
    p.groups = int((rows + kPromptRows - 1) / kPromptRows);
    p.splits = int(parts_of(pairs * p.groups, blocks, slots));
    p.parts = align256(attention_tickets());
    p.total = p.parts + align256(size_t(2 * slots) * part_floats((int)std::min(rows, long(kPromptRows)), s.D) * sizeof(float));
    return p;
}
size_t shared_workspace(const akb_shape& f, const akb_shape& s, int n) { return plan(f, s, std::max(n, 1), s.Ncap, f.Ncap).total; }

hipError_t launch_shared(const akb_cache& prefix, int prefix_max_len, const AttentionArgs& a, hipStream_t st)
{
    const akb_shape& s = a.c.shape;
    const SharedPlan p = plan(prefix.shape, s, a.n, a.max_len, prefix_max_len);
    const int G = s.Hq / s.Hkv, grid = s.B * s.Hkv * p.groups * p.splits;
    SharedArgs r;
    static_cast<RowArgs&>(r) = RowArgs{a.c, a.q, a.n_q, a.n, p.groups, p.splits, grid, a.out_dtype, a.out, a.c2, uint32_t(G > 1 ? ((uint64_t(1) << 32) + G - 1) / G : 0), nullptr,
                                       reinterpret_cast<float*>(a.ws + p.parts), nullptr, nullptr};
    r.prefix = prefix;
    r.per = s.B / prefix.shape.B;
    if (hipError_t e = launch_prompt_shared(r, grid, st)) return e;
    return p.splits > 1 ? launch_join(r, kPromptRows, st) : hipSuccess;
}

}  // namespace akb
