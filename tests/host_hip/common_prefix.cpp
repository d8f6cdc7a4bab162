// The rules by which an attention call with one common prefix is cut into pieces, callable from the tests.
#include "common_prefix_shape.hpp"

using namespace optgqa;

// out: row blocks, row tiles, ranges, keys of a range of the prefix; row blocks, shares of the own parts; pieces, pieces held.  0: refused.
extern "C" int common_plan_of(int64_t num_tokens, int64_t num_seqs, int num_heads, int num_kv_heads, int64_t prefix_len, int64_t max_context_len,
                              int64_t max_q_len, int64_t cus, int64_t* out)
{
    CommonPlan c;
    if (!plan_common(c, num_tokens, num_seqs, num_heads, num_kv_heads, prefix_len, max_context_len, max_q_len, cus)) return 0;
    const int64_t all[] = {c.p_row_waves, c.p_tiles, c.p_splits, c.p_keys, c.s_row_waves, c.s_shares, c.pieces(num_kv_heads), c.held};
    for (int i = 0; i < 8; ++i) out[i] = all[i];
    return 1;
}

// Where the prefix's workgroups of a launch find their work: out[3 n ..] = KV head, range, row tile, or -1.  The number of workgroups.
extern "C" int common_prefix_places(int kv_heads, int ranges, int tiles, int32_t* out)
{
    PrefixItems items;
    items.set(kv_heads, ranges, tiles);
    for (int n = 0; out && n < items.workgroups(); ++n)
        if (!items.place(n, ranges, tiles, out[3 * n], out[3 * n + 1], out[3 * n + 2])) out[3 * n] = out[3 * n + 1] = out[3 * n + 2] = -1;
    return items.workgroups();
}
