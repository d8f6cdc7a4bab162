// How long the pieces of an attention call for trees of new tokens are, callable from the tests.
#include "common_prefix_shape.hpp"

using namespace optgqa;

// out: rows of a KV head in 32s; row blocks of a workgroup, row tiles, ranges and keys of a range of the prefix; row blocks at most, shares of
// own parts; whether it is one launch.  0: refused.
extern "C" int tree_walk_plan(int64_t num_tokens, int64_t num_seqs, int num_heads, int num_kv_heads, int64_t prefix_len, int64_t max_context_len,
                              int64_t max_q_len, int64_t cus, int64_t* out)
{
    CommonPlan c;
    if (!plan_common(c, num_tokens, num_seqs, num_heads, num_kv_heads, prefix_len, max_context_len, max_q_len, cus, true)) return 0;
    const int64_t all[] = {c.p_slots, c.p_row_waves, c.p_tiles, c.p_splits, c.p_keys, c.s_row_waves, c.s_shares, c.direct_workgroups > 0};
    for (int i = 0; i < 8; ++i) out[i] = all[i];
    return 1;
}
extern "C" int tree_walk_one_piece(int steps, int share) { return tree_one_piece(steps, share); }
extern "C" int tree_walk_row_waves(int64_t rows) { return common_row_waves(rows); }
