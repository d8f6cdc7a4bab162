// The rules by which an attention call for trees of new tokens is cut into pieces, callable from the tests.
#include "common_prefix_shape.hpp"

using namespace optgqa;

// out: row tiles, ranges, keys of a range of the prefix; pieces, pieces held.  0: refused.
extern "C" int tree_plan_of(int64_t num_tokens, int64_t num_seqs, int num_heads, int num_kv_heads, int64_t prefix_len, int64_t max_context_len,
                            int64_t max_q_len, int64_t cus, int64_t* out)
{
    CommonPlan c;
    if (!plan_common(c, num_tokens, num_seqs, num_heads, num_kv_heads, prefix_len, max_context_len, max_q_len, cus, true)) return 0;
    const int64_t all[] = {c.p_tiles, c.p_splits, c.p_keys, c.pieces(num_kv_heads), c.held};
    for (int i = 0; i < 5; ++i) out[i] = all[i];
    return 1;
}
