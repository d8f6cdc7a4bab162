// A resize's last part - a row's new blocks, its length and its new tokens' slots - callable from the tests, one thread at a time.
#include "hip/hip_runtime.h"

#define __hip_atomic_load(p, ...) (*(p))
#define __hip_atomic_fetch_add(p, n, ...) (*(p) += (n))
#define __hip_atomic_fetch_min(p, n, ...) (*(p) = std::min(*(p), (n)))
#define __syncthreads_or(x) (x)
#define __builtin_amdgcn_ballot_w64(x) ((x) ? 1ull : 0ull)
#define __builtin_amdgcn_mbcnt_hi(m, x) (x)
#define __builtin_amdgcn_mbcnt_lo(m, x) (x)
inline dim3 gridDim;
#include "page_kernels.hpp"

using namespace optgqa;

// Row 0, `old` tokens long, which a plan gives the blocks `fresh` (enough: they are there); last: its shared last block, or -1.
extern "C" void resize_apply_of(int32_t* table, int32_t* length, int32_t* ref_counts, int32_t new_len, int64_t* slots, const int32_t* cu_new,
                                int num_slots, int max_blocks_per_seq, int num_blocks, int block_shift, int old, int last, const int32_t* fresh,
                                int enough, int step)
{
    ResizeParams p = {};
    p.block_tables = table;
    p.context_lens = length;
    p.ref_counts = ref_counts;
    p.new_lens = &new_len;
    p.slots = slots;
    p.cu_new = cu_new;
    p.max_blocks_per_seq = max_blocks_per_seq;
    p.num_blocks = num_blocks;
    p.block_shift = block_shift;
    p.num_slots = num_slots;
    int32_t zero = 0;
    const ResizeRows rows{&old, &last, &zero, fresh};
    for (int from = step - 1; from >= 0; --from) resize_apply(p, rows, 0, enough != 0, from, step);
}
