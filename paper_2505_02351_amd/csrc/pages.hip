// C ABI of the pages of the caches: blocks copied, accepted branches moved to the front, page tables that fork, grow, shrink and are
// compacted.  Declarations and the meaning of every argument: include/optgqa.h.
#include "optgqa.h"

#include <hip/hip_runtime.h>

#include <algorithm>

#include "host.hpp"
#include "page_kernels.hpp"

using namespace optgqa;

namespace {

// of 4-byte device arrays
bool aligned4(std::initializer_list<const void*> all)
{
    uintptr_t bits = 0;
    for (const void* p : all) bits |= reinterpret_cast<uintptr_t>(p);
    return !(bits & 3u);
}

bool tables_ok(int num_seqs, int max_blocks_per_seq, int num_blocks)
{
    return num_seqs >= 0 && max_blocks_per_seq > 0 && num_blocks > 0 && num_seqs <= most_workgroups(kPageThreads);
}

// a resize counts the blocks that all rows ask for in 32 bits
bool resize_ok(int num_seqs, int max_blocks_per_seq, int num_blocks)
{
    return tables_ok(num_seqs, max_blocks_per_seq, num_blocks) && (int64_t)num_seqs * ((int64_t)max_blocks_per_seq + 1) < (1ll << 31);
}

// workgroups of kPageThreads for the entries of a table's row, `each` a workgroup
unsigned row_parts(int64_t entries, int each) { return (unsigned)std::min<int64_t>(std::max<int64_t>((entries + each - 1) / each, 1), 65535); }

}  // namespace

extern "C" {

int optgqa_copy_blocks(void* const* caches, int num_caches, const int32_t* copies, const int32_t* num_copies, int max_copies, int num_blocks,
                       size_t block_bytes, void* stream)
{
    if (num_caches < 0 || max_copies < 0 || num_blocks <= 0 || block_bytes == 0) return OPTGQA_ERR_SHAPE;
    if (block_bytes % 16 || block_bytes / 16 > (1u << 30)) return OPTGQA_ERR_UNSUPPORTED;
    if (num_caches == 0 || max_copies == 0) return OPTGQA_OK;
    if (!caches || !copies || !num_copies) return OPTGQA_ERR_NULL;
    if (!aligned4({copies, num_copies}) || (reinterpret_cast<uintptr_t>(caches) & 7u)) return OPTGQA_ERR_UNSUPPORTED;
    CopyBlocksParams p;
    p.caches = reinterpret_cast<unsigned char* const*>(caches);
    p.copies = copies;
    p.num_copies = num_copies;
    p.num_caches = num_caches;
    p.max_copies = max_copies;
    p.num_blocks = num_blocks;
    p.pieces = (int)(block_bytes / 16);
    const double units = (double)max_copies * num_caches * ((p.pieces + kCopyUnit - 1) / kCopyUnit);
    const int workgroups = (int)std::min<double>(units, 8.0 * num_cus());
    return launch(copy_blocks_kernel, dim3(workgroups), dim3(kPageThreads), 0, static_cast<hipStream_t>(stream), p);
}

int optgqa_keep_tokens(void* const* caches, int num_caches, const int32_t* block_tables, const int32_t* start_lens, const int32_t* paths,
                       const int32_t* path_lens, int num_seqs, int max_path, int max_blocks_per_seq, int num_blocks, int num_kv_heads, int head_dim,
                       int block_size, int element_bytes, void* stream)
{
    if (num_caches < 0 || num_seqs < 0 || num_seqs > 65535 || max_path < 0 || max_blocks_per_seq <= 0 || num_blocks <= 0 || num_kv_heads <= 0 ||
        num_kv_heads > 65535)
        return OPTGQA_ERR_SHAPE;
    if (!head_dim_ok(head_dim) || !block_size_ok(block_size) || (element_bytes != 1 && element_bytes != 2)) return OPTGQA_ERR_UNSUPPORTED;
    if (num_caches == 0 || num_seqs == 0 || max_path == 0) return OPTGQA_OK;
    if (!caches || !block_tables || !start_lens || !paths || !path_lens) return OPTGQA_ERR_NULL;
    if (!aligned4({block_tables, start_lens, paths, path_lens}) || (reinterpret_cast<uintptr_t>(caches) & 7u)) return OPTGQA_ERR_UNSUPPORTED;
    KeepTokensParams p;
    p.caches = reinterpret_cast<unsigned char* const*>(caches);
    p.block_tables = block_tables;
    p.start_lens = start_lens;
    p.paths = paths;
    p.path_lens = path_lens;
    p.num_caches = num_caches;
    p.max_path = max_path;
    p.num_blocks = num_blocks;
    p.max_blocks_per_seq = max_blocks_per_seq;
    p.num_kv_heads = num_kv_heads;
    p.block_shift = __builtin_ctz(block_size);
    p.pieces_shift = __builtin_ctz(head_dim * element_bytes / 16);
    const int64_t items = (int64_t)num_caches * (num_kv_heads << p.pieces_shift);
    const int64_t workgroups = (items + kPageThreads - 1) / kPageThreads;
    if (workgroups > most_workgroups(kPageThreads)) return OPTGQA_ERR_SHAPE;
    return launch(keep_tokens_kernel, dim3((unsigned)workgroups, num_seqs), dim3(kPageThreads), 0, static_cast<hipStream_t>(stream), p);
}

int optgqa_fork_sequences(int32_t* tables_out, int32_t* lens_out, const int32_t* block_tables, const int32_t* context_lens, int32_t* ref_counts,
                          const int32_t* parents, int num_out, int num_seqs, int max_blocks_per_seq, int num_blocks, int block_size, void* stream)
{
    if (!tables_ok(num_seqs, max_blocks_per_seq, num_blocks) || !tables_ok(num_out, max_blocks_per_seq, num_blocks)) return OPTGQA_ERR_SHAPE;
    if (!block_size_ok(block_size)) return OPTGQA_ERR_UNSUPPORTED;
    if (num_out == 0 && num_seqs == 0) return OPTGQA_OK;
    if (!ref_counts || (num_out && (!tables_out || !lens_out || !parents)) || (num_seqs && (!block_tables || !context_lens))) return OPTGQA_ERR_NULL;
    if (!aligned4({tables_out, lens_out, block_tables, context_lens, ref_counts, parents})) return OPTGQA_ERR_UNSUPPORTED;
    // (rows of the new table are written while others still read the old one)
    struct Range { const int32_t* at; int64_t n; };
    auto apart = [](const Range& a, const Range& b) {
        const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.at), b0 = reinterpret_cast<uintptr_t>(b.at);
        return a.n == 0 || b.n == 0 || a0 + 4 * (uint64_t)a.n <= b0 || b0 + 4 * (uint64_t)b.n <= a0;
    };
    const Range rows{tables_out, (int64_t)num_out * max_blocks_per_seq}, lens{lens_out, num_out};
    const Range others[] = {{block_tables, (int64_t)num_seqs * max_blocks_per_seq}, {context_lens, num_seqs}, {ref_counts, num_blocks}, {parents, num_out}};
    bool all_apart = apart(rows, lens);
    for (const Range& other : others) all_apart = all_apart && apart(rows, other) && apart(lens, other);
    if (!all_apart) return OPTGQA_ERR_SHAPE;
    const ForkParams p{tables_out, lens_out, block_tables, context_lens, ref_counts, parents, num_out, num_seqs, max_blocks_per_seq, num_blocks,
                       __builtin_ctz(block_size)};
    return launch(fork_sequences_kernel, dim3(std::max(num_out, num_seqs), (unsigned)(((int64_t)max_blocks_per_seq + kForkEntries - 1) / kForkEntries)),
                  dim3(kPageThreads), 0, static_cast<hipStream_t>(stream), p);
}

size_t optgqa_resize_workspace_bytes(int num_seqs, int max_blocks_per_seq, int num_blocks)
{
    if (num_seqs <= 0 || !resize_ok(num_seqs, max_blocks_per_seq, num_blocks)) return 0;
    // three numbers a row, and every block that the rows could ask for
    return 4 * (3 * (size_t)num_seqs + (size_t)std::min<int64_t>(num_blocks, (int64_t)num_seqs * ((int64_t)max_blocks_per_seq + 1)));
}

int optgqa_resize_sequences(int32_t* block_tables, int32_t* context_lens, int32_t* ref_counts, const int32_t* new_lens, int64_t* slot_mapping,
                            const int32_t* cu_new_lens, int32_t* copies, int32_t* counts, int num_seqs, int max_blocks_per_seq, int num_blocks,
                            int block_size, int num_slots, int max_change, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!resize_ok(num_seqs, max_blocks_per_seq, num_blocks) || num_slots < 0 || max_change < 0) return OPTGQA_ERR_SHAPE;
    if (!block_size_ok(block_size)) return OPTGQA_ERR_UNSUPPORTED;
    if (!counts || (num_seqs && (!block_tables || !context_lens || !ref_counts || !new_lens || !copies || (slot_mapping && !cu_new_lens))))
        return OPTGQA_ERR_NULL;
    if (!aligned4({block_tables, context_lens, ref_counts, new_lens, cu_new_lens, copies, counts}) || (reinterpret_cast<uintptr_t>(slot_mapping) & 7u))
        return OPTGQA_ERR_UNSUPPORTED;
    if (num_seqs && (!workspace || !aligned16(workspace) || workspace_bytes < optgqa_resize_workspace_bytes(num_seqs, max_blocks_per_seq, num_blocks)))
        return OPTGQA_ERR_WORKSPACE;
    ResizeParams p;
    p.block_tables = block_tables;
    p.context_lens = context_lens;
    p.ref_counts = ref_counts;
    p.new_lens = new_lens;
    p.slots = slot_mapping && num_slots ? slot_mapping : nullptr;
    p.cu_new = cu_new_lens;
    p.copies = copies;
    p.counts = counts;
    p.old_lens = static_cast<int32_t*>(workspace);
    p.last = p.old_lens + num_seqs;
    p.first = p.last + num_seqs;
    p.free_blocks = p.first + num_seqs;
    p.num_seqs = num_seqs;
    p.max_blocks_per_seq = max_blocks_per_seq;
    p.num_blocks = num_blocks;
    p.block_shift = __builtin_ctz(block_size);
    p.num_slots = num_slots;
    p.max_free = (int)std::min<int64_t>(num_blocks, (int64_t)num_seqs * ((int64_t)max_blocks_per_seq + 1));
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (num_seqs <= kPlanThreads && (int64_t)num_seqs * max_change <= kResizeOneTokens)
        return launch(resize_one_kernel, dim3(1), dim3(kPlanThreads), 0, st, p);
    const int64_t most = std::min<int64_t>(max_change, (int64_t)max_blocks_per_seq * block_size);
    int rc = launch(resize_drop_kernel, dim3(num_seqs, row_parts(most / block_size + 1, kPageThreads)), dim3(kPageThreads), 0, st, p);
    if (rc == OPTGQA_OK) rc = launch(resize_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, p);
    if (rc == OPTGQA_OK) rc = launch(resize_apply_kernel, dim3(num_seqs, row_parts(most, 4 * kPageThreads)), dim3(kPageThreads), 0, st, p);
    return rc;
}

size_t optgqa_compact_workspace_bytes(int num_blocks) { return num_blocks > 0 ? 8 * (size_t)num_blocks : 0; }

int optgqa_compact_blocks(int32_t* block_tables, const int32_t* context_lens, int32_t* ref_counts, int32_t* copies, int32_t* counts, int num_seqs,
                          int max_blocks_per_seq, int num_blocks, int block_size, int max_copies, void* workspace, size_t workspace_bytes,
                          void* stream)
{
    if (!tables_ok(num_seqs, max_blocks_per_seq, num_blocks) || max_copies < 0) return OPTGQA_ERR_SHAPE;
    if (!block_size_ok(block_size)) return OPTGQA_ERR_UNSUPPORTED;
    if (!ref_counts || !counts || (max_copies && !copies) || (num_seqs && (!block_tables || !context_lens))) return OPTGQA_ERR_NULL;
    if (!aligned4({block_tables, context_lens, ref_counts, copies, counts})) return OPTGQA_ERR_UNSUPPORTED;
    if (!workspace || !aligned16(workspace) || workspace_bytes < optgqa_compact_workspace_bytes(num_blocks)) return OPTGQA_ERR_WORKSPACE;
    CompactParams p;
    p.block_tables = block_tables;
    p.context_lens = context_lens;
    p.ref_counts = ref_counts;
    p.copies = copies;
    p.counts = counts;
    p.holes = static_cast<int32_t*>(workspace);
    p.to = p.holes + num_blocks;
    p.num_seqs = num_seqs;
    p.max_blocks_per_seq = max_blocks_per_seq;
    p.num_blocks = num_blocks;
    p.block_shift = __builtin_ctz(block_size);
    p.max_copies = max_copies;
    // (a graph's call and a direct one, us, one launch and two: 5 rows of up to 12 blocks 3.4 and 4.7, 6.6 and 8.7; 64 of 95 4.8 and 5.3, 6.5 and 8.7; with a wave to a
    // row, not 16 threads, 64 of 250 7.8 and 6.8, 7.5 and 8.6, 16 of 1 000 6.7 and 6.1, 6.4 and 8.6)
    p.tables_too = num_seqs <= 4 * kPlanWaves && (int64_t)num_seqs * max_blocks_per_seq <= 8192;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int rc = launch(compact_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, p);
    if (rc != OPTGQA_OK || p.tables_too) return rc;
    return launch(compact_tables_kernel, dim3(num_seqs, row_parts(max_blocks_per_seq, 4 * kPageThreads)), dim3(kPageThreads), 0, st, p);
}

}  // extern "C"
