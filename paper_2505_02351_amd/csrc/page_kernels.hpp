// The pages of the caches: blocks copied, a branch's rows moved to the front, and page tables whose sequences fork, grow, shrink and
// are compacted, all of it on the device.
//
// A pool's state is one number a block: how many table entries hold it (0: it is free).  There is no list of free blocks to keep in
// order: blocks are taken lowest first, so that what a call gives depends on its inputs alone, whatever order its threads run
// in, and used blocks stay together.  Entries that name no block of the pool are passed over.
#pragma once
#include "common.hpp"

namespace optgqa {

constexpr int kPageThreads = 256;
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;

// Counts that other threads of the launch change by atomics are read where atomics work, in L2.
__device__ __forceinline__ int read_count(const int32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void add_count(int32_t* p, int n) { __hip_atomic_fetch_add(p, n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

__device__ __forceinline__ int blocks_of(int tokens, int shift) { return (int)(((int64_t)tokens + (1 << shift) - 1) >> shift); }

// ---- rows of caches ---------------------------------------------------------------------------------------------

struct CopyBlocksParams {
    unsigned char* const* caches;
    const int32_t* copies;      // [max_copies][2]: from, to
    const int32_t* num_copies;
    int num_caches, max_copies, num_blocks;
    int pieces;                 // of a block, 16 bytes each
};

// A unit is 16 KiB of one block of one cache (256 threads, four pieces each); workgroups take them in turn, as many as there are.
constexpr int kCopyPieces = 4, kCopyUnit = kPageThreads * kCopyPieces;
static __global__ __launch_bounds__(kPageThreads) void copy_blocks_kernel(const CopyBlocksParams p)
{
    const int n = min(max(*p.num_copies, 0), p.max_copies), per_block = (p.pieces + kCopyUnit - 1) / kCopyUnit;
    const int64_t units = (int64_t)n * p.num_caches * per_block;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int64_t block = u / per_block;
        const int part = (int)(u - block * per_block), pair = (int)(block / p.num_caches), cache = (int)(block - (int64_t)pair * p.num_caches);
        const int from = p.copies[2 * pair], to = p.copies[2 * pair + 1];
        if ((uint32_t)from >= (uint32_t)p.num_blocks || (uint32_t)to >= (uint32_t)p.num_blocks) continue;
        uint4* const base = reinterpret_cast<uint4*>(p.caches[cache]);
        const uint4* const src = base + (int64_t)from * p.pieces;
        uint4* const dst = base + (int64_t)to * p.pieces;
        const int first = part * kCopyUnit + threadIdx.x;
        uint4 x[kCopyPieces];
#pragma unroll
        for (int i = 0; i < kCopyPieces; ++i)
            if (first + i * kPageThreads < p.pieces) x[i] = src[first + i * kPageThreads];
#pragma unroll
        for (int i = 0; i < kCopyPieces; ++i)
            if (first + i * kPageThreads < p.pieces) dst[first + i * kPageThreads] = x[i];
    }
}

struct KeepTokensParams {
    unsigned char* const* caches;
    const int32_t* block_tables;
    const int32_t* start_lens;
    const int32_t* paths;       // [num_seqs][max_path]
    const int32_t* path_lens;
    int num_caches, max_path, num_blocks, max_blocks_per_seq, num_kv_heads, block_shift;
    int pieces_shift;           // of a row, 16 bytes each (log2)
};

// Row start + paths[i] to row start + i.  Paths ascend, so paths[i] >= i: no row is written before it has been read for a later
// place if, of any run of places, all are read before any is written; and a thread has one 16-byte column of all rows, so that
// nobody else's order matters.
constexpr int kKeepRun = 8;
static __global__ __launch_bounds__(kPageThreads) void keep_tokens_kernel(const KeepTokensParams p)
{
    const int seq = blockIdx.y, per_cache = p.num_kv_heads << p.pieces_shift;
    const int64_t item = (int64_t)blockIdx.x * kPageThreads + threadIdx.x;
    const int cache = (int)(item / per_cache), column = (int)(item - (int64_t)cache * per_cache);
    if (cache >= p.num_caches) return;
    const int head = column >> p.pieces_shift, piece = column & ((1 << p.pieces_shift) - 1);
    uint4* const base = reinterpret_cast<uint4*>(p.caches[cache]) + piece;
    const int start = p.start_lens[seq], count = min(p.path_lens[seq], p.max_path);
    const int32_t* const table = p.block_tables + (int64_t)seq * p.max_blocks_per_seq;
    const int64_t end = (int64_t)p.max_blocks_per_seq << p.block_shift;
    // where a position's row is, in 16-byte pieces; -1: nowhere
    auto at = [&](int64_t pos) __attribute__((always_inline)) -> int64_t {
        if (pos < 0 || pos >= end) return -1;
        const int block = table[pos >> p.block_shift];
        if ((uint32_t)block >= (uint32_t)p.num_blocks) return -1;
        return ((((int64_t)block * p.num_kv_heads + head) << p.block_shift) + (pos & ((1 << p.block_shift) - 1))) << p.pieces_shift;
    };
    for (int i0 = 0; i0 < count; i0 += kKeepRun) {
        uint4 x[kKeepRun];
        int64_t to[kKeepRun];
#pragma unroll
        for (int k = 0; k < kKeepRun; ++k) {
            to[k] = -1;
            if (i0 + k < count) {
                const int from = p.paths[(int64_t)seq * p.max_path + i0 + k];
                if (from > i0 + k) {                             // (equal: it lies there already)
                    const int64_t src = at((int64_t)start + from);
                    to[k] = src < 0 ? -1 : at((int64_t)start + i0 + k);
                    if (to[k] >= 0) x[k] = base[src];
                }
            }
        }
#pragma unroll
        for (int k = 0; k < kKeepRun; ++k)
            if (to[k] >= 0) base[to[k]] = x[k];
    }
}

// ---- page tables ----------------------------------------------------------------------------------------------------

struct ForkParams {
    int32_t* tables_out;
    int32_t* lens_out;
    const int32_t* block_tables;
    const int32_t* context_lens;
    int32_t* ref_counts;
    const int32_t* parents;
    int num_out, num_seqs, max_blocks_per_seq, num_blocks, block_shift;
};

__device__ __forceinline__ int clamped(int len, int max_blocks, int shift) { return (int)min((int64_t)max(len, 0), (int64_t)max_blocks << shift); }

// Row r of both tables: of the new one, what it takes over; of the old one, its blocks' holders, which change by the rows that take it
// over less itself.  (Sums of whole numbers: the same in any order.)
constexpr int kForkEntries = 1024;      // of a row, to a workgroup
static __global__ __launch_bounds__(kPageThreads) void fork_sequences_kernel(const ForkParams p)
{
    const int r = blockIdx.x, first = blockIdx.y * kForkEntries, lane = threadIdx.x & 63;
    __shared__ int sums[kPageThreads / 64];
    if (r < p.num_out) {
        const int from = p.parents[r];
        const bool there = (uint32_t)from < (uint32_t)p.num_seqs;
        const int len = there ? clamped(p.context_lens[from], p.max_blocks_per_seq, p.block_shift) : 0, n = blocks_of(len, p.block_shift);
        if (blockIdx.y == 0 && threadIdx.x == 0) p.lens_out[r] = len;
        const int32_t* const src = p.block_tables + (int64_t)(there ? from : 0) * p.max_blocks_per_seq;
        int32_t* const dst = p.tables_out + (int64_t)r * p.max_blocks_per_seq;
        for (int j = first + threadIdx.x; j < min(first + kForkEntries, n); j += kPageThreads) dst[j] = src[j];
    }
    if (r >= p.num_seqs) return;
    const int n = blocks_of(clamped(p.context_lens[r], p.max_blocks_per_seq, p.block_shift), p.block_shift);
    if (first >= n) return;
    int heirs = 0;
    for (int i = threadIdx.x; i < p.num_out; i += kPageThreads) heirs += p.parents[i] == r;
    heirs = wave_sum(heirs);
    if (lane == 0) sums[threadIdx.x >> 6] = heirs;
    __syncthreads();
    int change = -1;
#pragma unroll
    for (int w = 0; w < kPageThreads / 64; ++w) change += sums[w];
    if (change == 0) return;
    const int32_t* const row = p.block_tables + (int64_t)r * p.max_blocks_per_seq;
    for (int j = first + threadIdx.x; j < min(first + kForkEntries, n); j += kPageThreads) {
        const int block = row[j];
        if ((uint32_t)block < (uint32_t)p.num_blocks) add_count(p.ref_counts + block, change);
    }
}

// Exclusive sums over the threads of a workgroup of kPlanThreads; `all`: over all of them.  Between barriers of its own.
__device__ __forceinline__ int plan_sums(int x, int* lds, int& all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sum = lane_sums(x);
    __syncthreads();                                             // (lds is free again)
    if (lane == 63) lds[wave] = sum;
    __syncthreads();
    int before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < kPlanWaves; ++w) {
        const int s = lds[w];
        before += w < wave ? s : 0;
        all += s;
    }
    return before + sum - x;
}

// Every thread of the workgroup sees what the others stored or changed by atomics before.
__device__ __forceinline__ void plan_barrier()
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

struct ResizeParams {
    int32_t* block_tables;
    int32_t* context_lens;
    int32_t* ref_counts;
    const int32_t* new_lens;
    int64_t* slots;             // or nullptr
    const int32_t* cu_new;      // [num_seqs + 1]
    int32_t* copies;            // [num_seqs][2]
    int32_t* counts;            // copies, blocks lacking
    int32_t *old_lens, *replaced, *first;       // workspace, [num_seqs]: lengths before; the shared last block that a row replaces, or -1; its first new block's number
    int32_t* free_blocks;       // workspace, [max_free]
    int num_seqs, max_blocks_per_seq, num_blocks, block_shift, num_slots, max_free;
    __device__ __forceinline__ int old_len(int r) const { return clamped(context_lens[r], max_blocks_per_seq, block_shift); }
    __device__ __forceinline__ int new_len(int r) const { return clamped(new_lens[r], max_blocks_per_seq, block_shift); }
};

// Entries behind the new lengths are given back: row r, entries from the `first`-th such on, `step` apart.
__device__ __forceinline__ void resize_drop(const ResizeParams& p, int r, int first, int step)
{
    const int32_t* const row = p.block_tables + (int64_t)r * p.max_blocks_per_seq;
    const int have = blocks_of(p.old_len(r), p.block_shift), need = blocks_of(p.new_len(r), p.block_shift);
    for (int j = need + first; j < have; j += step) {
        const int block = row[j];
        if ((uint32_t)block < (uint32_t)p.num_blocks) add_count(p.ref_counts + block, -1);
    }
}

// Which blocks the growing rows get.  One workgroup.
__device__ __forceinline__ void resize_plan(const ResizeParams& p)
{
    __shared__ int lds[kPlanWaves];
    const int S = p.num_seqs, shift = p.block_shift, bmask = (1 << shift) - 1;
    // Rows whose last block is not full, is about to be written and is held by others too.  Each gives it up; where all of a block's
    // holders have done so, the last of them by number keeps it: the count, now 0, becomes the least -(1 + row).
    for (int r = threadIdx.x; r < S; r += kPlanThreads) {
        const int old = p.old_len(r);
        int last = -1;
        if (p.new_len(r) > old && (old & bmask)) {
            last = p.block_tables[(int64_t)r * p.max_blocks_per_seq + (old >> shift)];
            if ((uint32_t)last >= (uint32_t)p.num_blocks || read_count(p.ref_counts + last) <= 1) last = -1;
        }
        p.replaced[r] = last;
        p.old_lens[r] = old;
    }
    plan_barrier();
    for (int r = threadIdx.x; r < S; r += kPlanThreads)
        if (p.replaced[r] >= 0) add_count(p.ref_counts + p.replaced[r], -1);
    plan_barrier();
    for (int r = threadIdx.x; r < S; r += kPlanThreads) {
        const int last = p.replaced[r];
        if (last >= 0 && read_count(p.ref_counts + last) <= 0)
            __hip_atomic_fetch_min(p.ref_counts + last, -(1 + r), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    plan_barrier();
    // what each row asks for, numbered by rows; a replaced block comes first
    int wanted = 0, copies = 0;
    for (int r0 = 0; r0 < S; r0 += kPlanThreads) {
        const int r = r0 + threadIdx.x;
        int wants = 0, copy = 0;
        if (r < S) {
            const int last = p.replaced[r], old = p.old_lens[r];
            if (last >= 0) {
                if (read_count(p.ref_counts + last) == -(1 + r)) p.replaced[r] = -1 - (last + 1);        // keeps it: put right below
                else copy = 1;
            }
            wants = copy + max(blocks_of(p.new_len(r), shift) - blocks_of(old, shift), 0);
        }
        int all;
        const int at = wanted + plan_sums(wants, lds, all);
        wanted += all;
        if (r < S) p.first[r] = at;
        copies += plan_sums(copy, lds, all);                     // (of this thread's rows: put right below)
    }
    (void)copies;
    plan_barrier();
    for (int r = threadIdx.x; r < S; r += kPlanThreads) {
        const int last = p.replaced[r];
        if (last < -1) {
            p.ref_counts[-2 - last] = 1;
            p.replaced[r] = -1;
        }
    }
    plan_barrier();
    // the lowest free blocks, as many as are asked for
    int found = 0;
    for (int b0 = 0; b0 < p.num_blocks && found < wanted; b0 += 4 * kPlanThreads) {
        const int b = b0 + 4 * threadIdx.x;
        int n[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) n[i] = b + i < p.num_blocks ? p.ref_counts[b + i] : 1;
        int all, at = found + plan_sums((n[0] == 0) + (n[1] == 0) + (n[2] == 0) + (n[3] == 0), lds, all);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n[i] == 0) {
                if (at < p.max_free) p.free_blocks[at] = b + i;
                ++at;
            }
        found += all;
    }
    plan_barrier();
    const bool enough = found >= wanted;
    // copies are numbered by rows, a wave to a row from here on
    int copy0 = 0;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int r0 = 0; r0 < S; r0 += kPlanThreads) {
        const int r = r0 + threadIdx.x;
        const int last = r < S ? p.replaced[r] : -1;
        int all;
        const int at = copy0 + plan_sums(last >= 0 ? 1 : 0, lds, all);
        copy0 += all;
        if (last < 0) continue;
        if (enough) {
            p.copies[2 * at] = last;
            p.copies[2 * at + 1] = p.free_blocks[p.first[r]];
        } else {
            add_count(p.ref_counts + last, 1);                   // it stays
        }
    }
    if (threadIdx.x == 0) {
        p.counts[0] = enough ? copy0 : 0;
        p.counts[1] = enough ? 0 : wanted - found;
    }
    for (int r = wave; r < S; r += kPlanWaves) {
        const int old = p.old_lens[r], now = p.new_len(r);
        if (now > old && enough) {
            int32_t* const row = p.block_tables + (int64_t)r * p.max_blocks_per_seq;
            const int copy = p.replaced[r] >= 0 ? 1 : 0, have = blocks_of(old, shift) - copy, n = blocks_of(now, shift) - have, at = p.first[r];
            for (int i = lane; i < n; i += 64) {
                const int block = p.free_blocks[at + i];
                row[have + i] = block;
                p.ref_counts[block] = 1;
            }
        }
        if (lane == 0 && (now <= old || enough)) p.context_lens[r] = now;
    }
}

// Slots of the new tokens of row r: those from the `first`-th on, `step` apart.
__device__ __forceinline__ void resize_slots(const ResizeParams& p, int r, int first, int step)
{
    const int32_t* const row = p.block_tables + (int64_t)r * p.max_blocks_per_seq;
    const int old = p.old_lens[r], grown = p.context_lens[r] - old, begin = max(p.cu_new[r], 0), end = min(p.cu_new[r + 1], p.num_slots);
    for (int i = first; i < end - begin; i += step) {
        int64_t slot = -1;
        if (i < grown) slot = ((int64_t)row[(old + i) >> p.block_shift] << p.block_shift) + ((old + i) & ((1 << p.block_shift) - 1));
        p.slots[begin + i] = slot;
    }
}

// All of it in one workgroup, for changes of a few tokens.
constexpr int64_t kResizeOneTokens = 4096;      // rows times the most that one changes by
static __global__ __launch_bounds__(kPlanThreads) void resize_one_kernel(const ResizeParams p)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int r = wave; r < p.num_seqs; r += kPlanWaves) resize_drop(p, r, lane, 64);
    plan_barrier();
    resize_plan(p);
    if (!p.slots) return;
    plan_barrier();
    for (int r = wave; r < p.num_seqs; r += kPlanWaves) resize_slots(p, r, lane, 64);
}

// The same in three launches: rows x parts of a row, the plan, rows x parts.
static __global__ __launch_bounds__(kPageThreads) void resize_drop_kernel(const ResizeParams p)
{
    resize_drop(p, blockIdx.x, blockIdx.y * kPageThreads + threadIdx.x, gridDim.y * kPageThreads);
}
static __global__ __launch_bounds__(kPlanThreads) void resize_plan_kernel(const ResizeParams p) { resize_plan(p); }
static __global__ __launch_bounds__(kPageThreads) void resize_slots_kernel(const ResizeParams p)
{
    resize_slots(p, blockIdx.x, blockIdx.y * kPageThreads + threadIdx.x, gridDim.y * kPageThreads);
}

struct CompactParams {
    int32_t* block_tables;
    const int32_t* context_lens;
    int32_t* ref_counts;
    int32_t* copies;
    int32_t* counts;            // copies, blocks in use
    int32_t *holes, *to;        // workspace, [num_blocks] each: free blocks below the number in use; where a block from there on goes
    int num_seqs, max_blocks_per_seq, num_blocks, block_shift, max_copies;
};

// Of U blocks in use, the i-th highest goes to the i-th lowest free one, as far as that is below U.  One workgroup.
static __global__ __launch_bounds__(kPlanThreads) void compact_plan_kernel(const CompactParams p)
{
    __shared__ int lds[kPlanWaves];
    int used = 0, all;
    for (int b = threadIdx.x; b < p.num_blocks; b += kPlanThreads) used += p.ref_counts[b] > 0;
    plan_sums(used, lds, used);
    int holes = 0;
    for (int b0 = 0; b0 < used; b0 += kPlanThreads) {
        const int b = b0 + threadIdx.x;
        const bool hole = b < used && p.ref_counts[b] <= 0;
        const int at = holes + plan_sums(hole, lds, all);
        holes += all;
        if (hole) p.holes[at] = b;
    }
    plan_barrier();
    const int copies = min(holes, p.max_copies);
    int movers = 0;
    for (int b0 = p.num_blocks - 1; b0 >= used; b0 -= kPlanThreads) {
        const int b = b0 - threadIdx.x, held = b >= used ? p.ref_counts[b] : 0;
        const int at = movers + plan_sums(held > 0, lds, all);
        movers += all;
        if (b < used) continue;
        const bool moves = held > 0 && at < copies;
        const int to = moves ? p.holes[at] : b;
        p.to[b] = to;
        if (moves) {
            p.copies[2 * at] = b;
            p.copies[2 * at + 1] = to;
            p.ref_counts[to] = held;
            p.ref_counts[b] = 0;
        }
    }
    if (threadIdx.x == 0) {
        p.counts[0] = copies;
        p.counts[1] = used;
    }
}

static __global__ __launch_bounds__(kPageThreads) void compact_tables_kernel(const CompactParams p)
{
    const int used = p.counts[1], n = blocks_of(clamped(p.context_lens[blockIdx.x], p.max_blocks_per_seq, p.block_shift), p.block_shift);
    int32_t* const row = p.block_tables + (int64_t)blockIdx.x * p.max_blocks_per_seq;
    for (int j = blockIdx.y * kPageThreads + threadIdx.x; j < n; j += gridDim.y * kPageThreads) {
        const int block = row[j];
        if (block >= used && block < p.num_blocks) row[j] = p.to[block];
    }
}

}  // namespace optgqa
