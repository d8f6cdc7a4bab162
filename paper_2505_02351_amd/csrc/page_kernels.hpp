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

__device__ __forceinline__ void stream_store16(void* p, uint4 x)
{
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    const u32x4 v = {x.x, x.y, x.z, x.w};
    __builtin_nontemporal_store(v, static_cast<u32x4*>(p));
}

struct CopyBlocksParams {
    unsigned char* const* caches;
    const int32_t* copies;      // [max_copies][2]: from, to
    const int32_t* num_copies;
    int num_caches, max_copies, num_blocks;
    int pieces;                 // of a block, 16 bytes each
};

// A unit is 16 KiB of one block of one cache (256 threads, four pieces each); workgroups take them in turn, eight to a CU.  Memory bounds it: 750 blocks of
// 32 KiB in 32 caches, 1.57 GB read and written, 311 us, 5.05 TB/s, where one large copy does 5.15.  (The whole pass 322 us; 336 through the caches, 318 with
// a workgroup to each unit, which costs the usual call, whose bound is far above what there is to copy; 8 KiB units 385, 32 KiB 511.)
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
            if (first + i * kPageThreads < p.pieces) x[i] = stream_load16(src + first + i * kPageThreads);
#pragma unroll
        for (int i = 0; i < kCopyPieces; ++i)
            if (first + i * kPageThreads < p.pieces) stream_store16(dst + first + i * kPageThreads, x[i]);
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
// What bounds it are round trips one after another, four to a row: its path, its two block numbers, itself.  `x` is set under conditions and lies in scratch
// (144 bytes a lane), so that a row is waited for before the next one's path is asked for.  64 sequences, 249 tokens that move in 32 caches of 8 heads of 128
// (33 MB): 19 us, 17 - 18 a pass among others, where 33 MB take 6.6.  (Asking for a run's block numbers at once, the rows still in scratch, changed nothing there and
// cost 1.4 us where one small tree is all there is: 2.1 us.)
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
// of a row, to a workgroup (256 rows of up to 2 048 blocks, the call with its copy: 256 11.1 us, 512 10.8, 1 024 11.4, 2 048 12.2)
constexpr int kForkEntries = 512;
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
    const int of_lane = lds[lane & (kPlanWaves - 1)], sums = lane_sums(lane < kPlanWaves ? of_lane : 0);
    all = __builtin_amdgcn_readlane(sums, kPlanWaves - 1);
    return __builtin_amdgcn_readlane(sums, __builtin_amdgcn_readfirstlane(wave)) - __builtin_amdgcn_readlane(sum, 63) + sum - x;
}

// Every thread of the workgroup sees what the others stored or changed by atomics before.
__device__ __forceinline__ void plan_barrier()
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// Blocks begin .. end - 1 whose count `wanted` names, in ascending order: emit(block, how many of them come before it, count), until `most` have been
// met or passed -> how many there were.  One workgroup; the counts of a round are asked for a round ahead.  (What bounds such kernels of one workgroup is
// round trips to memory, those for their own instructions too: four counts to a thread and round, 16 in straight lines cost 4 us more.)
constexpr int kScanLoads = 4, kScanBlocks = kPlanThreads * kScanLoads;
template <typename Wanted, typename Emit>
__device__ __forceinline__ int plan_scan(const int32_t* ref_counts, int begin, int end, int most, int* lds, Wanted wanted, Emit emit)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int met = 0, n[kScanLoads], next[kScanLoads];
    auto ask = [&](int64_t first) __attribute__((always_inline)) {       // (past the end: the last one again)
#pragma unroll
        for (int i = 0; i < kScanLoads; ++i) next[i] = ref_counts[min(first + 64 * i, (int64_t)end - 1)];
    };
    if (begin < end && most > 0) ask((int64_t)begin + wave * (64 * kScanLoads) + lane);
#pragma unroll 1
    for (int64_t round = begin; round < end && met < most; round += kScanBlocks) {
        const int64_t first = round + wave * (64 * kScanLoads) + lane;
#pragma unroll
        for (int i = 0; i < kScanLoads; ++i) n[i] = next[i];
        if (round + kScanBlocks < end) ask(first + kScanBlocks);
        uint64_t mask[kScanLoads];
        int mine = 0;
#pragma unroll
        for (int i = 0; i < kScanLoads; ++i) {
            mask[i] = __builtin_amdgcn_ballot_w64(first + 64 * i < end && wanted(n[i]));
            mine += __builtin_popcountll(mask[i]);
        }
        __syncthreads();                                         // (lds is free again)
        if (lane == 0) lds[wave] = mine;
        __syncthreads();
        const int of_lane = lds[lane & (kPlanWaves - 1)];        // (a lane's sum over the waves before its own, by one wave's sums)
        const int sums = lane_sums(lane < kPlanWaves ? of_lane : 0);
        int at = met + __builtin_amdgcn_readlane(sums, wave) - mine;
        met += __builtin_amdgcn_readlane(sums, kPlanWaves - 1);
#pragma unroll
        for (int i = 0; i < kScanLoads; ++i) {
            if (mask[i] >> lane & 1) emit((int)(first + 64 * i), at + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask[i] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask[i], 0u)), n[i]);
            at += __builtin_popcountll(mask[i]);
        }
    }
    return met;
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
    int32_t *old_lens, *last, *first;           // workspace, [num_seqs]: ResizeRows
    int32_t* free_blocks;       // workspace, [max_free]
    int num_seqs, max_blocks_per_seq, num_blocks, block_shift, num_slots, max_free;
    __device__ __forceinline__ int old_len(int r) const { return clamped(context_lens[r], max_blocks_per_seq, block_shift); }
    __device__ __forceinline__ int new_len(int r) const { return clamped(new_lens[r], max_blocks_per_seq, block_shift); }
};

// What is known of the rows between the parts of a resize: lengths before; the shared last block that a row replaces, or -1; the number
// of its first new block among all new ones; and those.
struct ResizeRows {
    int32_t *old_lens, *last, *first;
    const int32_t* free_blocks;
};

// Entries behind the new lengths are given back: those from the `from`-th such on, `step` apart.
__device__ __forceinline__ void resize_drop(const ResizeParams& p, int r, int old, int now, int from, int step)
{
    const int32_t* const row = p.block_tables + (int64_t)r * p.max_blocks_per_seq;
    const int have = blocks_of(old, p.block_shift), need = blocks_of(now, p.block_shift);
    for (int j = need + from; j < have; j += step) {
        const int block = row[j];
        if ((uint32_t)block < (uint32_t)p.num_blocks) add_count(p.ref_counts + block, -1);
    }
}

// A row's new blocks and the slots of its new tokens, from the `from`-th on, `step` apart.
__device__ __forceinline__ void resize_apply(const ResizeParams& p, const ResizeRows& rows, int r, bool enough, int from, int step)
{
    const int old = rows.old_lens[r], now = p.new_len(r), shift = p.block_shift;
    const int have = blocks_of(old, shift) - (rows.last[r] >= 0 ? 1 : 0);        // blocks that it keeps
    int32_t* const row = p.block_tables + (int64_t)r * p.max_blocks_per_seq;
    const int32_t* const fresh = rows.free_blocks + rows.first[r];
    const bool grows = now > old && enough;
    if (grows)
        for (int i = from, n = blocks_of(now, shift) - have; i < n; i += step) {
            const int block = fresh[i];
            row[have + i] = block;
            p.ref_counts[block] = 1;
        }
    if (from == 0 && (now <= old || enough)) p.context_lens[r] = now;
    if (!p.slots) return;
    const int begin = max(p.cu_new[r], 0), end = max(min(p.cu_new[r + 1], p.num_slots), 0);
    // of the first tokens, where they fill a block (an entry that names none: they have no row, and the cache stores pass over slots below 0 alone)
    int kept = grows && have > 0 && (old >> shift) == have - 1 ? row[have - 1] : 0;
    if ((uint32_t)kept >= (uint32_t)p.num_blocks) kept = -1;
    const int grown = grows ? now - old : 0;                     // (lengths go up to 2^31 - 1, positions behind them would not)
    for (int i = from; i < end - begin; i += step) {
        int64_t slot = -1;
        if (i < grown) {
            const int pos = old + i, j = pos >> shift, block = j < have ? kept : fresh[j - have];
            if (block >= 0) slot = ((int64_t)block << shift) + (pos & ((1 << shift) - 1));
        }
        p.slots[begin + i] = slot;
    }
}

// Which blocks the growing rows get -> whether there are as many.  One workgroup.  ONE: what is known of the rows stays in LDS, up to
// kPlanThreads of them, and what they give back is given back here.
constexpr int kPlanFree = 4096;         // new blocks that LDS holds
template <bool ONE> __device__ __forceinline__ bool resize_plan(const ResizeParams& p, ResizeRows& rows)
{
    __shared__ int lds[kPlanWaves];
    __shared__ int32_t lds_rows[ONE ? 3 : 1][ONE ? kPlanThreads : 1], lds_free[ONE ? kPlanFree : 1];
    const int S = p.num_seqs, shift = p.block_shift, bmask = (1 << shift) - 1;
    rows = ONE ? ResizeRows{lds_rows[0], lds_rows[1], lds_rows[2], lds_free} : ResizeRows{p.old_lens, p.last, p.first, p.free_blocks};
    // (`first` holds the new lengths until it is known)
    int32_t* const news = rows.first;
    bool drops = false;
    for (int r = threadIdx.x; r < S; r += kPlanThreads) {
        const int old = p.old_len(r), now = p.new_len(r);
        int last = -1;
        if (now > old && (old & bmask)) last = p.block_tables[(int64_t)r * p.max_blocks_per_seq + (old >> shift)];
        rows.old_lens[r] = old;
        rows.last[r] = (uint32_t)last < (uint32_t)p.num_blocks ? last : -1;
        news[r] = now;
        drops = drops || blocks_of(now, shift) < blocks_of(old, shift);
    }
    if (ONE && __syncthreads_or(drops)) {
        for (int r = threadIdx.x >> 4; r < S; r += kPlanThreads / 16) resize_drop(p, r, rows.old_lens[r], news[r], threadIdx.x & 15, 16);
        plan_barrier();
    }
    // Rows whose last block is not full, is about to be written and is held by others too.  Each gives it up; where all of a block's
    // holders have done so, the last of them by number keeps it: the count, now 0, becomes the least -(1 + row).
    bool shared = false;
    for (int r = threadIdx.x; r < S; r += kPlanThreads) {
        const int last = rows.last[r];
        if (last >= 0 && read_count(p.ref_counts + last) <= 1) rows.last[r] = -1;
        shared = shared || rows.last[r] >= 0;
    }
    shared = __syncthreads_or(shared);
    if (shared) {
        for (int r = threadIdx.x; r < S; r += kPlanThreads)
            if (rows.last[r] >= 0) add_count(p.ref_counts + rows.last[r], -1);
        plan_barrier();
        for (int r = threadIdx.x; r < S; r += kPlanThreads) {
            const int last = rows.last[r];
            if (last >= 0 && read_count(p.ref_counts + last) <= 0)
                __hip_atomic_fetch_min(p.ref_counts + last, -(1 + r), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        plan_barrier();
        for (int r = threadIdx.x; r < S; r += kPlanThreads) {
            const int last = rows.last[r];
            if (last >= 0 && read_count(p.ref_counts + last) == -(1 + r)) rows.last[r] = -2 - last;
        }
        __syncthreads();                                         // (all have looked)
        for (int r = threadIdx.x; r < S; r += kPlanThreads) {
            const int last = rows.last[r];
            if (last < -1) {
                p.ref_counts[-2 - last] = 1;
                rows.last[r] = -1;
            }
        }
        plan_barrier();
    }
    // what each row asks for, numbered by rows; a replaced block comes first
    int wanted = 0;
    for (int r0 = 0; r0 < S; r0 += kPlanThreads) {
        const int r = r0 + threadIdx.x;
        int wants = 0;
        if (r < S) wants = (rows.last[r] >= 0) + max(blocks_of(news[r], shift) - blocks_of(rows.old_lens[r], shift), 0);
        int all;
        const int at = wanted + plan_sums(wants, lds, all);
        wanted += all;
        if (r < S) rows.first[r] = at;
    }
    // the lowest free blocks, as many as are asked for
    int32_t* const free = ONE && wanted <= kPlanFree ? lds_free : p.free_blocks;
    const int room = ONE && wanted <= kPlanFree ? kPlanFree : p.max_free;
    rows.free_blocks = free;
    const int found = plan_scan(p.ref_counts, 0, p.num_blocks, wanted, lds, [](int n) { return n == 0; },
                                [&](int block, int at, int) __attribute__((always_inline)) { if (at < room) free[at] = block; });
    plan_barrier();
    const bool enough = found >= wanted;
    int copies = 0;
    if (shared)
        for (int r0 = 0; r0 < S; r0 += kPlanThreads) {
            const int r = r0 + threadIdx.x, last = r < S ? rows.last[r] : -1;
            int all;
            const int at = copies + plan_sums(last >= 0 ? 1 : 0, lds, all);
            copies += all;
            if (last < 0) continue;
            if (enough) {
                p.copies[2 * at] = last;
                p.copies[2 * at + 1] = free[rows.first[r]];
            } else {
                add_count(p.ref_counts + last, 1);               // it stays
            }
        }
    if (threadIdx.x == 0) {
        p.counts[0] = enough ? copies : 0;
        p.counts[1] = enough ? 0 : wanted - found;
    }
    return enough;
}

// All of it in one workgroup, for changes of a few tokens.
constexpr int64_t kResizeOneTokens = 4096;      // rows times the most that one changes by
static __global__ __launch_bounds__(kPlanThreads) void resize_one_kernel(const ResizeParams p)
{
    ResizeRows rows;
    const bool enough = resize_plan<true>(p, rows);
    // (16 threads to a row, so that 64 rows' round trips are one another's: a step of 64 rows 10.4 us with a wave to a row, 7.7 so)
    for (int r = threadIdx.x >> 4; r < p.num_seqs; r += kPlanThreads / 16) resize_apply(p, rows, r, enough, threadIdx.x & 15, 16);
}

// The same in three launches: rows x parts of a row, the plan, rows x parts.
static __global__ __launch_bounds__(kPageThreads) void resize_drop_kernel(const ResizeParams p)
{
    resize_drop(p, blockIdx.x, p.old_len(blockIdx.x), p.new_len(blockIdx.x), blockIdx.y * kPageThreads + threadIdx.x, gridDim.y * kPageThreads);
}
static __global__ __launch_bounds__(kPlanThreads) void resize_plan_kernel(const ResizeParams p)
{
    ResizeRows rows;
    resize_plan<false>(p, rows);
}
static __global__ __launch_bounds__(kPageThreads) void resize_apply_kernel(const ResizeParams p)
{
    const ResizeRows rows{p.old_lens, p.last, p.first, p.free_blocks};
    resize_apply(p, rows, blockIdx.x, p.counts[1] == 0, blockIdx.y * kPageThreads + threadIdx.x, gridDim.y * kPageThreads);
}

struct CompactParams {
    int32_t* block_tables;
    const int32_t* context_lens;
    int32_t* ref_counts;
    int32_t* copies;
    int32_t* counts;            // copies, blocks in use
    int32_t *holes, *to;        // workspace, [num_blocks] each: free blocks below the number in use; where a block from there on goes
    int num_seqs, max_blocks_per_seq, num_blocks, block_shift, max_copies;
    bool tables_too;            // few entries: the plan's workgroup changes them as well
};

// Entries of row r, from the `from`-th on, `step` apart.
__device__ __forceinline__ void compact_row(const CompactParams& p, int used, int r, int from, int step)
{
    const int n = blocks_of(clamped(p.context_lens[r], p.max_blocks_per_seq, p.block_shift), p.block_shift);
    int32_t* const row = p.block_tables + (int64_t)r * p.max_blocks_per_seq;
    for (int j = from; j < n; j += step) {
        const int block = row[j];
        if (block >= used && block < p.num_blocks) row[j] = p.to[block];
    }
}

// Of U blocks in use, the i-th highest goes to the i-th lowest free one, as far as that is below U.  (As many are in use from U on as are free below
// it: what comes a-th from U on is the (holes - 1 - a)-th highest.)  One workgroup.
static __global__ __launch_bounds__(kPlanThreads) void compact_plan_kernel(const CompactParams p)
{
    __shared__ int lds[kPlanWaves];
    int mine = 0, used;
#pragma unroll 4
    for (int64_t b = threadIdx.x; b < p.num_blocks; b += kPlanThreads) mine += p.ref_counts[b] > 0;
    plan_sums(mine, lds, used);
    const int holes = plan_scan(p.ref_counts, 0, used, used, lds, [](int n) { return n <= 0; },
                                [&](int block, int at, int) __attribute__((always_inline)) { p.holes[at] = block; });
    plan_barrier();
    const int copies = min(holes, p.max_copies);
#pragma unroll 1
    for (int64_t b = (int64_t)used + threadIdx.x; b < p.num_blocks; b += kPlanThreads) p.to[b] = (int)b;
    plan_barrier();
    plan_scan(p.ref_counts, used, p.num_blocks, holes, lds, [](int n) { return n > 0; },
              [&](int block, int after, int held) __attribute__((always_inline)) {
                  const int at = holes - 1 - after;
                  if (at >= copies) return;
                  const int to = p.holes[at];
                  p.to[block] = to;
                  p.copies[2 * at] = block;
                  p.copies[2 * at + 1] = to;
                  p.ref_counts[to] = held;
                  p.ref_counts[block] = 0;
              });
    if (threadIdx.x == 0) {
        p.counts[0] = copies;
        p.counts[1] = used;
    }
    if (!p.tables_too) return;
    plan_barrier();
    for (int r = threadIdx.x >> 4; r < p.num_seqs; r += kPlanThreads / 16) compact_row(p, used, r, threadIdx.x & 15, 16);
}

static __global__ __launch_bounds__(kPageThreads) void compact_tables_kernel(const CompactParams p)
{
    compact_row(p, p.counts[1], blockIdx.x, blockIdx.y * kPageThreads + threadIdx.x, gridDim.y * kPageThreads);
}

}  // namespace optgqa
