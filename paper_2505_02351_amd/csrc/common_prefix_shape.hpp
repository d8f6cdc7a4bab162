// How an attention call with one common prefix is cut into pieces (common_prefix_kernels.hpp): the host's rules, for its launch and for
// its workspace.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "common.hpp"

namespace optgqa {

constexpr int kCommonThreads = 256, kCommonWaves = 4, kCommonXcds = 8;
constexpr int64_t kCommonMostWorkgroups = 0xffffffffLL / kCommonThreads;         // a dimension of a launch has fewer than 2^32 threads

// The prefix's part of a launch: an item for each (KV head, range of keys, row tile), by KV head, then range, then tile.  Workgroups go to
// XCD (number % 8), which has an L2 of its own: each XCD takes an eighth of the items, one behind another, so that the tiles of a
// range, which read the same keys, and the ranges of a KV head, which read the same queries, are together as far as
// all XCDs have as much to do.
struct PrefixItems {
    int items, per_xcd;
    FastDiv by_tiles, by_ranges;
    __host__ void set(int kv_heads, int ranges, int tiles)
    {
        items = kv_heads * ranges * tiles, per_xcd = (items + kCommonXcds - 1) / kCommonXcds;
        by_tiles.set((uint32_t)tiles), by_ranges.set((uint32_t)(ranges > 0 ? ranges : 1));
    }
    __host__ __device__ __forceinline__ int workgroups() const { return per_xcd * kCommonXcds; }
    // of a workgroup below workgroups(); false: it has none
    __host__ __device__ __forceinline__ bool place(int workgroup, int ranges, int tiles, int& g, int& range, int& tile) const
    {
        const int item = workgroup % kCommonXcds * per_xcd + workgroup / kCommonXcds, unit = by_tiles.div(item);
        g = by_ranges.div(unit);
        range = unit - g * ranges, tile = item - unit * tiles;
        return item < items;
    }
};

struct CommonPlan {
    int p_row_waves, p_tiles, p_splits, p_keys, s_row_waves, s_shares;
    int64_t rows, p_slots, p_units, s_workgroups;                // s_workgroups: own pieces at most
    int64_t held;                                                // pieces of 32 rows that the workspace has to hold
    int64_t direct_workgroups;                                   // trees: more than 0: no join; a workgroup to a token and a piece
    int64_t p_pieces(int num_kv_heads) const { return num_kv_heads * p_splits * p_slots; }
    int64_t workgroups() const { return (p_units * p_tiles + kCommonXcds - 1) / kCommonXcds * kCommonXcds + s_workgroups; }
    int64_t pieces(int num_kv_heads) const { return p_pieces(num_kv_heads) + s_workgroups * s_row_waves; }
    size_t bytes(int head_dim) const { return (size_t)held * 32 * (head_dim * sizeof(float) + 2 * sizeof(float)); }
};

// Row blocks of a workgroup for so many rows: 1, 2 or 4 of 32.
inline int common_row_waves(int64_t rows) { return rows > 64 ? 4 : rows > 32 ? 2 : 1; }

// Ranges of the prefix for trees, which bring many rows: `units` KV heads times row tiles, each of `steps` steps.  A CU's workgroups, two at a time, take
// as long as their steps one after another, so what counts are the most workgroups that a CU gets; every range costs the join
// a hundredth of a step more for each of its pieces (of 32 rows, 33 KB written and read; a step is 0.67 us), a workgroup some 4 steps to begin and
// end.  (As many ranges as the CUs hold once, the other calls' rule, leave CUs idle where units are more than a few: 16 trees of 20 - 60 behind
// 8 192 tokens, 32 / 4 heads, E4M3, 180 units: one range 218 us, four 153.  Equal shares that begin and end anywhere, two to a CU, took 150, and
// 8 % more of every other call: one workgroup's loop over units kept too much in registers.)
constexpr int kTreeRounds = 4;                                   // workgroups of a CU at most, where ranges are more than one
inline int64_t tree_ranges(int64_t units, int64_t steps, int64_t slots, int64_t cus)
{
    if (8 * units <= cus) return std::max<int64_t>(std::min(cus / units, steps / 2), 1);          // (they leave an eighth of the CUs idle at most)
    int64_t best = 1, least = INT64_MAX;
    for (int64_t n = 1; n == 1 || (units * n <= kTreeRounds * cus && 2 * n <= steps); ++n) {
        const int64_t cost = 100 * ((units * n + cus - 1) / cus) * ((steps + n - 1) / n + 4) + n * slots;
        if (cost < least) best = n, least = cost;
    }
    return best;
}

// Shares of all own parts: half a workgroup to a CU beside the prefix's; trees with no prefix have the CUs to themselves, two
// workgroups to each, and with one as much of that as their steps are of all.  (1, 2, 3, 4 and 6 to a CU, replayed graphs with the join: two trees of 64 behind 32 000, 64 / 8 heads of
// 128, bf16, 245, 199, 215, 205 and 216 us; 64 trees of 12 - 24 behind 511 - 2 047, 32 / 8, 106, 103, 108, 108 and 110; one of 16 behind 32 000 40, 41, 49, 52 and 61.  Behind a prefix of as
// much again it varies: four of 40 - 64, 8 192 common and 6 000 - 8 000 own, 128, 135, 114, 112 and 121; eight of 16, 4 096 and 3 000 - 4 000, 50, 60, 57, 59 and 62.)
inline int64_t common_most_shares(int64_t cus, bool alone) { return std::max<int64_t>(alone ? 2 * cus : cus / 2, 1); }

// Trees with no prefix whose segments have so many steps at most are one piece each, whatever the shares; the call is one launch then, that writes the
// output.  (A replayed graph's call, us, of one and of two launches: one tree of 8, 8 / 2 heads of 64, behind 120 tokens 6.8 and 10.4, 500 (4 steps) 8.4 and 10.5,
// 1 000 11.9 and 10.7; one of 16, 32 / 8 heads of 128, 250 (4 steps) 11.8 and 13.2, 500 16.7 and 13.4; eight of those 250 14.0 and 17.3, 500 17.5 and 22.1, 1 000
// 26.9 and 24.5.)
constexpr int kTreeOneSteps = 5;

// Trees with no prefix: a segment of up to a share and a half, or four steps more than one, stays one piece, whose workgroup writes the output and leaves
// nothing to join.  (64 trees of 16 behind 1 000 - 2 000, 32 / 8 heads of 128, a line at one share 100 us, at a half more 86; of 24 130 and 117.  Lines at 1, 1.25, 2, 2.5 and 3
// shares over 67 shapes of 4 to 128 trees, 4 to 64 tokens, contexts of 500 to 16 000, seven numbers of heads: 1.010, 1.015, 1.014, 1.021 and 1.044 times as long in
// the geometric mean, single shapes 0.8 to 1.6 times: 32 trees of 16 behind 1 000 - 2 000 take 74 us, 59 with the line at 2.5; 18 of 12 behind 7 258, 40 / 8 heads of 64, 66
// and 87.)
__host__ __device__ __forceinline__ bool tree_one_piece(int steps, int share)
{
    return steps <= share + (share / 2 > kTreeOneSteps - 1 ? share / 2 : kTreeOneSteps - 1);
}

// Pieces that any call has that is no larger in its tokens, sequences, prefix, longest context and new tokens of a sequence: what is
// held for a call serves all smaller ones.  (The pieces of the calls themselves go up and down: a workgroup's worth of rows more
// means fewer ranges of the prefix.)
inline int64_t common_held(int64_t rows, int64_t num_seqs, int64_t own_rows, int num_kv_heads, int64_t prefix_len, int64_t max_context_len, int64_t cus,
                           int64_t most_shares, bool tree)
{
    int64_t prefix = 0, own = 0;
    if (prefix_len > 0) {
        // Of a KV head: t tiles of w row blocks, s <= w t of them there, in max(1, min(cus / (KV heads t), keys / (256 / w))) ranges; s
        // times either is at most 4 cus / KV heads, or s keys / 64.
        const int64_t slots = (rows + 31) / 32;
        prefix = num_kv_heads * std::max(slots, std::min(4 * (cus / num_kv_heads), slots * std::max<int64_t>(prefix_len / 64, 1)));
        // (tree_ranges: a range for 64 keys begun at most, and kTreeRounds cus workgroups of up to 4 row blocks where they are more than one)
        if (tree) prefix = num_kv_heads * std::max(slots, std::min(4 * kTreeRounds * cus / num_kv_heads + 1, slots * ((prefix_len + 63) / 64)));
    }
    // (a shorter prefix leaves all of the context behind it)
    for (int w = 1; max_context_len > 0 && w <= common_row_waves(own_rows); w *= 2) {
        const int64_t tile_rows = 32 * w, r = w < 4 ? std::min(own_rows, tile_rows) : own_rows;
        const int64_t tiles = std::min(num_seqs * ((r + tile_rows - 1) / tile_rows), rows / tile_rows + num_seqs);
        const int64_t step = 32 * (kCommonWaves / w);
        const int64_t shares = std::min(most_shares, std::min(most_shares, num_kv_heads * tiles) * ((max_context_len + step - 1) / step));
        own = std::max(own, w * (shares + num_kv_heads * (rows / tile_rows + num_seqs)));
    }
    return prefix + own;
}

// false: sizes beyond the kernels' 32-bit counts or a launch's workgroups
inline bool plan_common(CommonPlan& c, int64_t num_tokens, int64_t num_seqs, int num_heads, int num_kv_heads, int64_t prefix_len, int64_t max_context_len,
                        int64_t max_q_len, int64_t cus, bool tree = false)
{
    const int64_t group = num_heads / num_kv_heads;
    c = CommonPlan{};
    c.rows = num_tokens * group;
    c.p_slots = (c.rows + 31) / 32;
    c.p_row_waves = common_row_waves(c.rows);
    c.p_tiles = 1, c.p_keys = 32;
    if (c.rows >= (1ll << 31) - 64 || c.p_slots * num_kv_heads > kCommonMostWorkgroups) return false;        // (the join's)
    // A workgroup of each kind to a CU: the prefix's is bound by its matrix and vector instructions, the own parts' by memory.
    if (prefix_len > 0) {
        c.p_tiles = (int)((c.p_slots + c.p_row_waves - 1) / c.p_row_waves);
        // ranges: none shorter than two tiles of 32 for each key group of a workgroup
        const int64_t step = 32 * (kCommonWaves / c.p_row_waves), units = (int64_t)num_kv_heads * c.p_tiles;
        const int64_t n = tree ? tree_ranges(units, (prefix_len + step - 1) / step, c.p_slots * num_kv_heads, cus)
                               : std::max<int64_t>(std::min(cus / units, prefix_len / (2 * step)), 1);
        const int64_t each = ((prefix_len + n - 1) / n + step - 1) / step * step;
        c.p_keys = (int)each;
        c.p_splits = (int)((prefix_len + each - 1) / each);
        c.p_units = (int64_t)num_kv_heads * c.p_splits;
    }
    const int64_t behind = max_context_len - prefix_len, own_rows = std::min(max_q_len, num_tokens) * group;
    c.s_row_waves = common_row_waves(own_rows);
    if (behind > 0) {
        const int64_t tile_rows = 32 * c.s_row_waves, step = 32 * (kCommonWaves / c.s_row_waves);
        // row tiles: of all sequences at the bound, or of all tokens and one begun by each sequence
        const int64_t tiles = std::min(num_seqs * ((own_rows + tile_rows - 1) / tile_rows), c.rows / tile_rows + num_seqs);
        const int64_t each = (behind + step - 1) / step;
        if (each > (1 << 20) || num_kv_heads * tiles >= (1ll << 30) || num_kv_heads * tiles * each >= (1ll << 30)) return false;
        // (a piece of half of all CUs' share: with more pieces, and with fewer, 64 sequences behind 4 096 tokens, own parts of 127 - 1 023, take
        // 37 - 38 us instead of 32, behind 32 768, 1 023 - 2 047, 110 - 125 instead of 110)
        const int64_t own = num_kv_heads * tiles * each, prefix = c.p_units * c.p_tiles * ((c.p_keys + step - 1) / step);      // steps
        int64_t most = common_most_shares(cus, false);
        if (tree) most = std::max<int64_t>(most, (int64_t)(common_most_shares(cus, true) * ((double)own / (double)(own + prefix))));
        c.s_shares = (int)std::min(most, own);
        // no more than the shares and one for each segment
        c.s_workgroups = c.s_shares + num_kv_heads * (c.rows / tile_rows + num_seqs);
    }
    if (tree && prefix_len == 0 && (max_context_len + 32 * (kCommonWaves / c.s_row_waves) - 1) / (32 * (kCommonWaves / c.s_row_waves)) <= kTreeOneSteps &&
        num_tokens + c.s_workgroups <= kCommonMostWorkgroups)
        c.direct_workgroups = num_tokens + c.s_workgroups;
    if (c.workgroups() > kCommonMostWorkgroups) return false;
    c.held = common_held(c.rows, num_seqs, own_rows, num_kv_heads, prefix_len, max_context_len, cus, common_most_shares(cus, tree), tree);
    return true;
}

}  // namespace optgqa
