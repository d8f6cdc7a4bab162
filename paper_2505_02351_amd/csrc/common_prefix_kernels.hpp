// Attention for a batch whose sequences all begin with the same cached blocks: the common prefix is computed once for all.
//
// Softmax over a row's keys can be cut anywhere: a piece leaves its reference m, its sum l = sum 2^(s - m) and its weighted
// sum o = sum 2^(s - m) V, and pieces join as
//     out = sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i,   M = max m_i          (s: scores in base 2)
// Here the cuts are
//   the prefix     the rows of ALL sequences - every new token, every head of the group - against its keys, cut into ranges of
//                  p_keys: a dense contraction whose K and V tiles serve up to 128 rows at a time;
//   own parts      the rows of ONE sequence against the keys behind the prefix.  Lengths are ragged and known on the device only: the
//                  steps (of 128, 64 or 32 keys) of all (sequence, KV head, row tile) segments, divided by a number of shares, are
//                  the longest that a piece may be, and each segment is cut into so many equal pieces.
// One launch computes all pieces (a workgroup each), a second joins them.  A row sees keys 0 .. its position, wherever the
// prefix ends.
//
// A workgroup is four waves of 32 rows: RW row blocks by KS key groups, RW * KS = 4.  The waves of a key group share its
// tiles of 32 keys in LDS; the KS groups take tiles in turn, and their results are joined through LDS.  With many rows 4 x 1 reads
// each tile once for 128 rows, with few (a sequence's own part: the heads of a group, times its new tokens) 1 x 4 lets each wave
// stream tiles of its own.  Scores, softmax and output as in prefill_kernels.hpp: both contractions transposed on
// v_mfma_f32_32x32x16, sums and output in fp32, weights rounded to fp16 once (CommonSoftmax) or split into two bf16.
//
// Own parts are bound by memory, the prefix by its matrix instructions, their LDS reads and the softmax between them, which one wave to a SIMD does
// one after another, short launches by their chains of loads.  Measured (both launches, inputs in turn): 64 sequences, 32 / 8 heads of 128, bf16, behind
// 32 768 tokens, 1 023 - 2 047 own: 108 - 110 us, 5.0 TB/s; 32 / 4 heads behind 4 096, 127 - 1 023 own, slopes: 30 - 31; 16 of 2 - 9 drafts, 64 / 8 heads,
// fp16, behind 8 192: 44.6 us, 480 TFLOP/s; 32 behind 8 192, E4M3 caches: 27.6 - 28.3.
// (head_dim 128 with bf16 takes all 256 registers that two workgroups to a CU leave a wave, and one more, which lies in scratch.)
#pragma once
#include <type_traits>

#include "common_prefix_shape.hpp"
#include "mfma_tiles.hpp"

namespace optgqa {

// A tile of 32 keys in LDS, as the memory system writes it (see PfDirect): 2-byte rows, or 8-bit codes as they are.  Rows of as many
// bytes lie alike; the 64 bytes of a row of 64 codes, 16 rows to a group, with their columns of 16 bytes exchanged by
// row, so that a column of 16 rows again lies in 16 different sixteenths of the banks.
template <int D, bool KV8> struct CommonTile {
    static constexpr bool kShort = KV8 && D == 64;
    static constexpr int kRowBytes = KV8 ? D : 2 * D;
    typedef PfDirect<kShort ? 64 : kRowBytes / 2> Like;
    static constexpr int kRows = 1024 / kRowBytes, kGroups = kPfKeys / kRows;
    static constexpr int kGroup = kShort ? 1024 + 64 : Like::kGroup, kTile = kGroups * kGroup;
    static constexpr int kBuffers = KV8 ? 8 : 4;                 // of a K and a V tile, of a workgroup, over its key groups
    static __device__ __forceinline__ int load_row(int l) { return kShort ? l >> 2 : Like::load_row(l); }
    static __device__ __forceinline__ int load_col(int l) { return kShort ? (l & 3) ^ ((l >> 4) & 3) : Like::load_col(l); }
    // byte offset of a row's 16-byte column 0 or 1, and of the one 2m further on
    static __device__ __forceinline__ int at(int row, int col)
    {
        return kShort ? (row >> 4) * kGroup + (row & 15) * 64 + ((col ^ ((row >> 2) & 3)) << 4) : Like::row_at(row, col);
    }
    static __device__ __forceinline__ int further(int at, int m) { return kShort ? at ^ (32 * m) : at + Like::dims_at(m); }
};

struct CommonParams {
    void* out;                  // [T][Hq][D]
    const void* q;
    const void* k_cache;        // [NB][Hkv][bs][D]
    const void* v_cache;
    const int32_t* prefix_table;
    const int32_t* block_tables;
    const int32_t* context_lens;
    const int32_t* cu_q_lens;   // [B + 1], or nullptr: a new token each
    const float* slopes;        // [Hq] or nullptr
    float scale2, out_scale;    // log2(e) * scale (times k_scale); v_scale
    const float *k_scales, *v_scales;           // E4M3 caches, one pair per KV head, or nullptr
    int num_tokens, num_seqs, num_heads, num_kv_heads, group, block_shift, max_blocks_per_seq;
    int prefix_len;             // keys
    int rows;                   // num_tokens * group: of a KV head
    int p_row_waves, p_tiles, p_splits, p_keys;                              // tiles: workgroups' row tiles; splits: ranges of p_keys keys
    int s_row_waves, s_shares;
    // pieces, 32 rows each: of the prefix [range][KV head][p_slots]; then s_row_waves for each own one
    int p_slots;
    int64_t s_first;
    float4* o;                  // per piece [D / 8][64]: what lane l of the wave holds, dims 8i + 4 (l / 32) .. + 3 of row l % 32
    float2* ml;                 // per piece [32]: m, l
    PrefixItems p_items;
    FastDiv by_group, by_kv_heads, by_s_shares;
};

template <int D, bool KV8> constexpr int kCommonLds = [] {
    const int tiles = CommonTile<D, KV8>::kBuffers * 2 * CommonTile<D, KV8>::kTile, join = kCommonWaves * 64 * (D / 8 * 16 + 8);
    return tiles > join ? tiles : join;
}();

// The sequence of token t (seq < 0: none has it), its context length, its first token and the one behind its last.  All lanes of a wave
// together: first the guess that every sequence has one new token, which one round trip to memory confirms, else the sequences'
// ends and lengths, 64 at a time, one a lane.
struct TokenPlace {
    int seq, len, first, end;
    __device__ __forceinline__ int pos(int t) const { return seq < 0 ? -1 : len - end + t; }
};
// What the guess needs, asked for here and used by find() (so that other loads can be asked for in between).
struct PlaceGuess {
    int seq, first, end, len;   // seq: the t-th, or the last
    __device__ __forceinline__ PlaceGuess(const CommonParams& p, int t)
    {
        seq = min(t, p.num_seqs - 1);
        first = seq, end = seq + 1;
        if (p.cu_q_lens) first = p.cu_q_lens[seq], end = p.cu_q_lens[seq + 1];
        len = p.context_lens[seq];
    }
    __device__ __forceinline__ TokenPlace find(const CommonParams& p, int t) const
    {
        if (__builtin_amdgcn_ballot_w64(first != t || end != t + 1) == 0) return {seq, len, first, end};
        const int lane = threadIdx.x & 63;
        TokenPlace at{-1, 0, 0, 0};
        for (int from = 0; from < p.num_seqs; from += 64) {
            const int n = min(p.num_seqs - from, 64), b = from + min(lane, n - 1);
            const int starts = p.cu_q_lens[b], ends = p.cu_q_lens[b + 1], lens = p.context_lens[b];
            int k = 0;                                           // of the n sequences, those that end at or before t
#pragma unroll
            for (int s = 32; s; s >>= 1) {
                const int e = __shfl(ends, (k + s - 1) & 63);    // (all lanes exchange, also those that do not want it)
                if (k + s <= n && e <= t) k += s;
            }
            const int next = __shfl(ends, k & 63);
            if (k + 1 <= n && next <= t) ++k;
            const int first_k = __shfl(starts, k & 63), len_k = __shfl(lens, k & 63);
            if (at.seq < 0 && k < n) at = {from + k, len_k, first_k, next};
        }
        return at;
    }
};

// Own parts of 64 sequences, one a lane.  A segment: one KV head, one row tile.
struct OwnParts {
    int len, first, rows;       // context length, first token, rows (new tokens x heads of the group)
    int steps, segments;        // of a segment; segments (0: nothing to do)
    int pieces, before;         // of a segment; pieces of all sequences before this one (number())
    static __device__ __forceinline__ int keys_shift(const CommonParams& p) { return 7 - (p.s_row_waves >> 1); }       // a step's: 128, 64, 32 for 1, 2, 4
    static __device__ __forceinline__ int steps_of(const CommonParams& p, int keys) { return (keys + (1 << keys_shift(p)) - 1) >> keys_shift(p); }
    // those from number `from` on
    __device__ __forceinline__ OwnParts(const CommonParams& p, int from)
    {
        const int lane = threadIdx.x & 63, b = min(from + lane, p.num_seqs - 1);
        len = p.context_lens[b];
        first = p.cu_q_lens ? p.cu_q_lens[b] : b;
        rows = (p.cu_q_lens ? p.cu_q_lens[b + 1] - first : 1) * p.group;
        const int behind = from + lane < p.num_seqs && rows > 0 ? max(len - p.prefix_len, 0) : 0;
        steps = steps_of(p, behind);
        segments = behind > 0 ? ((rows + 32 * p.s_row_waves - 1) >> (4 + 32 - __builtin_clz(p.s_row_waves))) * p.num_kv_heads : 0;
    }
    // a segment has as many equal pieces as shares of `most` steps take; `all`: pieces before these sequences, and then with them
    __device__ __forceinline__ void number(int most, int& all)
    {
        pieces = div_by_inverse(steps + most - 1, most, __builtin_amdgcn_rcpf((float)most));
        const int mine = pieces * segments, sum = lane_sums(mine);
        before = all + sum - mine;
        all += __builtin_amdgcn_readlane(sum, 63);
    }
    // steps of a piece
    static __device__ __forceinline__ int each(int steps, int pieces) { return div_by_inverse(steps + pieces - 1, pieces, __builtin_amdgcn_rcpf((float)pieces)); }
};
// The most steps of a piece.  `parts`: the first 64 sequences'.
__device__ __forceinline__ int own_share(const CommonParams& p, const OwnParts& parts)
{
    int total = wave_sum(parts.steps * parts.segments);
    for (int from = 64; from < p.num_seqs; from += 64) {
        const OwnParts more(p, from);
        total += wave_sum(more.steps * more.segments);
    }
    return max(p.by_s_shares.div(total + p.s_shares - 1), 1);
}

// How far a tile's maximum may lie above a row's reference, and where the reference is put when one does (log2 units above that
// maximum).  bf16: as everywhere.  fp16 weights are rounded once, and a range may be a whole long prefix whose many small
// weights add up beside one large one: the reference lies below the maximum, so that weights down to 24 binary orders under the largest are
// normal numbers and those down to 35 are there (2 above it, as in the prefill kernel: 12 and 23; 32 767 keys 21.25 orders under one
// key came to 1.54e-2 in place of 1.30e-2).  The room up to 2^15 is what keeps rescales few: maxima that grow by less than 5 orders need none.  (16 of
// 2 - 9 drafts, 64 / 8 heads, behind 8 192: scores of variance 1 44.3 -> 44.5 us, 16 45 -> 53, 100 53 -> 55; a threshold of 2^15.9 53, a reference 8 below 52.)
template <int DT> struct CommonSoftmax { static constexpr float kThreshold = PfSoftmax<DT>::kThreshold, kHeadroom = PfSoftmax<DT>::kHeadroom; };
template <> struct CommonSoftmax<kF16> { static constexpr float kThreshold = 15.f, kHeadroom = -10.f; };

// A workgroup's rows and keys.
struct CommonJob {
    bool prefix;
    int g;
    const int32_t* table;
    int kbeg, kend;             // keys; kend > kbeg
    int row0, num_rows;         // its first row, of the batch's (prefix) or of the sequence's
    int tok0, pos0;             // token and position of row 0 (pos0: own parts)
    int64_t slot;               // piece of its first 32 rows
    int held_first, held;       // the lane's entry of `table`: held_first + lane
};

// of 16 bytes of values, or of codes (whose only such value is NaN)
template <int DT, bool KV8> __device__ __forceinline__ bool any_not_finite(uint4 x)
{
    constexpr uint32_t kExp = DT == kF16 ? 0x7c00u : 0x7f80u;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w;
        if (KV8) odd = odd || (w & 0x7fu) == 0x7fu || (w & 0x7f00u) == 0x7f00u || (w & 0x7f0000u) == 0x7f0000u || (w & 0x7f000000u) == 0x7f000000u;
        else odd = odd || (w & kExp) == kExp || ((w >> 16) & kExp) == kExp;
    }
    return odd;
}

// a pair of 2-byte values with those that are no finite numbers put to 0
template <int DT> __device__ __forceinline__ uint32_t finite_pair(uint32_t w)
{
    constexpr uint32_t kExp = DT == kF16 ? 0x7c00u : 0x7f80u;
    if ((w & kExp) == kExp) w &= 0xffff0000u;
    if (((w >> 16) & kExp) == kExp) w &= 0x0000ffffu;
    return w;
}

template <int DT, bool KV8, int D, int RW>
__device__ __forceinline__ void common_body(const CommonParams& p, const CommonJob& job)
{
    constexpr int KS = kCommonWaves / RW;
    constexpr int kQ = D / 16, kDB = D / 32, kPieces = D / 8;
    constexpr int ES = KV8 ? 1 : 2;
    typedef CommonTile<D, KV8> Tile;
    constexpr int NBUF = Tile::kBuffers / KS > 4 ? 4 : Tile::kBuffers / KS;
    constexpr bool kHalfLoad = Tile::kGroups < RW;               // fewer 1 KiB groups than waves: half of them bring K, half V
    constexpr int kWaveGroups = kHalfLoad ? 1 : Tile::kGroups / RW;              // groups of a K (or V) tile that a wave brings
    constexpr int kWaveKeys = kWaveGroups * Tile::kRows;
    constexpr int kHalves = kWaveKeys > 16 ? 2 : 1;              // runs of up to 16 keys, each in one block, they lie in
    constexpr int kRunGroups = kWaveGroups / kHalves;
    extern __shared__ __attribute__((aligned(16))) unsigned char common_lds[];
    unsigned char* const lds = common_lds;
    const int lane = threadIdx.x & 63, n32 = lane & 31, h2 = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), rw = wave % RW, kw = wave / RW;
    const int kbeg = job.kbeg, kend = job.kend;
    const int ntiles = (kend - kbeg + kPfKeys - 1) / kPfKeys, steps = (ntiles + KS - 1) / KS;
    // ---- the lane's row, its query and what its position is made of: asked for in front of everything that is waited for -----
    const int r = job.row0 + 32 * rw + n32;
    const bool row_ok = r < job.num_rows;
    const int rc = min(r, job.num_rows - 1), ti = p.by_group.div(rc), head = job.g * p.group + (rc - ti * p.group);
    const int t = job.tok0 + ti;
    uint4 qb[kQ];
    {
        // (the lane's dims of score MFMA m: 16m + 8 h2 .. + 7; of codes, 16 of which are one read: 32 (m / 2) + 16 h2 + 8 (m % 2) ..)
        const unsigned char* const qp = static_cast<const unsigned char*>(p.q) + ((int64_t)t * p.num_heads + head) * (D * 2) + (KV8 ? 32 : 16) * h2;
#pragma unroll
        for (int m = 0; m < kQ; ++m) qb[m] = *reinterpret_cast<const uint4*>(qp + (KV8 ? 64 * (m >> 1) + 16 * (m & 1) : 32 * m));
    }
    float slope = p.slopes ? p.slopes[head] : 0.f;
    int pos = job.pos0 + ti;
    if (job.prefix) pos = PlaceGuess(p, t).find(p, t).pos(t);
    auto has = [&](int j) __attribute__((always_inline)) { return j * KS + kw < ntiles; };

    // ---- where tiles come from: a lane holds one of 64 block numbers -------------------------------------
    const int bshift = p.block_shift, bmask = (1 << bshift) - 1;
    const uint32_t blk_bytes = (uint32_t)p.num_kv_heads << bshift << (D == 128 ? 7 : 6) << (ES - 1);
    const uint32_t head_bytes = (uint32_t)job.g << bshift << (D == 128 ? 7 : 6) << (ES - 1);
    const unsigned char* const kc = static_cast<const unsigned char*>(p.k_cache) + head_bytes;
    const unsigned char* const vc = static_cast<const unsigned char*>(p.v_cache) + head_bytes;
    const int last_block = (kend - 1) >> bshift;
    int held_first = job.held_first, held = job.held;
    const int load_row = Tile::load_row(lane), load_col = Tile::load_col(lane);
    const uint32_t lane_off = (uint32_t)(load_row * Tile::kRowBytes + 16 * load_col);
    // byte offset, in either cache from its KV head's first block on, of key `key` (wave-uniform)
    auto key_at = [&](int key) __attribute__((always_inline)) -> uint64_t {
        const int block = key >> bshift;
        if (__builtin_expect(block - held_first >= 64, 0)) {
            held_first = block - 8;                              // (V tiles follow K tiles by a step: up to 64 keys)
            held = job.table[min(held_first + lane, last_block)];
            asm volatile("" : "+v"(held));                       // (waited for here, not on the way that reads no table)
        }
        return (uint64_t)(uint32_t)__builtin_amdgcn_readlane(held, block - held_first) * blk_bytes + (uint32_t)((key & bmask) * Tile::kRowBytes);
    };
    // offsets, and this lane's, of the wave's runs of the group's tile j; `first`: its first 1 KiB group of the tile
    const int first_k = kHalfLoad ? rw : rw * kWaveGroups, first_v = kHalfLoad ? rw - (RW - Tile::kGroups) : first_k;
    struct Runs { uint64_t at[kHalves]; uint32_t lane_at[kWaveGroups]; };
    auto runs_of = [&](int j, int first_group) __attribute__((always_inline)) {
        Runs r;
        const int key0 = kbeg + kPfKeys * (j * KS + kw) + first_group * Tile::kRows;
        const bool tail = key0 + kWaveKeys > kend;               // keys from kend on: kend - 1 again
#pragma unroll
        for (int h = 0; h < kHalves; ++h) r.at[h] = key_at(min(key0 + 16 * h, kend - 1));
#pragma unroll
        for (int n = 0; n < kWaveGroups; ++n) {
            r.lane_at[n] = (uint32_t)((n % kRunGroups) * 1024) + lane_off;
            if (tail) {
                const int first = min(key0 + 16 * (n / kRunGroups), kend - 1);
                const int key = min(key0 + n * Tile::kRows + load_row, kend - 1);
                r.lane_at[n] = (uint32_t)((key - first) * Tile::kRowBytes + 16 * load_col);
            }
        }
        return r;
    };
    auto buffer = [&](int j) __attribute__((always_inline)) { return (kw * NBUF + (j & (NBUF - 1))) * 2 * Tile::kTile; };     // K tile, then V tile
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;
    // (of the wave's groups; nothing for a wave that does not bring this tensor)
    auto ask = [&](const Runs& r, const unsigned char* cache, int at, int first_group) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < kWaveGroups; ++n) {
            const uint32_t to = lds0 + at + (first_group + n) * Tile::kGroup;
            if (RW == 1) stream_direct(to, cache + r.at[n / kRunGroups], r.lane_at[n]);      // (no other row tile reads them)
            else load_direct(to, cache + r.at[n / kRunGroups], r.lane_at[n]);
        }
    };

    // ---- the first tiles -------------------------------------------------------------------------------------
    // RW > 1: a key group's K and V tiles in rings of NBUF buffers.  The scores of a step's tile are made a step ahead, under the
    // softmax of the tile before, so K tiles run one ahead of V tiles: step j asks for K tile j + 1 + kLead and V tile j + kLead.
    // RW == 1: a wave's own tiles, NBUF buffers: K tile j + NBUF is asked for when the scores of tile j are there, its V
    // tile when the output of tile j is.
    constexpr int kLead = NBUF / 2;
    constexpr int kLoads = kHalfLoad ? 1 : 2 * kWaveGroups;      // of a wave, per K and V tile
    auto buffer_v = [&](int j) __attribute__((always_inline)) { return buffer(j) + Tile::kTile; };
    auto ask_k = [&](int j) __attribute__((always_inline)) {
        if (has(j) && (!kHalfLoad || first_k < Tile::kGroups)) ask(runs_of(j, first_k), kc, buffer(j), first_k);
    };
    auto ask_v = [&](int j) __attribute__((always_inline)) {
        if (has(j) && first_v >= 0) ask(runs_of(j, first_v), vc, buffer_v(j), first_v);
    };
    asm volatile("" : "+v"(held) :: "memory");
    if constexpr (RW > 1) {
        ask_k(0);
        ask_k(1);
        ask_v(0);
        if constexpr (kLead == 2) ask_k(2), ask_v(1);
    } else {
#pragma unroll
        for (int j = 0; j < NBUF; ++j) ask_k(j), ask_v(j);
    }
    const int lim = row_ok ? min(pos + 1, kend) : kend;          // keys below it are visible
    const int least = -wave_max(-lim);                           // tiles that end at or below it need no mask
    const uint32_t keep_q = row_ok ? 0xffffffffu : 0u;
#pragma unroll
    for (int m = 0; m < kQ; ++m) qb[m] = make_uint4(qb[m].x & keep_q, qb[m].y & keep_q, qb[m].z & keep_q, qb[m].w & keep_q);
    const float scale2 = KV8 && p.k_scales ? p.scale2 * p.k_scales[job.g] : p.scale2;
    const float slope2 = row_ok ? slope * kLog2e : 0.f;
    f32x16 key_bias;                                             // slope * (key's offset in its tile) / score scale: the scores start from it
    {
        const float per_key = slope2 / scale2;
#pragma unroll
        for (int e = 0; e < 16; ++e) key_bias[e] = per_key * (float)(8 * (e >> 2) + (e & 3));
    }
    f32x16 acc[kDB];
#pragma unroll
    for (int db = 0; db < kDB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[db][e] = 0.f;
    float m_ref = 0.f, lsum = 0.f;
    bool started = !row_ok;

    const int k_at = Tile::at(n32, h2);
    // `between`: what is issued behind the reads of the first operands (a step's loads to LDS)
    auto scores = [&](int at, auto between) __attribute__((always_inline)) {
        constexpr int kReads = KV8 ? kQ / 2 : kQ, kEarly = kReads < 4 ? kReads : 4;
        f32x16 st = key_bias;
        auto read = [&](int m) __attribute__((always_inline)) { return *reinterpret_cast<const uint4*>(lds + at + Tile::further(k_at, m)); };
        uint4 ka[kEarly];
#pragma unroll
        for (int m = 0; m < kEarly; ++m) ka[m] = read(m);
        between();
#pragma unroll
        for (int m = 0; m < kReads; ++m) {
            const uint4 x = m < kEarly ? ka[m < kEarly ? m : 0] : read(m);
            if constexpr (KV8) {
                st = mfma32<DT>(widen8_e4m3<DT>(x.x, x.y), qb[2 * m], st);
                st = mfma32<DT>(widen8_e4m3<DT>(x.z, x.w), qb[2 * m + 1], st);
            } else {
                st = mfma32<DT>(x, qb[m], st);
            }
        }
        return st;
    };
    uint32_t pk[2][4], pk_lo[2][4];                              // weights as pairs of 2-byte values (and what is left of them)
    // key0: the tile's first key
    auto softmax = [&](int key0, f32x16 st, auto masked) __attribute__((always_inline)) {
        constexpr bool MASKED = decltype(masked)::value;
        const float b0 = fmaf(slope2, (float)(key0 + 4 * h2 - pos), -m_ref);         // (whole numbers' difference: exact near the row, however far)
        float x[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            x[e] = fmaf(st[e], scale2, b0);
            if (MASKED) x[e] = key0 + 4 * h2 + 8 * (e >> 2) + (e & 3) < lim ? x[e] : -INFINITY;
        }
        float mx = x[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mx = fmaxf(mx, x[e]);
        const bool first = !started;
        if (__builtin_amdgcn_ballot_w64(first || mx > CommonSoftmax<DT>::kThreshold) != 0) {
            mx = fmaxf(mx, __shfl_xor(mx, 32));                  // the row's keys live in 2 lanes (h2)
            const bool sees = mx > -INFINITY;
            float to = mx + CommonSoftmax<DT>::kHeadroom;
            // (beyond 2^27 this rounds by more than there is room for above the threshold)
            if (CommonSoftmax<DT>::kHeadroom < 0.f && mx - to > CommonSoftmax<DT>::kThreshold) to = mx;
            // (0 for a row that did not ask: no row's bits depend on what its neighbours hold)
            const float delta = (first ? sees : mx > CommonSoftmax<DT>::kThreshold) ? to : 0.f;
            const float alpha = first ? 1.f : fast_exp2(-delta);
            started = started || sees;
            m_ref += delta;
            lsum *= alpha;
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] -= delta;
#pragma unroll
            for (int db = 0; db < kDB; ++db)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[db][e] *= alpha;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float w0 = fast_exp2(x[2 * e]), w1 = fast_exp2(x[2 * e + 1]);
            if (PfSoftmax<DT>::kSplitWeights) {
                split_bf16(w0, w1, pk[e >> 2][e & 3], pk_lo[e >> 2][e & 3]);
                lsum += w0 + w1;
            } else {
                // one rounding: the sum is that of the weights as rounded, the output an exact convex combination
                const uint32_t two = narrow2<DT>(w0, w1);
                pk[e >> 2][e & 3] = two;
                lsum = dot2<DT>(two, 0x3c003c00u, lsum);         // (times 1, 1: one instruction for a pair)
            }
        }
    };
    // V^T: keys 16m + 4 h2 .. + 3 and 16m + 8 + 4 h2 .. + 3 of dim 32 db + n32, by transposing loads, in which lane s of 16 addresses
    //   2-byte  key s / 4 of four, dims 4 (s % 4) .. + 3, and gets its dim's four keys (two loads);
    //   codes   key s / 2 of eight (as they lie: four, four behind the next), dims 8 (s % 2) .. + 7, and gets its dim's eight keys.
    const int s16 = lane & 15, dhalf = (lane >> 4) & 1;
    int v_at;
    if constexpr (KV8) v_at = Tile::at(4 * h2 + ((s16 >> 1) & 3) + 8 * (s16 >> 3), dhalf) + 8 * (s16 & 1);
    else v_at = Tile::Like::keys_at(s16, dhalf, h2);
    auto v_operand = [&](int at, int m, int db) __attribute__((always_inline)) {
        if constexpr (KV8) {
            typedef int i32x2 __attribute__((ext_vector_type(2)));
            typedef __attribute__((address_space(3))) i32x2* lds_i32x2_ptr;
            const i32x2 x = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2_ptr)(lds + at + Tile::further(v_at + m * (16 / Tile::kRows) * Tile::kGroup, db)));
            return widen8_e4m3<DT>((uint32_t)x[0], (uint32_t)x[1]);
        } else {
            typedef short i16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) i16x4* lds_i16x4_ptr;
            const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_ptr)(lds + at + v_at + Tile::Like::further(2 * m, db)));
            const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_ptr)(lds + at + v_at + Tile::Like::further(2 * m + 1, db)));
            const uint2 lo2 = __builtin_bit_cast(uint2, lo), hi2 = __builtin_bit_cast(uint2, hi);
            return make_uint4(lo2.x, lo2.y, hi2.x, hi2.y);
        }
    };
    auto weighted = [&](uint4 va, int m, f32x16 c) __attribute__((always_inline)) {
        c = mfma32<DT>(va, make_uint4(pk[m][0], pk[m][1], pk[m][2], pk[m][3]), c);
        if (PfSoftmax<DT>::kSplitWeights) c = mfma32<DT>(va, make_uint4(pk_lo[m][0], pk_lo[m][1], pk_lo[m][2], pk_lo[m][3]), c);
        return c;
    };
    auto output = [&](int at) __attribute__((always_inline)) {
#pragma unroll
        for (int db = 0; db < kDB; ++db)
#pragma unroll
            for (int m = 0; m < 2; ++m) acc[db] = weighted(v_operand(at, m, db), m, acc[db]);
    };
    // A tile that some row's end cuts.  A weight of 0 does not hide a V that is no finite number from the matrix instruction.  Where
    // such a V lies beyond some row's end, the matrix instructions see 0 in its place, and the rows that do see its
    // key get it by itself (a positive weight times it is it again).
    auto output_cut = [&](int key0, int at) __attribute__((always_inline)) {
        bool odd = false;
#pragma unroll
        for (int n = 0; n < Tile::kGroups; ++n)
            odd = odd || (key0 + n * Tile::kRows + load_row >= least && any_not_finite<DT, KV8>(*reinterpret_cast<const uint4*>(lds + at + n * Tile::kGroup + 16 * lane)));
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(odd) == 0, 1)) {
            output(at);
            return;
        }
#pragma unroll
        for (int db = 0; db < kDB; ++db)
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const uint4 va = v_operand(at, m, db);
                acc[db] = weighted(make_uint4(finite_pair<DT>(va.x), finite_pair<DT>(va.y), finite_pair<DT>(va.z), finite_pair<DT>(va.w)), m, acc[db]);
            }
#pragma unroll 1
        for (int k = 0; k < kPfKeys; ++k) {
            const bool sees = key0 + k < lim;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {                  // dims 8i + 4 h2 .. + 3
                uint2 v;
                if constexpr (KV8) {
                    const uint32_t c = *reinterpret_cast<const uint32_t*>(lds + at + Tile::further(Tile::at(k, (i >> 1) & 1), i >> 2) + 8 * (i & 1) + 4 * h2);
                    v = make_uint2(widen2_e4m3<DT>(c, false), widen2_e4m3<DT>(c, true));
                } else {
                    v = *reinterpret_cast<const uint2*>(lds + at + Tile::further(Tile::at(k, i & 1), i >> 1) + 8 * h2);
                }
                const uint32_t bad[2] = {v.x ^ finite_pair<DT>(v.x), v.y ^ finite_pair<DT>(v.y)};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float x = j & 1 ? widen_hi<DT>(bad[j >> 1]) : widen_lo<DT>(bad[j >> 1]);
                    acc[i >> 2][4 * (i & 3) + j] += sees ? x : 0.f;
                }
            }
        }
    };
    auto first_key = [&](int j) __attribute__((always_inline)) { return kbeg + kPfKeys * (j * KS + kw); };
    auto finish = [&](int j, const f32x16& st, int at_v, auto masked) __attribute__((always_inline)) {
        softmax(first_key(j), st, masked);
        if (decltype(masked)::value) output_cut(first_key(j), at_v);
        else output(at_v);
    };
    auto reads_done = [] __attribute__((always_inline)) () { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };

    // ---- the walk -----------------------------------------------------------------------------------------
    // Steps [0, whole) of this wave's need no mask: loops of their own, whose bodies are straight lines.  (Waves of a workgroup may be in
    // different loops: both have the same barriers.)
    const int mine = (ntiles - kw + KS - 1) / KS;                // tiles of this wave's key group
    const int whole = min(mine, max(0, (least - kbeg) / kPfKeys - kw + KS - 1) / KS);
    if constexpr (RW > 1) {
        auto step = [&](int j, const f32x16& st_cur, f32x16& st_ahead, auto masked) __attribute__((always_inline)) {
            // K tile j + 1 and V tile j are there; newer: step j - 1's, where it asked for all of its own
            if (kLead > 1 && j + kLead < mine) wait_direct<(kLead - 1) * kLoads>();
            else wait_direct();
            __syncthreads();                                     // ... for all; and the buffers read in step j - 1 are free
            st_ahead = scores(buffer(j + 1), [&]() __attribute__((always_inline)) {
                if (j + kLead < mine) {
                    ask_k(j + 1 + kLead);
                    ask_v(j + kLead);
                }
            });
            if (!decltype(masked)::value || j < mine) finish(j, st_cur, buffer_v(j), masked);
        };
        f32x16 st, st_other;
        if (mine > kLead) wait_direct<kLead * kLoads>();         // K tile 0 (newer: kLead K tiles, kLead V tiles)
        else wait_direct();
        __syncthreads();
        st = scores(buffer(0), [] {});
        int j = 0;
        for (; j + 1 < whole; j += 2) {
            step(j, st, st_other, std::false_type{});
            step(j + 1, st_other, st, std::false_type{});
        }
        if (j < whole) {
            step(j, st, st_other, std::false_type{});
            st = st_other;
            ++j;
        }
        for (; j < steps; ++j) {
            step(j, st, st_other, std::true_type{});
            st = st_other;
        }
    } else {
        auto step = [&](int j, auto masked) __attribute__((always_inline)) {
            // K tile j is there; newer: its V tile and what was asked for since
            if (NBUF > 1 && j + NBUF - 1 < mine) wait_direct<(2 * NBUF - 1) * kWaveGroups>();
            else wait_direct<kWaveGroups>();
            const f32x16 st = scores(buffer(j), [] {});
            reads_done();
            const bool more = j + NBUF < mine;
            Runs runs;
            if (more) {
                runs = runs_of(j + NBUF, 0);
                ask(runs, kc, buffer(j), 0);
            }
            softmax(first_key(j), st, masked);
            if (more) wait_direct<(2 * NBUF - 1) * kWaveGroups>();
            else if (NBUF > 1 && j + 1 < mine) wait_direct<2 * kWaveGroups>();
            else wait_direct();
            if (decltype(masked)::value) output_cut(first_key(j), buffer_v(j));
            else output(buffer_v(j));
            reads_done();
            if (more) ask(runs, vc, buffer_v(j), 0);
        };
        static_assert(NBUF <= 2, "what is newer than a V tile");
        int j = 0;
        for (; j < whole; ++j) step(j, std::false_type{});
        for (; j < mine; ++j) step(j, std::true_type{});
    }

    // ---- what it leaves: the key groups' results joined, one piece for each row block ---------------------------
    const float l_row = lsum + __shfl_xor(lsum, 32);
    // (a row whose scores here are all NaN, a NaN query's, has no maximum; its sum says so, and has to reach the join)
    const float m_row = row_ok && (started || l_row != l_row) ? m_ref : -INFINITY;
    float4* const o = p.o + (job.slot + rw) * (kPieces * 64) + lane;
    float2* const ml = p.ml + (job.slot + rw) * 32 + n32;
    auto piece_of = [&](int i) __attribute__((always_inline)) {
        const f32x16& a = acc[i >> 2];
        const int e = 4 * (i & 3);
        return make_float4(a[e], a[e + 1], a[e + 2], a[e + 3]);
    };
    if constexpr (KS == 1) {
        if (row_ok) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) o[64 * i] = piece_of(i);
            if (h2 == 0) *ml = make_float2(m_row, l_row);
        }
    } else {
        float4* const xo = reinterpret_cast<float4*>(lds);       // [wave][piece][lane]
        float2* const xml = reinterpret_cast<float2*>(lds + kCommonWaves * 64 * kPieces * 16);
        __syncthreads();                                         // the tiles are done with
#pragma unroll
        for (int i = 0; i < kPieces; ++i) xo[(wave * kPieces + i) * 64 + lane] = piece_of(i);
        xml[wave * 64 + lane] = make_float2(m_row, l_row);
        __syncthreads();
        float m_all = -INFINITY, f[KS], l_all = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) m_all = fmaxf(m_all, xml[(k * RW + rw) * 64 + lane].x);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const float2 t2 = xml[(k * RW + rw) * 64 + lane];
            f[k] = t2.x == -INFINITY ? 0.f : fast_exp2(t2.x - m_all);
            l_all = fmaf(f[k], t2.y, l_all);
        }
#pragma unroll
        for (int i = 0; i < kPieces / KS; ++i) {
            const int piece = kw * (kPieces / KS) + i;
            float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const float4 x = xo[((k * RW + rw) * kPieces + piece) * 64 + lane];
                s.x = fmaf(f[k], x.x, s.x), s.y = fmaf(f[k], x.y, s.y), s.z = fmaf(f[k], x.z, s.z), s.w = fmaf(f[k], x.w, s.w);
            }
            if (row_ok) o[64 * piece] = s;
        }
        if (kw == 0 && h2 == 0 && row_ok) *ml = make_float2(m_all, l_all);
    }
}

template <int DT, bool KV8, int D>
__global__ __launch_bounds__(kCommonThreads, 2) void common_prefix_kernel(const CommonParams p)
{
    const int lane = threadIdx.x & 63;
    CommonJob job;
    const int p_workgroups = p.p_items.workgroups();
    job.prefix = (int)blockIdx.x < p_workgroups;
    const int row_waves = job.prefix ? p.p_row_waves : p.s_row_waves;
    if (job.prefix) {
        int range, tile;
        if (!p.p_items.place(blockIdx.x, p.p_splits, p.p_tiles, job.g, range, tile)) return;
        job.table = p.prefix_table;
        job.kbeg = range * p.p_keys;
        job.kend = min(job.kbeg + p.p_keys, p.prefix_len);
        job.row0 = tile * 32 * row_waves;
        job.num_rows = p.rows;
        job.tok0 = job.pos0 = 0;
        job.slot = ((int64_t)range * p.num_kv_heads + job.g) * p.p_slots + tile * row_waves;
    } else {
        const int me = blockIdx.x - p_workgroups;              // the piece
        OwnParts parts(p, 0);
        const int share = own_share(p, parts);
        int all = 0, from = 0;
        parts.number(share, all);
        while (all <= me) {                                      // not one of these sequences'
            from += 64;
            if (from >= p.num_seqs) return;                      // (nobody's)
            parts = OwnParts(p, from);
            parts.number(share, all);
        }
        const int l = 63 - __builtin_clzll(__builtin_amdgcn_ballot_w64(parts.segments > 0 && parts.before <= me));
        const int b = from + l, len = __builtin_amdgcn_readlane(parts.len, l), steps = __builtin_amdgcn_readlane(parts.steps, l);
        const int pieces = __builtin_amdgcn_readlane(parts.pieces, l), in_seq = me - __builtin_amdgcn_readlane(parts.before, l);
        const int segment = __builtin_amdgcn_readfirstlane(in_seq / pieces), each = __builtin_amdgcn_readfirstlane(OwnParts::each(steps, pieces));
        const int lo = (in_seq - segment * pieces) * each, hi = min(lo + each, steps);
        if (hi <= lo) return;                                    // (equal pieces of, say, 7 steps in 4: the last is empty)
        job.num_rows = __builtin_amdgcn_readlane(parts.rows, l);
        job.tok0 = __builtin_amdgcn_readlane(parts.first, l);
        const int tiles = (job.num_rows + 32 * row_waves - 1) / (32 * row_waves);
        job.g = __builtin_amdgcn_readfirstlane(segment / tiles);
        job.row0 = (segment - job.g * tiles) * 32 * row_waves;
        job.pos0 = len - p.by_group.div(job.num_rows);
        // to the position of the tile's last row
        job.kbeg = p.prefix_len + (lo << OwnParts::keys_shift(p));
        job.kend = min(job.pos0 + p.by_group.div(min(job.row0 + 32 * row_waves, job.num_rows) - 1) + 1, p.prefix_len + (hi << OwnParts::keys_shift(p)));
        if (job.kend <= job.kbeg) return;                        // (beyond what its rows see; the join knows)
        job.table = p.block_tables + (int64_t)b * p.max_blocks_per_seq;
        job.slot = p.s_first + (int64_t)me * row_waves;
    }
    job.held_first = job.kbeg >> p.block_shift;
    job.held = job.table[min(job.held_first + lane, (job.kend - 1) >> p.block_shift)];
    if (row_waves == 4) common_body<DT, KV8, D, 4>(p, job);
    else if (row_waves == 2) common_body<DT, KV8, D, 2>(p, job);
    else common_body<DT, KV8, D, 1>(p, job);
}

// N pieces of a lane's row: i0, i0 + 4, ..; of 8 J of their dims the lane's halves.
template <int D, int J, int N> struct JoinBatch {
    static constexpr int kPieceVectors = D / 8 * 64;
    float2 ml[N];
    float4 x[N][J];
    // at(i, row): number of piece i, and how far the row in it lies from row n32; those below n are there
    template <typename At>
    __device__ __forceinline__ void load(const CommonParams& p, const float4* o, int n32, int i0, int n, At at)
    {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int i = i0 + kCommonWaves * k;
            ml[k] = make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int j = 0; j < J; ++j) x[k][j] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (i < n) {
                int row;
                const int64_t piece = at(i, row);
                ml[k] = p.ml[piece * 32 + n32 + row];
                const float4* const from = o + piece * kPieceVectors + row;
#pragma unroll
                for (int j = 0; j < J; ++j) x[k][j] = from[64 * j];
            }
        }
    }
};
template <int J> struct JoinState {
    float m = -INFINITY, l = 0.f;
    float4 acc[J] = {};
    template <int D, int N> __device__ __forceinline__ void add(const JoinBatch<D, J, N>& b)
    {
        float m_new = m;
#pragma unroll
        for (int k = 0; k < N; ++k) m_new = fmaxf(m_new, b.ml[k].x);
        const float f0 = m == -INFINITY ? 0.f : fast_exp2(m - m_new);
        m = m_new;
        l *= f0;
#pragma unroll
        for (int j = 0; j < J; ++j) acc[j].x *= f0, acc[j].y *= f0, acc[j].z *= f0, acc[j].w *= f0;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float f = b.ml[k].x == -INFINITY ? 0.f : fast_exp2(b.ml[k].x - m);
            l = fmaf(f, b.ml[k].y, l);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                acc[j].x = fmaf(f, b.x[k][j].x, acc[j].x), acc[j].y = fmaf(f, b.x[k][j].y, acc[j].y);
                acc[j].z = fmaf(f, b.x[k][j].z, acc[j].z), acc[j].w = fmaf(f, b.x[k][j].w, acc[j].w);
            }
        }
    }
};
// The pieces of 32 rows joined: workgroup (row block x KV head, DIMS dims), the pieces dealt to its four waves.
template <int DT, int D, int DIMS>
__global__ __launch_bounds__(kCommonThreads) void common_join_kernel(const CommonParams p)
{
    constexpr int J = DIMS / 8;
    __shared__ float4 xo[kCommonWaves][J][64];
    __shared__ float2 xml[kCommonWaves][64];
    const int lane = threadIdx.x & 63, n32 = lane & 31, h2 = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = p.by_kv_heads.div(blockIdx.x), g = blockIdx.x - tile * p.num_kv_heads, part = blockIdx.y;
    const int r = 32 * tile + n32, rc = min(r, p.rows - 1), t = p.by_group.div(rc), head = g * p.group + (rc - t * p.group);
    const PlaceGuess guess(p, t);
    OwnParts parts(p, 0);
    JoinState<J> state;
    const float4* const o = p.o + part * J * 64 + n32 + 32 * h2;
    // the prefix's pieces are there for every row, whatever it sees (m = -inf: nothing): those of a wave, four at a time, the
    // first ones under way while it is found out which are the row's own
    JoinBatch<D, J, 4> prefix;
    auto prefix_at = [&](int i, int& row) __attribute__((always_inline)) {
        row = 0;
        return ((int64_t)i * p.num_kv_heads + g) * p.p_slots + tile;
    };
    prefix.load(p, o, n32, wave, p.p_splits, prefix_at);
    // its own: the steps in which it sees a key, and the workgroups that had them
    int n = 0, row_off = 0;
    int64_t piece0 = 0;
    if (p.s_shares > 0) {
        const TokenPlace at = guess.find(p, t);
        const int behind = at.pos(t) + 1 - p.prefix_len;
        const int share = own_share(p, parts);
        int all = 0;
        for (int from = 0;;) {
            parts.number(share, all);
            const int l = at.seq - from;                         // (all lanes exchange)
            const int before = __shfl(parts.before, l & 63), pieces = __shfl(parts.pieces, l & 63), steps = __shfl(parts.steps, l & 63);
            if (behind > 0 && l >= 0 && l < 64) {
                const int in_seq = rc - at.first * p.group, tile_rows = 32 * p.s_row_waves, tile_shift = 31 - __builtin_clz(tile_rows);
                const int tiles = ((at.end - at.first) * p.group + tile_rows - 1) >> tile_shift;
                const int each = OwnParts::each(steps, pieces);
                n = div_by_inverse(OwnParts::steps_of(p, behind) + each - 1, each, __builtin_amdgcn_rcpf((float)each));
                row_off = (in_seq & 31) - n32;
                piece0 = p.s_first + (int64_t)(before + (g * tiles + (in_seq >> tile_shift)) * pieces) * p.s_row_waves + ((in_seq >> 5) & (p.s_row_waves - 1));
            }
            from += 64;
            if (from >= p.num_seqs) break;
            parts = OwnParts(p, from);
        }
    }
    auto own_at = [&](int i, int& row) __attribute__((always_inline)) {
        row = row_off;
        return piece0 + (int64_t)i * p.s_row_waves;
    };
    JoinBatch<D, J, 2> own;
    own.load(p, o, n32, wave, n, own_at);
    state.add(prefix);
    for (int i0 = wave + 4 * kCommonWaves; i0 < p.p_splits; i0 += 4 * kCommonWaves) {
        prefix.load(p, o, n32, i0, p.p_splits, prefix_at);
        state.add(prefix);
    }
    state.add(own);
    for (int i0 = wave + 2 * kCommonWaves, most = wave_max(n); i0 < most; i0 += 2 * kCommonWaves) {
        own.load(p, o, n32, i0, n, own_at);
        state.add(own);
    }
    const float m = state.m, l = state.l;
    const auto& acc = state.acc;
    xml[wave][lane] = make_float2(m, l);
#pragma unroll
    for (int j = 0; j < J; ++j) xo[wave][j][lane] = acc[j];
    __syncthreads();
    if (wave >= J) return;
    // wave w: dims 8w + 4 h2 .. + 3 of the workgroup's
    float m_all = -INFINITY, l_all = 0.f;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < kCommonWaves; ++k) m_all = fmaxf(m_all, xml[k][lane].x);
#pragma unroll
    for (int k = 0; k < kCommonWaves; ++k) {
        const float2 t2 = xml[k][lane];
        const float f = t2.x == -INFINITY ? 0.f : fast_exp2(t2.x - m_all);
        const float4 x = xo[k][wave][lane];
        l_all = fmaf(f, t2.y, l_all);
        s.x = fmaf(f, x.x, s.x), s.y = fmaf(f, x.y, s.y), s.z = fmaf(f, x.z, s.z), s.w = fmaf(f, x.w, s.w);
    }
    if (r >= p.rows) return;
    // (a row that sees no key: +0; a sum that is no number stays one)
    const float inv = l_all == 0.f ? 0.f : (p.v_scales ? p.v_scales[g] : p.out_scale) / l_all;
    uint2 packed;
    packed.x = l_all == 0.f ? 0u : narrow2<DT>(s.x * inv, s.y * inv);
    packed.y = l_all == 0.f ? 0u : narrow2<DT>(s.z * inv, s.w * inv);
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + ((int64_t)t * p.num_heads + head) * D + part * DIMS + 8 * wave + 4 * h2) = packed;
}

}  // namespace optgqa
