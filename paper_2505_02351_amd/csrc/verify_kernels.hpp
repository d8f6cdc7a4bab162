// Verification of drafted tokens: draft i of a sequence, token x, is kept iff u_i q_i(x) < p_i(x), up to the first that is
// not; there the sequence's next token is drawn from max(p - q, 0), or behind the last kept draft from p: the lowest index j with
//     sum of the entries up to j  >  u * sum of all entries.
//
// The comparison's product and all differences and sums are taken in 64 bits (p and q in 32: the differences and the
// product are exact or nearly so), so that a draw depends on no order of summation that a program could see.
//
// Bound by memory: one row of p and one of q per sequence, everything else is a few scattered entries.  Rows are long
// (10^4 to 10^5 entries) and sequences few, so a row is cut into chunks of 1 024 entries, a wave each, with all its loads in
// flight at once; they leave their sums.  In a second launch a wave for each sequence looks up the chunk that the draw falls in and reads
// that one again; rows of up to 32 chunks mostly have both in one.  What is left is latency: three dependent round trips to memory to judge the drafts, one for the row, then two in the second
// launch.
// Measured: 64 sequences of 128 255 entries, fp32: 17.6 us (kernels 13.5, 4.9 TB/s, and 4.3), bf16 17.3, certain drafts 14.1; one of 32 000: 8.6, the call.
#pragma once
#include "common.hpp"

namespace optgqa {

constexpr int kF32 = 2;                     // probabilities may be fp32 as well
constexpr int kVerifyThreads = 256;         // of a workgroup of the first launch
constexpr int kVerifyEach = 16;             // entries of a lane
constexpr int kVerifyChunk = 64 * kVerifyEach;

// What the drafts of a sequence came to.
struct Verdict {
    int kept;
    int minus;                              // 1: the row of q is taken off
    int64_t drop;                           // entry that counts as 0 (a certain draft's), or -1
};

struct VerifyParams {
    int64_t* tokens;            // [B][max_drafts + 1]
    int32_t* accepted;          // [B]
    const void* target;         // [drafts + B][V], rows target_stride elements apart
    const void* draft;          // [drafts][V] or nullptr: every draft was certain
    const int64_t* draft_tokens;
    const int32_t* cu;          // [B + 1]
    const float *accept_u, *sample_u;
    double2* sums;              // [B][chunks]: of the entries to draw from, of p
    Verdict* verdicts;          // [B]
    int64_t target_stride, draft_stride;
    int vocab, max_drafts, chunks;
    int looked_at;              // drafts of a sequence at most: max_drafts, or 0 where there are none at all
};

template <int DT> constexpr int kProbabilityBytes = DT == kF32 ? 4 : 2;

template <int DT> __device__ __forceinline__ float probability(const unsigned char* row, int64_t e)
{
    if constexpr (DT == kF32) return reinterpret_cast<const float*>(row)[e];
    else return widen_lo<DT>(reinterpret_cast<const uint16_t*>(row)[e]);
}

// Entries of a lane of the wave that has those from e0 on: its own one behind another (CONSECUTIVE), or the lanes' 16-byte pieces side by
// side, as memory likes them where the order does not matter.
template <int DT, bool CONSECUTIVE> __device__ __forceinline__ int64_t entry_of(int64_t e0, int i)
{
    constexpr int VEC = 16 / kProbabilityBytes<DT>;
    const int lane = threadIdx.x & 63;
    return e0 + (CONSECUTIVE ? lane * kVerifyEach + i : (i / VEC * 64 + lane) * VEC + i % VEC);
}

// a lane's entries of a row, those from n on 0; rows lie on their elements only
template <int DT, bool CONSECUTIVE> __device__ __forceinline__ void probabilities(const unsigned char* row, int64_t e0, int64_t n, float (&x)[kVerifyEach])
{
    constexpr int ES = kProbabilityBytes<DT>, VEC = 16 / ES;
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4), aligned(2)));      // (one load all the same: the hardware takes any address)
#pragma unroll
    for (int i = 0; i < kVerifyEach; i += VEC) {
        const int64_t e = entry_of<DT, CONSECUTIVE>(e0, i);
        if (e + VEC <= n) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(row + e * ES);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                if constexpr (DT == kF32) x[i + j] = __uint_as_float(w[j & 3]);
                else x[i + j] = j & 1 ? widen_hi<DT>(w[j >> 1]) : widen_lo<DT>(w[j >> 1]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) x[i + j] = e + j < n ? probability<DT>(row, e + j) : 0.f;
        }
    }
}

// A sequence's rows from its first draft on.
template <int DT> __device__ __forceinline__ const unsigned char* target_rows(const VerifyParams& a, int b, int c0)
{
    return static_cast<const unsigned char*>(a.target) + ((int64_t)c0 + b) * a.target_stride * kProbabilityBytes<DT>;
}
template <int DT> __device__ __forceinline__ const unsigned char* draft_rows(const VerifyParams& a, int c0)
{
    return static_cast<const unsigned char*>(a.draft) + (int64_t)c0 * a.draft_stride * kProbabilityBytes<DT>;
}

// The same in every lane of a wave.
template <int DT> __device__ __forceinline__ Verdict judge_drafts(const VerifyParams& a, int b, int c0, int count)
{
    constexpr int ES = kProbabilityBytes<DT>;
    const int lane = threadIdx.x & 63;
    const unsigned char *const target = target_rows<DT>(a, b, c0), *const draft = draft_rows<DT>(a, c0);
    Verdict v{count, 0, -1};
    for (int base = 0; base < count; base += 64) {
        const int i = base + lane;
        bool good = i >= count;
        int64_t token = -1;
        if (i < count) {
            const float u = a.accept_u[(int64_t)c0 + i];
            token = a.draft_tokens[(int64_t)c0 + i];
            if (token >= 0 && token < a.vocab) {
                const float p = probability<DT>(target + i * a.target_stride * ES, token);
                const float q = a.draft ? probability<DT>(draft + i * a.draft_stride * ES, token) : 1.f;
                good = (double)u * (double)q < (double)p;
            }
        }
        const uint64_t bad = __builtin_amdgcn_ballot_w64(!good);
        if (bad) {
            const int l = __builtin_ctzll(bad);
            v.kept = base + l;
            token = __shfl((long long)token, l);
            if (token >= 0 && token < a.vocab) {                 // (an id that is none has no row to take off)
                if (a.draft) v.minus = 1;
                else v.drop = token;
            }
            break;
        }
    }
    return v;
}

// an entry counts if it is a positive finite number
__device__ __forceinline__ double counted(double x) { return x > 0.0 && x < __builtin_inf() ? x : 0.0; }

// A lane's entries to draw from, in 64 bits.
template <int DT, bool CONSECUTIVE>
__device__ __forceinline__ void entries(const VerifyParams& a, const unsigned char* p, const unsigned char* q, int64_t drop, int64_t e0, double (&left)[kVerifyEach],
                                        double (&all)[kVerifyEach])
{
    float px[kVerifyEach], qx[kVerifyEach] = {};
    probabilities<DT, CONSECUTIVE>(p, e0, a.vocab, px);
    if (q) probabilities<DT, CONSECUTIVE>(q, e0, a.vocab, qx);
#pragma unroll
    for (int i = 0; i < kVerifyEach; ++i) {
        all[i] = counted(px[i]);
        left[i] = entry_of<DT, CONSECUTIVE>(e0, i) == drop ? 0.0 : counted((double)px[i] - (double)qx[i]);
    }
}

// Sums of a chunk of the entries to draw from and of p, in lane 63.
template <int DT> __device__ __forceinline__ double2 chunk_sums(const VerifyParams& a, int b, int c0, const Verdict& v, int chunk)
{
    constexpr int ES = kProbabilityBytes<DT>;
    double left[kVerifyEach], all[kVerifyEach];
    entries<DT, false>(a, target_rows<DT>(a, b, c0) + v.kept * a.target_stride * ES, v.minus ? draft_rows<DT>(a, c0) + v.kept * a.draft_stride * ES : nullptr,
                       v.drop, (int64_t)chunk * kVerifyChunk, left, all);
    double l = 0.0, p = 0.0;
#pragma unroll
    for (int i = 0; i < kVerifyEach; ++i) l += left[i], p += all[i];
    return make_double2(lane_sums(l), lane_sums(p));
}

// The draw of sequence b by one wave, from the sums of its chunks, and its row of tokens.  Where rounding lets no sum pass the bar, the last
// entry that counts is drawn.
template <int DT> __device__ __forceinline__ void select_token(const VerifyParams& a, int b, int c0, const Verdict& v, const double2* sums)
{
    constexpr int ES = kProbabilityBytes<DT>;
    const int lane = threadIdx.x & 63;
    const double u = a.sample_u[b];
    // a lane has `each` consecutive chunks
    const int each = (a.chunks + 63) / 64, first = lane * each, end = min(first + each, a.chunks);
    double l = 0.0, p = 0.0;
#pragma unroll 4
    for (int c = first; c < end; ++c) l += sums[c].x, p += sums[c].y;
    const double l_to = lane_sums(l), p_to = lane_sums(p), l_total = __shfl(l_to, 63), p_total = __shfl(p_to, 63);
    const bool rest = l_total > 0.0;                             // else nothing is left of p - q: p itself
    const double mine = rest ? l : p, to = rest ? l_to : p_to, bar = u * (rest ? l_total : p_total);
    int64_t token = -1;
    const uint64_t any = __builtin_amdgcn_ballot_w64(mine > 0.0);
    if (any != 0) {
        // the lane and, in it, the chunk whose entries pass the bar
        uint64_t over = __builtin_amdgcn_ballot_w64(mine > 0.0 && to > bar);
        const bool none = over == 0;
        const int w = none ? 63 - __builtin_clzll(any) : __builtin_ctzll(over);
        double before = __shfl(to - mine, w), base = before;
        int chunk = -1;
        for (int c = w * each; c < min((w + 1) * each, a.chunks); ++c) {
            const double x = rest ? sums[c].x : sums[c].y;
            if (x > 0.0) base = before, chunk = c;
            before += x;
            if (x > 0.0 && !none && before > bar) break;
        }
        // the lane and, in it, the entry
        double left[kVerifyEach], all[kVerifyEach];
        entries<DT, true>(a, target_rows<DT>(a, b, c0) + v.kept * a.target_stride * ES, v.minus ? draft_rows<DT>(a, c0) + v.kept * a.draft_stride * ES : nullptr,
                          v.drop, (int64_t)chunk * kVerifyChunk, left, all);
        double own = 0.0;
#pragma unroll
        for (int i = 0; i < kVerifyEach; ++i) own += rest ? left[i] : all[i];
        double sum = base + (lane_sums(own) - own);
        int at = -1, last = -1;
#pragma unroll
        for (int i = 0; i < kVerifyEach; ++i) {
            const double x = rest ? left[i] : all[i];
            sum += x;
            if (x > 0.0) {
                last = i;
                if (at < 0 && sum > bar) at = i;
            }
        }
        over = __builtin_amdgcn_ballot_w64(at >= 0 && !none);
        const uint64_t some = __builtin_amdgcn_ballot_w64(last >= 0);
        const int from = over != 0 ? __builtin_ctzll(over) : 63 - __builtin_clzll(some);
        token = (int64_t)chunk * kVerifyChunk + from * kVerifyEach + __shfl(over != 0 ? at : last, from);
    }
    if (lane == 0) a.accepted[b] = v.kept;
    for (int i = lane; i <= a.max_drafts; i += 64)
        a.tokens[(int64_t)b * (a.max_drafts + 1) + i] = i < v.kept ? a.draft_tokens[(int64_t)c0 + i] : i == v.kept ? token : -1;
}

// Sums of sequence blockIdx.x's rows, a chunk to a wave.
template <int DT>
__global__ __launch_bounds__(kVerifyThreads) void verify_sums_kernel(const VerifyParams a)
{
    const int b = blockIdx.x, lane = threadIdx.x & 63;
    const int chunk = blockIdx.y * (kVerifyThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (chunk >= a.chunks) return;
    const int c0 = a.cu[b], count = min(max(a.cu[b + 1] - c0, 0), a.looked_at);
    const Verdict v = judge_drafts<DT>(a, b, c0, count);
    const double2 s = chunk_sums<DT>(a, b, c0, v, chunk);
    if (lane == 63) {
        a.sums[(int64_t)b * a.chunks + chunk] = s;
        if (chunk == 0) a.verdicts[b] = v;
    }
}

// The draw of sequence blockIdx.x.
template <int DT>
__global__ __launch_bounds__(64) void verify_select_kernel(const VerifyParams a)
{
    const int b = blockIdx.x;
    select_token<DT>(a, b, a.cu[b], a.verdicts[b], a.sums + (int64_t)b * a.chunks);
}

// Both in one launch, for rows of up to two chunks to each of a workgroup's sixteen waves; the same bits.  A call on a stream is bound by its
// launches, and one is always the faster (one sequence of 4 096 entries, fp32: 9.4 us against 12.2, of 32 000 9.4 / 12.2, 64 of 16 000 9.5 / 12.2,
// 256 of 32 000 14.6 / 17.7).  In a graph only the GPU's time counts, and there a workgroup has one CU for a sequence's chunks where two
// launches have one for every four.  Us in a replayed graph, one launch against two, fp32:
//     sequences   16 chunks    20           22           24           28           32
//       1         6.3 / 6.7   6.8 / 6.8    7.1 / 6.8    7.1 / 6.7    7.8 / 6.8    8.3 / 6.7
//      32                     7.2 / 7.5    7.6 / 7.5    7.5 / 7.4    8.1 / 7.6    8.9 / 7.5
//      64         7.7 / 8.3   7.6 / 8.3    8.3 / 8.8    8.5 / 8.8    9.1 / 9.3   10.1 / 9.6
//     128                     9.0 / 10.8   9.3 / 11.0   9.4 / 11.1   9.9 / 11.9  10.9 / 12.4
// so a captured call has two where chunks are more than 20 and sequences fewer than 64.
constexpr int kVerifyOneWaves = 16, kVerifyOneChunks = 2 * kVerifyOneWaves, kVerifyOneQuick = 20, kVerifyOneSeqs = 64;
template <int DT>
__global__ __launch_bounds__(64 * kVerifyOneWaves) void verify_one_kernel(const VerifyParams a)
{
    __shared__ double2 sums[kVerifyOneChunks];
    const int b = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c0 = a.cu[b], count = min(max(a.cu[b + 1] - c0, 0), a.looked_at);
    const Verdict v = judge_drafts<DT>(a, b, c0, count);
    for (int chunk = wave; chunk < a.chunks; chunk += kVerifyOneWaves) {
        const double2 s = chunk_sums<DT>(a, b, c0, v, chunk);
        if (lane == 63) sums[chunk] = s;
    }
    __syncthreads();
    if (wave == 0) select_token<DT>(a, b, c0, v, sums);
}

}  // namespace optgqa
