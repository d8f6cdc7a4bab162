// Verification of drafted tokens: draft i of a sequence, token x, is kept iff u_i q_i(x) < p_i(x), up to the first that is
// not; there the sequence's next token is drawn from max(p - q, 0), or behind the last kept draft from p: the lowest index j with
//     sum of the entries up to j  >  u * sum of all entries.
//
// The comparison's product and all differences and sums are taken in 64 bits (p and q in 32: the differences and the
// product are exact or nearly so), so that a draw depends on no order of summation that a program could see.
//
// Bound by memory: one row of p and one of q per sequence, everything else is a few scattered entries.  Rows are long
// (10^4 to 10^5 entries) and sequences few, so a row is cut into chunks, one workgroup each, which leave their sums; a second launch,
// a workgroup for each sequence, looks up the chunk that the draw falls in and reads that one again.
#pragma once
#include "common.hpp"

namespace optgqa {

constexpr int kF32 = 2;                     // probabilities may be fp32 as well
constexpr int kVerifyThreads = 256;
constexpr int kVerifyChunk = 4096;          // entries

struct VerifyParams {
    int64_t* tokens;            // [B][max_drafts + 1]
    int32_t* accepted;          // [B]
    const void* target;         // [drafts + B][V], rows target_stride elements apart
    const void* draft;          // [drafts][V] or nullptr: every draft was certain
    const int64_t* draft_tokens;
    const int32_t* cu;          // [B + 1]
    const float *accept_u, *sample_u;
    double* sums;               // [B][2][chunks]: of the entries to draw from, of p
    int64_t target_stride, draft_stride;
    int vocab, max_drafts, chunks;
    int looked_at;              // drafts of a sequence at most: max_drafts, or 0 where there are none at all
};

template <int DT> __device__ __forceinline__ float probability(const void* row, int64_t e)
{
    if constexpr (DT == kF32) return static_cast<const float*>(row)[e];
    else return widen_lo<DT>(static_cast<const uint16_t*>(row)[e]);
}

// VEC entries from e on (16 bytes, or one), those from n on 0
template <int DT, int VEC> __device__ __forceinline__ void probabilities(const void* row, int64_t e, int64_t n, float (&x)[VEC])
{
    constexpr int ES = DT == kF32 ? 4 : 2;
    if (VEC > 1 && e + VEC <= n) {
        const uint4 raw = *reinterpret_cast<const uint4*>(static_cast<const unsigned char*>(row) + e * ES);
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            if constexpr (DT == kF32) x[j] = __uint_as_float(w[j & 3]);
            else x[j] = j & 1 ? widen_hi<DT>(w[j >> 1]) : widen_lo<DT>(w[j >> 1]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) x[j] = e + j < n ? probability<DT>(row, e + j) : 0.f;
    }
}

// A sequence's kept drafts and what its next token is drawn from.
struct Verdict {
    int kept;
    const unsigned char *p, *q;             // rows; q may be nullptr
    int64_t drop;                           // entry that counts as 0 (a certain draft's), or -1
};

// The same in every thread of a wave.
template <int DT> __device__ __forceinline__ Verdict judge_drafts(const VerifyParams& a, int b)
{
    constexpr int ES = DT == kF32 ? 4 : 2;
    const int lane = threadIdx.x & 63;
    const int c0 = a.cu[b], count = min(max(a.cu[b + 1] - c0, 0), a.looked_at);
    const unsigned char* const target = static_cast<const unsigned char*>(a.target) + ((int64_t)c0 + b) * a.target_stride * ES;
    const unsigned char* const draft = static_cast<const unsigned char*>(a.draft) + (int64_t)c0 * a.draft_stride * ES;
    Verdict v{count, nullptr, nullptr, -1};
    int64_t token = -1;
    for (int base = 0; base < count; base += 64) {
        const int i = base + lane;
        bool good = i >= count;
        if (i < count) {
            token = a.draft_tokens[(int64_t)c0 + i];
            if (token >= 0 && token < a.vocab) {
                const float p = probability<DT>(target + i * a.target_stride * ES, token);
                const float q = a.draft ? probability<DT>(draft + i * a.draft_stride * ES, token) : 1.f;
                good = (double)a.accept_u[(int64_t)c0 + i] * (double)q < (double)p;
            }
        }
        const uint64_t bad = __builtin_amdgcn_ballot_w64(!good);
        if (bad) {
            const int l = __builtin_ctzll(bad);
            v.kept = base + l;
            token = __shfl((long long)token, l);
            if (token >= 0 && token < a.vocab) {                 // (an id that is none has no row to take off)
                if (a.draft) v.q = draft + v.kept * a.draft_stride * ES;
                else v.drop = token;
            }
            break;
        }
    }
    v.p = target + v.kept * a.target_stride * ES;
    return v;
}

// an entry counts if it is a positive finite number
__device__ __forceinline__ double counted(double x) { return x > 0.0 && x < __builtin_inf() ? x : 0.0; }

__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int off = 32; off; off >>= 1) x += __shfl_xor(x, off);
    return x;
}

// Sums of chunk blockIdx.y of sequence blockIdx.x's rows.
template <int DT, int VEC>
__global__ __launch_bounds__(kVerifyThreads) void verify_sums_kernel(const VerifyParams a)
{
    __shared__ double part[2][kVerifyThreads / 64];
    const int b = blockIdx.x;
    const Verdict v = judge_drafts<DT>(a, b);
    const int64_t e0 = (int64_t)blockIdx.y * kVerifyChunk;
    const int64_t n = min((int64_t)a.vocab, e0 + kVerifyChunk);
    double rest = 0.0, all = 0.0;
#pragma unroll 4
    for (int64_t e = e0 + threadIdx.x * VEC; e < n; e += kVerifyThreads * VEC) {
        float p[VEC], q[VEC] = {};
        probabilities<DT, VEC>(v.p, e, n, p);
        if (v.q) probabilities<DT, VEC>(v.q, e, n, q);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            all += counted(p[j]);
            rest += e + j == v.drop ? 0.0 : counted((double)p[j] - (double)q[j]);
        }
    }
    rest = wave_sum(rest), all = wave_sum(all);
    if ((threadIdx.x & 63) == 0) part[0][threadIdx.x >> 6] = rest, part[1][threadIdx.x >> 6] = all;
    __syncthreads();
    if (threadIdx.x < 2) {
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < kVerifyThreads / 64; ++i) s += part[threadIdx.x][i];
        a.sums[((int64_t)b * 2 + threadIdx.x) * a.chunks + blockIdx.y] = s;
    }
}

// Inclusive sums over the workgroup's threads, in their order; `total` that of all.
__device__ __forceinline__ double scan(double x, double (&part)[kVerifyThreads / 64], double& total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const double y = __shfl_up(x, off);
        if (lane >= off) x += y;
    }
    __syncthreads();                                             // (part may still be read from the last scan)
    if (lane == 63) part[wave] = x;
    __syncthreads();
    double before = 0.0;
    total = 0.0;
#pragma unroll
    for (int i = 0; i < kVerifyThreads / 64; ++i) {
        if (i < wave) before += part[i];
        total += part[i];
    }
    return before + x;
}

// The draw of sequence blockIdx.x, and its row of tokens.
template <int DT, int VEC>
__global__ __launch_bounds__(kVerifyThreads) void verify_select_kernel(const VerifyParams a)
{
    __shared__ double part[kVerifyThreads / 64];
    __shared__ double base_of;
    __shared__ int first_over, last_chunk, first_entry, last_entry;
    const int b = blockIdx.x, tid = threadIdx.x;
    Verdict v = judge_drafts<DT>(a, b);
    if (tid == 0) first_over = 0x7fffffff, last_chunk = -1, first_entry = 0x7fffffff, last_entry = -1;
    // total of what is drawn from; where nothing is left of p - q, p itself
    const double* sums = a.sums + (int64_t)b * 2 * a.chunks;
    double total = 0.0;
    for (int pass = 0; pass < 2; ++pass) {
        total = 0.0;
        for (int c = 0; c < a.chunks; c += kVerifyThreads) {
            double t;
            scan(c + tid < a.chunks ? sums[c + tid] : 0.0, part, t);
            total += t;
        }
        if (total > 0.0) break;                                  // the same for all threads
        sums += a.chunks;
        v.q = nullptr, v.drop = -1;
    }
    const double bar = (double)a.sample_u[b] * total;
    int64_t token = -1;
    if (total > 0.0) {
        // the first chunk whose entries pass the bar (the last that has any, where rounding lets none pass)
        double carry = 0.0;
        for (int c = 0; c < a.chunks; c += kVerifyThreads) {
            double t;
            const double own = c + tid < a.chunks ? sums[c + tid] : 0.0;
            const double over = carry + scan(own, part, t);
            if (own > 0.0) {
                atomicMax(&last_chunk, c + tid);
                if (over > bar) atomicMin(&first_over, c + tid);
            }
            __syncthreads();
            if (own > 0.0 && c + tid == first_over) base_of = over - own;
            carry += t;
            if (first_over != 0x7fffffff) break;
        }
        __syncthreads();
        const bool none = first_over == 0x7fffffff;
        const int chunk = none ? last_chunk : first_over;
        const double base = none ? 0.0 : base_of;
        // a thread's entries of the chunk are consecutive
        constexpr int kEach = kVerifyChunk / kVerifyThreads;
        static_assert(kEach % VEC == 0, "whole loads");
        const int64_t e0 = (int64_t)chunk * kVerifyChunk + tid * kEach;
        double r[kEach], own = 0.0;
#pragma unroll
        for (int i = 0; i < kEach; i += VEC) {
            float p[VEC], q[VEC] = {};
            probabilities<DT, VEC>(v.p, e0 + i, a.vocab, p);
            if (v.q) probabilities<DT, VEC>(v.q, e0 + i, a.vocab, q);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                r[i + j] = e0 + i + j == v.drop ? 0.0 : counted((double)p[j] - (double)q[j]);
                own += r[i + j];
            }
        }
        double t;
        double sum = base + (scan(own, part, t) - own);
        int over = -1, last = -1;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            sum += r[i];
            if (r[i] > 0.0) {
                last = i;
                if (over < 0 && sum > bar) over = i;
            }
        }
        if (over >= 0) atomicMin(&first_entry, tid * kEach + over);
        if (last >= 0) atomicMax(&last_entry, tid * kEach + last);
        __syncthreads();
        token = (int64_t)chunk * kVerifyChunk + (none || first_entry == 0x7fffffff ? last_entry : first_entry);
    }
    if (tid == 0) a.accepted[b] = v.kept;
    const int c0 = a.cu[b];
    for (int i = tid; i <= a.max_drafts; i += kVerifyThreads)
        a.tokens[(int64_t)b * (a.max_drafts + 1) + i] = i < v.kept ? a.draft_tokens[(int64_t)c0 + i] : i == v.kept ? token : -1;
}

}  // namespace optgqa
