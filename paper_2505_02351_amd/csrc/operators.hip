// C ABI of a step of drafted tokens behind a common prompt: rotary positions, rotated cache appends, attention with a prefix that
// all sequences have in common, the verification of drafts.
// Declarations and the meaning of every argument: include/optgqa.h.
#include "optgqa.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "common_prefix_kernels.hpp"
#include "common_prefix_shape.hpp"
#include "host.hpp"
#include "rotary_kernels.hpp"
#include "verify_kernels.hpp"

using namespace optgqa;

namespace {

// What the rotary entry points are called with.
struct RotaryCall {
    void* q_out;
    const void* q;
    void* k_out;
    const void *k, *v;
    void *k_cache, *v_cache;
    const int64_t* slots;
    const int32_t* positions;
    const double* freqs;
    int num_tokens, num_heads, num_kv_heads, head_dim, rotary_dim, interleaved, block_size;
    int64_t q_out_stride, q_stride, k_out_stride, k_stride, v_stride;
    float magnitude;
    bool backward;
    const KvScales* scales;     // E4M3 caches
    int dtype;
};

template <int DT, RotaryTo TO, bool INTERLEAVED>
int launch_rotary_v(const RotaryParams& p, bool wide, dim3 grid, hipStream_t st)
{
    return wide ? launch(rotary_kernel<DT, TO, INTERLEAVED, 8>, grid, dim3(kRotaryThreads), 0, st, p)
                : launch(rotary_kernel<DT, TO, INTERLEAVED, 1>, grid, dim3(kRotaryThreads), 0, st, p);
}

template <RotaryTo TO>
int launch_rotary(const RotaryParams& p, int dtype, bool interleaved, bool wide, dim3 grid, hipStream_t st)
{
    if (dtype == OPTGQA_F16)
        return interleaved ? launch_rotary_v<kF16, TO, true>(p, wide, grid, st) : launch_rotary_v<kF16, TO, false>(p, wide, grid, st);
    return interleaved ? launch_rotary_v<kBF16, TO, true>(p, wide, grid, st) : launch_rotary_v<kBF16, TO, false>(p, wide, grid, st);
}

int rotary_impl(const RotaryCall& c, RotaryTo to, hipStream_t st)
{
    const bool store = to != RotaryTo::kRows;
    if (c.num_tokens < 0 || c.num_heads < 0 || c.num_kv_heads < 0 || (store && (c.num_heads <= 0 || c.num_kv_heads <= 0)) ||
        c.num_heads + (int64_t)c.num_kv_heads <= 0 || c.num_heads > 65535 || c.num_kv_heads > 65535)
        return OPTGQA_ERR_SHAPE;
    if (!dtype_ok(c.dtype) || !head_dim_ok(c.head_dim) || (store && !block_size_ok(c.block_size))) return OPTGQA_ERR_UNSUPPORTED;
    if (c.rotary_dim <= 0 || c.rotary_dim > c.head_dim || c.rotary_dim % 2) return OPTGQA_ERR_SHAPE;
    if (!std::isfinite(c.magnitude)) return OPTGQA_ERR_SHAPE;
    if (to == RotaryTo::kCacheE4M3) {
        if (c.scales->per_head() && !c.scales->v_heads) return OPTGQA_ERR_NULL;
        if (!c.scales->valid()) return OPTGQA_ERR_SHAPE;
    }
    const int64_t q_row = (int64_t)c.num_heads * c.head_dim, kv_row = (int64_t)c.num_kv_heads * c.head_dim;
    if (c.num_heads && (c.q_stride < q_row || c.q_out_stride < q_row)) return OPTGQA_ERR_SHAPE;
    if (c.num_kv_heads && (c.k_stride < kv_row || (store ? c.v_stride < kv_row : c.k_out_stride < kv_row))) return OPTGQA_ERR_SHAPE;
    if (c.num_tokens == 0) return OPTGQA_OK;
    if (!c.positions || !c.freqs || (c.num_heads && (!c.q || !c.q_out)) || (c.num_kv_heads && !c.k)) return OPTGQA_ERR_NULL;
    if (store ? !c.v || !c.k_cache || !c.v_cache || !c.slots : c.num_kv_heads && !c.k_out) return OPTGQA_ERR_NULL;

    // (what a call does not have is a null pointer or a zero stride here, and on any alignment)
    const uintptr_t rows = reinterpret_cast<uintptr_t>(c.q) | reinterpret_cast<uintptr_t>(c.q_out) | reinterpret_cast<uintptr_t>(c.k) |
                           reinterpret_cast<uintptr_t>(c.k_out) | reinterpret_cast<uintptr_t>(c.v);
    const uintptr_t caches = reinterpret_cast<uintptr_t>(c.k_cache) | reinterpret_cast<uintptr_t>(c.v_cache);
    if ((rows & 1u) || (to == RotaryTo::kCache && (caches & 1u)) || (reinterpret_cast<uintptr_t>(c.freqs) & 7u) ||
        (reinterpret_cast<uintptr_t>(c.positions) & 3u))
        return OPTGQA_ERR_UNSUPPORTED;
    const bool wide = !(rows & 15u) && !(caches & (to == RotaryTo::kCacheE4M3 ? 7u : 15u)) && c.rotary_dim % 16 == 0 &&
                      (c.q_stride | c.q_out_stride | c.k_stride | c.k_out_stride | c.v_stride) % 8 == 0;

    RotaryParams p;
    p.k_cache = c.k_cache;
    p.v_cache = c.v_cache;
    p.freqs = c.freqs;
    p.q_stride = c.q_stride;
    p.q_out_stride = c.q_out_stride;
    p.k_stride = c.k_stride;
    p.k_out_stride = c.k_out_stride;
    p.v_stride = c.v_stride;
    p.magnitude = c.magnitude;
    p.sign = c.backward ? -1.f : 1.f;
    p.k_inv_scale = p.v_inv_scale = 1.f;
    p.k_scales = p.v_scales = nullptr;
    if (to == RotaryTo::kCacheE4M3) {
        p.k_scales = c.scales->k_heads;
        p.v_scales = c.scales->v_heads;
        if (!c.scales->per_head()) {
            p.k_inv_scale = 1.0f / c.scales->k;
            p.v_inv_scale = 1.0f / c.scales->v;
        }
    }
    p.q_heads = c.num_heads;
    p.kv_heads = c.num_kv_heads;
    p.heads = c.num_heads + c.num_kv_heads * (store ? 2 : 1);
    p.pairs = c.rotary_dim / 2;
    p.head_dim = c.head_dim;
    p.pieces_shift = __builtin_ctz(c.head_dim / (wide ? 16 : 2));
    p.block_shift = store ? __builtin_ctz(c.block_size) : 0;

    // Many tokens: whole tokens, up to 8, as many as make 512 items for a workgroup's 256 threads, so that a token's angles are
    // worked out once (512: 20 480 tokens of 40 heads of 128 76 us; 1 536: 81, 3 000: 86).  Fewer than four such workgroups to
    // a CU: one token each, its heads dealt to workgroups of one item a thread.
    const int64_t per_token = (int64_t)p.heads << p.pieces_shift;
    p.tokens_per_wg = (int)std::min<int64_t>(std::max<int64_t>(512 / per_token, 1), kRotaryMaxTokens);
    p.heads_per_wg = p.heads;
    if (c.num_tokens < (int64_t)4 * num_cus() * p.tokens_per_wg) {
        p.tokens_per_wg = 1;
        p.heads_per_wg = std::min(p.heads, kRotaryThreads >> p.pieces_shift);
    }
    p.by_heads_per_wg.set((uint32_t)p.heads_per_wg);
    p.by_pairs.set((uint32_t)p.pairs);
    // slices of tokens, one but for 2^24 and more
    const int64_t most = most_workgroups(kRotaryThreads) * p.tokens_per_wg;
    auto from = [](auto* at, int64_t bytes) { return at ? reinterpret_cast<decltype(at)>(reinterpret_cast<uintptr_t>(at) + bytes) : at; };
    for (int64_t first = 0; first < c.num_tokens; first += most) {
        p.q = from(c.q, first * c.q_stride * 2);
        p.q_out = from(c.q_out, first * c.q_out_stride * 2);
        p.k = from(c.k, first * c.k_stride * 2);
        p.k_out = from(c.k_out, first * c.k_out_stride * 2);
        p.v = from(c.v, first * c.v_stride * 2);
        p.slots = c.slots ? c.slots + first : nullptr;
        p.positions = c.positions + first;
        p.num_tokens = (int)std::min(c.num_tokens - first, most);
        const dim3 grid((unsigned)(((int64_t)p.num_tokens + p.tokens_per_wg - 1) / p.tokens_per_wg),
                        (unsigned)((p.heads + p.heads_per_wg - 1) / p.heads_per_wg));
        const int rc = to == RotaryTo::kRows    ? launch_rotary<RotaryTo::kRows>(p, c.dtype, c.interleaved != 0, wide, grid, st)
                       : to == RotaryTo::kCache ? launch_rotary<RotaryTo::kCache>(p, c.dtype, c.interleaved != 0, wide, grid, st)
                                                : launch_rotary<RotaryTo::kCacheE4M3>(p, c.dtype, c.interleaved != 0, wide, grid, st);
        if (rc != OPTGQA_OK) return rc;
    }
    return OPTGQA_OK;
}

int rotary_and_cache_impl(void* q_out, const void* q, const void* k, const void* v, void* k_cache, void* v_cache,
                          const int64_t* slot_mapping, const int32_t* positions, const double* freqs, int num_tokens, int num_heads,
                          int num_kv_heads, int head_dim, int rotary_dim, int interleaved, float magnitude, int block_size,
                          int64_t q_out_stride, int64_t q_stride, int64_t k_stride, int64_t v_stride, const KvScales* scales, int dtype, void* stream)
{
    const RotaryCall c{q_out, q, nullptr, k, v, k_cache, v_cache, slot_mapping, positions, freqs, num_tokens, num_heads, num_kv_heads, head_dim,
                       rotary_dim, interleaved, block_size, q_out_stride, q_stride, 0, k_stride, v_stride, magnitude, false, scales, dtype};
    return rotary_impl(c, scales ? RotaryTo::kCacheE4M3 : RotaryTo::kCache, static_cast<hipStream_t>(stream));
}

// Whether calls on this stream are recorded for a graph (the null stream never is).
bool is_captured(hipStream_t st)
{
    hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
    return st && hipStreamIsCapturing(st, &status) == hipSuccess && status == hipStreamCaptureStatusActive;
}

template <int DT>
int launch_verify(const VerifyParams& a, int num_seqs, hipStream_t st)
{
    if (a.chunks <= kVerifyOneChunks && !(a.chunks > kVerifyOneQuick && num_seqs < kVerifyOneSeqs && is_captured(st)))
        return launch(verify_one_kernel<DT>, dim3(num_seqs), dim3(64 * kVerifyOneWaves), 0, st, a);
    constexpr int kWaves = kVerifyThreads / 64;
    const int rc = launch(verify_sums_kernel<DT>, dim3(num_seqs, (a.chunks + kWaves - 1) / kWaves), dim3(kVerifyThreads), 0, st, a);
    return rc != OPTGQA_OK ? rc : launch(verify_select_kernel<DT>, dim3(num_seqs), dim3(64), 0, st, a);
}

template <int DT, bool KV8, int D>
int launch_common(const CommonParams& p, int workgroups, hipStream_t st)
{
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&common_prefix_kernel<DT, KV8, D>),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, kCommonLds<D, KV8>);
    if (attr != hipSuccess) return OPTGQA_ERR_LAUNCH;
    if (workgroups > 0) {
        const int rc = launch(common_prefix_kernel<DT, KV8, D>, dim3(workgroups), dim3(kCommonThreads), kCommonLds<D, KV8>, st, p);
        if (rc != OPTGQA_OK) return rc;
    }
    // 32 dims to a workgroup of the join, 16 where those would not be one to a CU (16 sequences of 32 / 8 heads of 128 behind 6 528
    // tokens: 16.0 us against 16.4; 32 of 3 - 6 new tokens each, 40 / 8 heads: 47.1 against 44.9)
    const int tiles = p.p_slots * p.num_kv_heads;
    return (int64_t)tiles * (D / 32) < num_cus() ? launch(common_join_kernel<DT, D, 16>, dim3(tiles, D / 16), dim3(kCommonThreads), 0, st, p)
                                                 : launch(common_join_kernel<DT, D, 32>, dim3(tiles, D / 32), dim3(kCommonThreads), 0, st, p);
}

template <int DT, bool KV8>
int launch_common_d(const CommonParams& p, int head_dim, int workgroups, hipStream_t st)
{
    return head_dim == 128 ? launch_common<DT, KV8, 128>(p, workgroups, st) : launch_common<DT, KV8, 64>(p, workgroups, st);
}

int common_impl(void* out, const void* q, const void* k_cache, const void* v_cache, const int32_t* prefix_table,
                const int32_t* block_tables, const int32_t* context_lens, const int32_t* cu_q_lens, const float* alibi_slopes, float scale,
                int num_tokens, int num_seqs, int num_heads, int num_kv_heads, int head_dim, int block_size, int num_prefix_blocks,
                int max_blocks_per_seq, int max_context_len, int max_q_len, void* workspace, size_t workspace_bytes, int dtype,
                const KvScales* scales, void* stream)
{
    if (num_tokens < 0 || num_seqs < 0 || num_heads <= 0 || num_kv_heads <= 0 || head_dim <= 0 || block_size <= 0 || num_prefix_blocks < 0 ||
        max_blocks_per_seq < 0 || max_context_len < 0 || max_q_len < 0)
        return OPTGQA_ERR_SHAPE;
    if (!std::isfinite(scale) || num_heads % num_kv_heads || num_heads > 65535) return OPTGQA_ERR_SHAPE;
    if (!dtype_ok(dtype) || !head_dim_ok(head_dim) || !block_size_ok(block_size)) return OPTGQA_ERR_UNSUPPORTED;
    const int64_t prefix_len = (int64_t)num_prefix_blocks * block_size;
    if (max_context_len > (int64_t)max_blocks_per_seq * block_size && max_context_len > prefix_len) return OPTGQA_ERR_SHAPE;
    if (prefix_len > (1ll << 30) || max_context_len > (1 << 30)) return OPTGQA_ERR_SHAPE;
    if (scales && scales->per_head() && !scales->v_heads) return OPTGQA_ERR_NULL;
    if (scales && !scales->valid()) return OPTGQA_ERR_SHAPE;
    if (num_tokens == 0) return OPTGQA_OK;
    if (num_seqs == 0 || (!cu_q_lens && num_tokens != num_seqs)) return OPTGQA_ERR_SHAPE;
    if (max_q_len == 0) return OPTGQA_ERR_SHAPE;
    if (!out || !q || !k_cache || !v_cache || !context_lens || (num_prefix_blocks && !prefix_table) || (max_context_len > prefix_len && !block_tables))
        return OPTGQA_ERR_NULL;
    if (!aligned16(out) || !aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache)) return OPTGQA_ERR_UNSUPPORTED;
    CommonPlan c;
    if (!plan_common(c, num_tokens, num_seqs, num_heads, num_kv_heads, prefix_len, max_context_len, cu_q_lens ? max_q_len : 1, num_cus())) return OPTGQA_ERR_SHAPE;
    if (!workspace || !aligned16(workspace) || workspace_bytes < c.bytes(head_dim)) return OPTGQA_ERR_WORKSPACE;

    CommonParams p;
    p.out = out;
    p.q = q;
    p.k_cache = k_cache;
    p.v_cache = v_cache;
    p.prefix_table = prefix_table;
    p.block_tables = block_tables;
    p.context_lens = context_lens;
    p.cu_q_lens = cu_q_lens;
    p.slopes = alibi_slopes;
    p.scale2 = prefill_scale2(scale);                            // (the bias rides in the scores here too)
    p.out_scale = 1.f;
    p.k_scales = p.v_scales = nullptr;
    if (scales && scales->per_head()) {
        p.k_scales = scales->k_heads;
        p.v_scales = scales->v_heads;
    } else if (scales) {
        p.scale2 *= scales->k;
        p.out_scale = scales->v;
    }
    p.num_tokens = num_tokens;
    p.num_seqs = num_seqs;
    p.num_heads = num_heads;
    p.num_kv_heads = num_kv_heads;
    p.group = num_heads / num_kv_heads;
    p.block_shift = __builtin_ctz(block_size);
    p.max_blocks_per_seq = max_blocks_per_seq;
    p.prefix_len = (int)prefix_len;
    p.rows = (int)c.rows;
    p.p_row_waves = c.p_row_waves;
    p.p_tiles = c.p_tiles;
    p.p_splits = c.p_splits;
    p.p_keys = c.p_keys;
    p.p_items.set(num_kv_heads, c.p_splits, c.p_tiles);
    p.s_row_waves = c.s_row_waves;
    p.s_shares = c.s_shares;
    p.p_slots = (int)c.p_slots;
    p.s_first = c.p_pieces(num_kv_heads);
    const size_t pieces = (size_t)c.pieces(num_kv_heads);
    p.o = static_cast<float4*>(workspace);
    p.ml = reinterpret_cast<float2*>(static_cast<unsigned char*>(workspace) + pieces * 32 * head_dim * sizeof(float));
    p.by_group.set((uint32_t)p.group);
    p.by_kv_heads.set((uint32_t)num_kv_heads);
    p.by_s_shares.set((uint32_t)std::max(c.s_shares, 1));
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int workgroups = (int)c.workgroups();
    if (dtype == OPTGQA_F16)
        return scales ? launch_common_d<kF16, true>(p, head_dim, workgroups, st) : launch_common_d<kF16, false>(p, head_dim, workgroups, st);
    return scales ? launch_common_d<kBF16, true>(p, head_dim, workgroups, st) : launch_common_d<kBF16, false>(p, head_dim, workgroups, st);
}

}  // namespace

static_assert(kF16 == OPTGQA_F16 && kBF16 == OPTGQA_BF16 && kF32 == OPTGQA_F32, "the header's values");

extern "C" {

int optgqa_rotary_frequencies_host(double* freqs_host, float* magnitude_host, int rotary_dim, double base, int scaling, double factor,
                                   double original_len, double a, double b)
{
    if (!freqs_host || !magnitude_host) return OPTGQA_ERR_NULL;
    if (rotary_dim <= 0 || rotary_dim % 2 || !(base > 1.0) || !std::isfinite(base)) return OPTGQA_ERR_SHAPE;
    if (scaling < OPTGQA_ROTARY_PLAIN || scaling > OPTGQA_ROTARY_WAVELENGTH) return OPTGQA_ERR_UNSUPPORTED;
    if (scaling != OPTGQA_ROTARY_PLAIN && !(factor >= 1.0 && std::isfinite(factor))) return OPTGQA_ERR_SHAPE;
    const bool by_length = scaling == OPTGQA_ROTARY_YARN || scaling == OPTGQA_ROTARY_WAVELENGTH;
    if (by_length && !(original_len > 0.0 && std::isfinite(original_len) && a > 0.0 && b > 0.0 && std::isfinite(a) && std::isfinite(b)))
        return OPTGQA_ERR_SHAPE;
    if (scaling == OPTGQA_ROTARY_YARN && !(a > b)) return OPTGQA_ERR_SHAPE;
    if (scaling == OPTGQA_ROTARY_WAVELENGTH && !(b > a)) return OPTGQA_ERR_SHAPE;
    if (scaling == OPTGQA_ROTARY_BASE && rotary_dim <= 2) return OPTGQA_ERR_SHAPE;
    const double two_pi = 6.283185307179586476925;
    const int pairs = rotary_dim / 2;
    if (scaling == OPTGQA_ROTARY_BASE) base *= std::pow(factor, rotary_dim / (rotary_dim - 2.0));
    // YaRN: the pair that makes `turns` turns over the original length
    auto pair_of = [&](double turns) { return rotary_dim * std::log(original_len / (turns * two_pi)) / (2.0 * std::log(base)); };
    double lo = 0.0, hi = 0.0;
    if (scaling == OPTGQA_ROTARY_YARN) {
        lo = std::max(std::floor(pair_of(a)), 0.0);
        hi = std::min(std::ceil(pair_of(b)), rotary_dim - 1.0);
    }
    for (int i = 0; i < pairs; ++i) {
        double f = std::pow(base, -2.0 * i / rotary_dim);
        if (scaling == OPTGQA_ROTARY_LINEAR) f /= factor;
        if (scaling == OPTGQA_ROTARY_YARN) {
            const double ramp = std::min(std::max((i - lo) / std::max(hi - lo, 0.001), 0.0), 1.0);
            f = f * (1.0 - ramp) + f / factor * ramp;
        }
        if (scaling == OPTGQA_ROTARY_WAVELENGTH) {
            const double turns = original_len * f / two_pi;                  // over the original length
            const double keep = std::min(std::max((turns - a) / (b - a), 0.0), 1.0);
            f = f * keep + f / factor * (1.0 - keep);
        }
        freqs_host[i] = f;
    }
    *magnitude_host = scaling == OPTGQA_ROTARY_YARN ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
    return OPTGQA_OK;
}

int optgqa_rotary_embedding(void* q_out, const void* q, void* k_out, const void* k, const int32_t* positions, const double* freqs,
                            int num_tokens, int num_heads, int num_kv_heads, int head_dim, int rotary_dim, int interleaved,
                            float magnitude, int backward, int64_t q_out_stride, int64_t q_stride, int64_t k_out_stride,
                            int64_t k_stride, int dtype, void* stream)
{
    const RotaryCall c{q_out, q, k_out, k, nullptr, nullptr, nullptr, nullptr, positions, freqs, num_tokens, num_heads, num_kv_heads, head_dim,
                       rotary_dim, interleaved, 16, q_out_stride, q_stride, k_out_stride, k_stride, 0, magnitude, backward != 0, nullptr, dtype};
    return rotary_impl(c, RotaryTo::kRows, static_cast<hipStream_t>(stream));
}

int optgqa_rotary_and_cache(void* q_out, const void* q, const void* k, const void* v, void* k_cache, void* v_cache,
                            const int64_t* slot_mapping, const int32_t* positions, const double* freqs, int num_tokens,
                            int num_heads, int num_kv_heads, int head_dim, int rotary_dim, int interleaved, float magnitude,
                            int block_size, int64_t q_out_stride, int64_t q_stride, int64_t k_stride, int64_t v_stride, int dtype,
                            void* stream)
{
    return rotary_and_cache_impl(q_out, q, k, v, k_cache, v_cache, slot_mapping, positions, freqs, num_tokens, num_heads, num_kv_heads, head_dim,
                                 rotary_dim, interleaved, magnitude, block_size, q_out_stride, q_stride, k_stride, v_stride, nullptr, dtype, stream);
}

int optgqa_rotary_and_cache_fp8(void* q_out, const void* q, const void* k, const void* v, void* k_cache, void* v_cache,
                                const int64_t* slot_mapping, const int32_t* positions, const double* freqs, int num_tokens,
                                int num_heads, int num_kv_heads, int head_dim, int rotary_dim, int interleaved, float magnitude,
                                int block_size, int64_t q_out_stride, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                                float k_scale, float v_scale, int dtype, void* stream)
{
    const KvScales scales{k_scale, v_scale, nullptr, nullptr};
    return rotary_and_cache_impl(q_out, q, k, v, k_cache, v_cache, slot_mapping, positions, freqs, num_tokens, num_heads, num_kv_heads, head_dim,
                                 rotary_dim, interleaved, magnitude, block_size, q_out_stride, q_stride, k_stride, v_stride, &scales, dtype, stream);
}

int optgqa_rotary_and_cache_fp8_heads(void* q_out, const void* q, const void* k, const void* v, void* k_cache, void* v_cache,
                                      const int64_t* slot_mapping, const int32_t* positions, const double* freqs, int num_tokens,
                                      int num_heads, int num_kv_heads, int head_dim, int rotary_dim, int interleaved,
                                      float magnitude, int block_size, int64_t q_out_stride, int64_t q_stride, int64_t k_stride,
                                      int64_t v_stride, const float* k_scales, const float* v_scales, int dtype, void* stream)
{
    if (!k_scales || !v_scales) return OPTGQA_ERR_NULL;
    const KvScales scales{0.f, 0.f, k_scales, v_scales};
    return rotary_and_cache_impl(q_out, q, k, v, k_cache, v_cache, slot_mapping, positions, freqs, num_tokens, num_heads, num_kv_heads, head_dim,
                                 rotary_dim, interleaved, magnitude, block_size, q_out_stride, q_stride, k_stride, v_stride, &scales, dtype, stream);
}

size_t optgqa_verify_drafts_workspace_bytes(int num_seqs, int vocab_size)
{
    if (num_seqs <= 0 || vocab_size <= 0) return 0;
    return (size_t)num_seqs * (((size_t)vocab_size + kVerifyChunk - 1) / kVerifyChunk * sizeof(double2) + sizeof(Verdict));
}

int optgqa_verify_drafts(int64_t* tokens, int32_t* num_accepted, const void* target_probs, const void* draft_probs,
                         const int64_t* draft_tokens, const int32_t* cu_draft_lens, const float* accept_uniforms,
                         const float* sample_uniforms, int num_seqs, int vocab_size, int max_drafts, int64_t target_stride,
                         int64_t draft_stride, void* workspace, size_t workspace_bytes, int dtype, void* stream)
{
    if (num_seqs < 0 || vocab_size <= 0 || max_drafts < 0 || target_stride < vocab_size || (draft_probs && draft_stride < vocab_size))
        return OPTGQA_ERR_SHAPE;
    if (!dtype_ok(dtype) && dtype != OPTGQA_F32) return OPTGQA_ERR_UNSUPPORTED;
    const int chunks = (int)(((int64_t)vocab_size + kVerifyChunk - 1) / kVerifyChunk);
    if (chunks > 4 * 65535 || num_seqs > most_workgroups(64 * kVerifyOneWaves)) return OPTGQA_ERR_SHAPE;     // (2^28 entries, 2^22 sequences)
    if (num_seqs == 0) return OPTGQA_OK;
    if (!tokens || !num_accepted || !target_probs || !cu_draft_lens || !sample_uniforms)
        return OPTGQA_ERR_NULL;
    const uintptr_t size = dtype == OPTGQA_F32 ? 4 : 2, rows = reinterpret_cast<uintptr_t>(target_probs) | reinterpret_cast<uintptr_t>(draft_probs);
    if ((rows & (size - 1)) || ((reinterpret_cast<uintptr_t>(tokens) | reinterpret_cast<uintptr_t>(draft_tokens)) & 7u) ||
        ((reinterpret_cast<uintptr_t>(num_accepted) | reinterpret_cast<uintptr_t>(cu_draft_lens) | reinterpret_cast<uintptr_t>(accept_uniforms) |
          reinterpret_cast<uintptr_t>(sample_uniforms)) & 3u))
        return OPTGQA_ERR_UNSUPPORTED;
    if (!workspace || !aligned16(workspace) || workspace_bytes < optgqa_verify_drafts_workspace_bytes(num_seqs, vocab_size)) return OPTGQA_ERR_WORKSPACE;
    VerifyParams a;
    a.tokens = tokens;
    a.accepted = num_accepted;
    a.target = target_probs;
    a.draft = draft_probs;
    a.draft_tokens = draft_tokens;
    a.cu = cu_draft_lens;
    a.accept_u = accept_uniforms;
    a.sample_u = sample_uniforms;
    a.sums = static_cast<double2*>(workspace);
    a.verdicts = reinterpret_cast<Verdict*>(a.sums + (size_t)num_seqs * chunks);
    a.target_stride = target_stride;
    a.draft_stride = draft_stride;
    a.vocab = vocab_size;
    a.max_drafts = max_drafts;
    a.looked_at = draft_tokens && accept_uniforms ? max_drafts : 0;
    a.chunks = chunks;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == OPTGQA_F32) return launch_verify<kF32>(a, num_seqs, st);
    return dtype == OPTGQA_F16 ? launch_verify<kF16>(a, num_seqs, st) : launch_verify<kBF16>(a, num_seqs, st);
}

size_t optgqa_common_prefix_workspace_bytes(int num_tokens, int num_seqs, int num_heads, int num_kv_heads, int head_dim,
                                            int block_size, int num_prefix_blocks, int max_context_len, int max_q_len)
{
    if (num_tokens <= 0 || num_seqs <= 0 || num_heads <= 0 || num_heads > 65535 || num_kv_heads <= 0 || num_heads % num_kv_heads || !head_dim_ok(head_dim) ||
        !block_size_ok(block_size) || num_prefix_blocks < 0 || max_context_len < 0 || max_q_len <= 0)
        return 0;
    // (without prefix sums of new tokens a sequence has one, whatever the bound: the call needs the larger of the two)
    size_t bytes = 16;
    for (const int n : {max_q_len, 1}) {
        CommonPlan c;
        if (!plan_common(c, num_tokens, num_seqs, num_heads, num_kv_heads, (int64_t)num_prefix_blocks * block_size, max_context_len, n, num_cus())) return 0;
        bytes = std::max(bytes, c.bytes(head_dim));
    }
    return bytes;
}

int optgqa_paged_attention_common(void* out, const void* q, const void* k_cache, const void* v_cache, const int32_t* prefix_table,
                                  const int32_t* block_tables, const int32_t* context_lens, const int32_t* cu_q_lens,
                                  const float* alibi_slopes, float scale, int num_tokens, int num_seqs, int num_heads, int num_kv_heads,
                                  int head_dim, int block_size, int num_prefix_blocks, int max_blocks_per_seq, int max_context_len,
                                  int max_q_len, void* workspace, size_t workspace_bytes, int dtype, void* stream)
{
    return common_impl(out, q, k_cache, v_cache, prefix_table, block_tables, context_lens, cu_q_lens, alibi_slopes, scale, num_tokens, num_seqs,
                       num_heads, num_kv_heads, head_dim, block_size, num_prefix_blocks, max_blocks_per_seq, max_context_len, max_q_len, workspace,
                       workspace_bytes, dtype, nullptr, stream);
}

int optgqa_paged_attention_common_fp8(void* out, const void* q, const void* k_cache, const void* v_cache, const int32_t* prefix_table,
                                  const int32_t* block_tables, const int32_t* context_lens, const int32_t* cu_q_lens,
                                  const float* alibi_slopes, float scale, float k_scale, float v_scale, int num_tokens, int num_seqs, int num_heads, int num_kv_heads,
                                  int head_dim, int block_size, int num_prefix_blocks, int max_blocks_per_seq, int max_context_len,
                                  int max_q_len, void* workspace, size_t workspace_bytes, int dtype, void* stream)
{
    const KvScales scales{k_scale, v_scale, nullptr, nullptr};
    return common_impl(out, q, k_cache, v_cache, prefix_table, block_tables, context_lens, cu_q_lens, alibi_slopes, scale, num_tokens, num_seqs,
                       num_heads, num_kv_heads, head_dim, block_size, num_prefix_blocks, max_blocks_per_seq, max_context_len, max_q_len, workspace,
                       workspace_bytes, dtype, &scales, stream);
}

int optgqa_paged_attention_common_fp8_heads(void* out, const void* q, const void* k_cache, const void* v_cache, const int32_t* prefix_table,
                                  const int32_t* block_tables, const int32_t* context_lens, const int32_t* cu_q_lens,
                                  const float* alibi_slopes, float scale, const float* k_scales, const float* v_scales, int num_tokens, int num_seqs, int num_heads, int num_kv_heads,
                                  int head_dim, int block_size, int num_prefix_blocks, int max_blocks_per_seq, int max_context_len,
                                  int max_q_len, void* workspace, size_t workspace_bytes, int dtype, void* stream)
{
    if (!k_scales || !v_scales) return OPTGQA_ERR_NULL;
    const KvScales scales{0.f, 0.f, k_scales, v_scales};
    return common_impl(out, q, k_cache, v_cache, prefix_table, block_tables, context_lens, cu_q_lens, alibi_slopes, scale, num_tokens, num_seqs,
                       num_heads, num_kv_heads, head_dim, block_size, num_prefix_blocks, max_blocks_per_seq, max_context_len, max_q_len, workspace,
                       workspace_bytes, dtype, &scales, stream);
}

}  // extern "C"
