// Rotary positions, alone or on the way into the paged caches.
//
// Pair i of a head's first rotary_dim dims, (x, y) = dims (i, i + rotary_dim / 2) or, interleaved, (2i, 2i + 1), of the
// token at position p turns by a = p * freqs[i]:
//     x' = m (x cos a - y sin a),   y' = m (y cos a + x sin a),      m: the caller's magnitude
// and the dims from rotary_dim on pass through.  The gradient is the transpose: the same with -a.
//
// Angles: the product p * freqs[i] and its remainder modulo a whole turn are taken in 64 bits - in 32, position 100 000 would
// be known to 2^-8 of a radian, a bf16 value's whole precision - sine and cosine of the remainder in 32.
//
// Bound by memory: every row is read and written once, and the trigonometry (some 60 instructions a pair) must not show.
// It is the same for all heads of a token, so a workgroup works it out once per (token, pair), into LDS, and its threads
// then take (token, head, piece) items.  A piece is 8 pairs - two 16-byte loads and stores - or, past those, 16 dims
// that pass through; where rows do not lie on 16 bytes or rotary_dim is no multiple of 16, one pair.  (Measured, inputs in
// turn: 20 480 tokens, 32 / 8 heads of 128, bf16: 76 us, 5.5 TB/s, a large copy reaches 5.1; 4 099 tokens, 40 / 8 heads, the gradient of
// 64 interleaved dims, fp16: 21.6 us; 2 943 tokens into E4M3 caches 13.5 us; one token 1.9 us.  Non-temporal loads: 72, 22 and 17 us, and
// the rows of a step are what the projection before has just written, so they are not taken.)
#pragma once
#include "common.hpp"

namespace optgqa {

constexpr int kRotaryThreads = 256;
constexpr int kRotaryMaxTokens = 8;         // of a workgroup (its angles: 8 x 64 pairs of 8 bytes in LDS)

struct RotaryParams {
    const void* q;              // [T][Hq][D], token strides in elements
    void* q_out;
    const void* k;              // [T][Hkv][D]
    void* k_out;                // rotary_embedding only
    const void* v;              // the cache stores only
    void* k_cache;
    void* v_cache;
    const int64_t* slots;
    const int32_t* positions;
    const double* freqs;        // [pairs], radians a token
    int64_t q_stride, q_out_stride, k_stride, k_out_stride, v_stride;
    float magnitude, sign;      // sign: -1 for the gradient
    float k_inv_scale, v_inv_scale;                 // E4M3 caches: one pair per tensor, or
    const float *k_scales, *v_scales;               // one per KV head
    int num_tokens, q_heads, kv_heads, heads;       // heads: of a token in all, q, k, then v
    int pairs, head_dim, pieces_shift;              // log2 of the pieces of a head
    int block_shift;
    int tokens_per_wg, heads_per_wg;                // of a workgroup (blockIdx.x, blockIdx.y)
    FastDiv by_heads_per_wg, by_pairs;
};

enum class RotaryTo { kRows, kCache, kCacheE4M3 };

// (x, y) turned by (cos, sin) = w.  Which product an FMA takes is said here, not left to the compiler: every kernel below, and so
// rows turned alone and rows turned on their way into a cache, give the same bits.
__device__ __forceinline__ void turn_pair(float& x, float& y, float2 w)
{
    const float nx = fmaf(x, w.x, -(y * w.y)), ny = fmaf(y, w.x, x * w.y);
    x = nx, y = ny;
}

// VEC: pairs of a piece
template <int DT, RotaryTo TO, bool INTERLEAVED, int VEC>
__global__ __launch_bounds__(kRotaryThreads) void rotary_kernel(const RotaryParams p)
{
    static_assert(VEC == 8 || VEC == 1, "two 16-byte pieces, or a pair");
    __shared__ float2 turn[kRotaryMaxTokens * 64];
    __shared__ int64_t slot_of[kRotaryMaxTokens];
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    const int t0 = blockIdx.x * p.tokens_per_wg, tokens = min(p.tokens_per_wg, p.num_tokens - t0);
    const int h0 = blockIdx.y * p.heads_per_wg, heads = min(p.heads_per_wg, p.heads - h0);

    for (int i = threadIdx.x; i < tokens * p.pairs; i += kRotaryThreads) {
        const int t = p.by_pairs.div(i), pair = i - t * p.pairs;
        const double half_turns = (double)p.positions[t0 + t] * p.freqs[pair] * 0.31830988618379067154;
        const float r = (float)(half_turns - 2.0 * rint(0.5 * half_turns));          // [-1, 1]
        float s, c;
        sincospif(r, &s, &c);
        turn[t * 64 + pair] = make_float2(c * p.magnitude, s * p.magnitude * p.sign);
    }
    if constexpr (TO != RotaryTo::kRows)
        if (threadIdx.x < tokens) slot_of[threadIdx.x] = p.slots[t0 + threadIdx.x];
    __syncthreads();

    const int pieces = 1 << p.pieces_shift, turning = p.pairs / VEC;
    const int items = tokens * p.heads_per_wg << p.pieces_shift;
    for (int i = threadIdx.x; i < items; i += kRotaryThreads) {
        const int piece = i & (pieces - 1), rest = i >> p.pieces_shift;
        const int t = p.by_heads_per_wg.div(rest), in_wg = rest - t * p.heads_per_wg;
        if (in_wg >= heads) continue;
        const int head = h0 + in_wg;
        const bool is_q = head < p.q_heads, is_v = head >= p.q_heads + p.kv_heads;
        const int g = is_q ? head : is_v ? head - p.q_heads - p.kv_heads : head - p.q_heads;
        int64_t slot = 0;
        if constexpr (TO != RotaryTo::kRows) {
            slot = slot_of[t];
            if (!is_q && slot < 0) continue;                     // padding token: its rows need not exist
        }
        // The piece's dims: VEC from d0 on and VEC from d1 on, half of the dims that turn (or pass through) apart, so that neighbouring
        // threads' 16 bytes are neighbours; of interleaved pairs each half has four.  (Both halves of a thread side by side: half of
        // every line to an instruction, 4 099 tokens, 40 / 8 heads of 128 26.2 us.)
        const bool turns = !is_v && piece < turning;
        const bool pair = INTERLEAVED && VEC == 1 && turns;
        const int rest0 = is_v ? 0 : 2 * p.pairs;                // the first dim that passes through
        const int d0 = turns ? (pair ? 2 : VEC) * piece : rest0 + VEC * (is_v ? piece : piece - turning);
        const int d1 = d0 + (pair ? 1 : turns ? p.pairs : (p.head_dim - rest0) / 2);
        const uint16_t* src = static_cast<const uint16_t*>(is_q ? p.q : is_v ? p.v : p.k) +
            (t0 + t) * (is_q ? p.q_stride : is_v ? p.v_stride : p.k_stride) + (int64_t)g * p.head_dim;
        uint32_t raw[VEC];                                       // VEC 8: two pieces of four dwords; 1: two elements in a dword
        if constexpr (VEC == 8) {
            const u32x4 a = *reinterpret_cast<const u32x4*>(src + d0), b = *reinterpret_cast<const u32x4*>(src + d1);
#pragma unroll
            for (int j = 0; j < 4; ++j) raw[j] = a[j], raw[4 + j] = b[j];
        } else {
            raw[0] = (uint32_t)src[d0] | (uint32_t)src[d1] << 16;
        }
        // x[], y[]: the values of dims d0 .. and d1 ..
        float x[VEC], y[VEC];
        if constexpr (VEC == 8) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[2 * j] = widen_lo<DT>(raw[j]), x[2 * j + 1] = widen_hi<DT>(raw[j]);
                y[2 * j] = widen_lo<DT>(raw[4 + j]), y[2 * j + 1] = widen_hi<DT>(raw[4 + j]);
            }
        } else {
            x[0] = widen_lo<DT>(raw[0]), y[0] = widen_hi<DT>(raw[0]);
        }
        if (turns) {
            const float2* const cs = &turn[t * 64];
            if constexpr (INTERLEAVED && VEC == 8) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    turn_pair(x[2 * j], x[2 * j + 1], cs[(d0 >> 1) + j]);
                    turn_pair(y[2 * j], y[2 * j + 1], cs[(d1 >> 1) + j]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < VEC; ++j) turn_pair(x[j], y[j], cs[VEC * piece + j]);
            }
        }
        if (TO == RotaryTo::kCacheE4M3 && !is_q) {
            // one rounding, of the turned value times the inverse scale; V by the same formula
            const float inv = p.k_scales ? 1.0f / (is_v ? p.v_scales : p.k_scales)[g] : is_v ? p.v_inv_scale : p.k_inv_scale;
            const int64_t row = (((slot >> p.block_shift) * p.kv_heads + g) << p.block_shift) + (slot & ((1 << p.block_shift) - 1));
            unsigned char* dst = static_cast<unsigned char*>(is_v ? p.v_cache : p.k_cache) + row * p.head_dim;
            if constexpr (VEC == 8) {
                uint32_t c[4] = {0u, 0u, 0u, 0u};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    c[j >> 1] |= e4m3_codes2(x[2 * j] * inv, x[2 * j + 1] * inv) << (16 * (j & 1));
                    c[2 + (j >> 1)] |= e4m3_codes2(y[2 * j] * inv, y[2 * j + 1] * inv) << (16 * (j & 1));
                }
                *reinterpret_cast<uint2*>(dst + d0) = make_uint2(c[0], c[1]);
                *reinterpret_cast<uint2*>(dst + d1) = make_uint2(c[2], c[3]);
            } else {
                const uint32_t two = e4m3_codes2(x[0] * inv, y[0] * inv);
                dst[d0] = (unsigned char)two;
                dst[d1] = (unsigned char)(two >> 8);
            }
            continue;
        }
        uint16_t* dst;
        if (is_q) {
            dst = static_cast<uint16_t*>(p.q_out) + (t0 + t) * p.q_out_stride + (int64_t)g * p.head_dim;
        } else if constexpr (TO == RotaryTo::kRows) {
            dst = static_cast<uint16_t*>(p.k_out) + (t0 + t) * p.k_out_stride + (int64_t)g * p.head_dim;
        } else {
            const int64_t row = (((slot >> p.block_shift) * p.kv_heads + g) << p.block_shift) + (slot & ((1 << p.block_shift) - 1));
            dst = static_cast<uint16_t*>(is_v ? p.v_cache : p.k_cache) + row * p.head_dim;
        }
        // (what passes through leaves as the bits that came: a NaN's payload too)
        if constexpr (VEC == 8) {
            u32x4 a, b;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                a[j] = turns ? narrow2<DT>(x[2 * j], x[2 * j + 1]) : raw[j];
                b[j] = turns ? narrow2<DT>(y[2 * j], y[2 * j + 1]) : raw[4 + j];
            }
            *reinterpret_cast<u32x4*>(dst + d0) = a;
            *reinterpret_cast<u32x4*>(dst + d1) = b;
        } else {
            const uint32_t two = turns ? narrow2<DT>(x[0], y[0]) : raw[0];
            dst[d0] = (uint16_t)two;
            dst[d1] = (uint16_t)(two >> 16);
        }
    }
}

}  // namespace optgqa
