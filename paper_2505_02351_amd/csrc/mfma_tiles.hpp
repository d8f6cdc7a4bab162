// Tiles of 32 rows of keys or values in LDS, as v_mfma_f32_32x32x16 reads them, and the loads that bring them there: what the
// kernels with 32 query rows to a wave share (prefill_kernels.hpp, common_prefix_kernels.hpp).
#pragma once
#include "common.hpp"

namespace optgqa {

constexpr int kPfKeys = 32;                              // keys per tile
// LDS rows of 8-bit caches' tiles and of a wave's strip, elements: K rows padded by 8 (16-byte reads of 16 keys then
// cover all 64 banks), V rows by 16 (so do the rows a transposing load touches) - head_dim 128: 272 / 288 bytes, 64: 144 / 160
template <int D> struct PfTile {
    static constexpr int kKRow = D + 8, kVRow = D + 16;
    static constexpr int kLdsBytes = 2 * kPfKeys * (kKRow + kVRow) * 2;   // two buffers of one K and one V tile (PfDirect's are smaller)
    static constexpr int kWaveBytes = 32 * kKRow * 2;                     // a wave's 32 query (output) rows, pitched as K rows
    // a workgroup of `waves` waves in `groups` key groups
    static constexpr int lds_bytes(int waves, int groups) { return groups * kLdsBytes + waves * kWaveBytes; }
};

// Tiles of 2-byte elements are written to LDS by the memory system itself (global_load_lds_dwordx4: 64 lanes' 16-byte
// pieces to 1 KiB from the address in m0 on, lane by lane): no registers hold a tile on its way, no LDS stores, and with
// wave-uniform addresses not one vector instruction.  (Through registers - loads, 16-byte LDS stores and their addresses -
// a tile cost a wave 20 to 30 instructions.  32 / 8 heads, head_dim 128, the same caches again and again: 8 prompts of 1 024 96.8 -> 86.0 us,
// 8 chunks of 512 behind 2 048 107.5 -> 103.3, without slopes 201 -> 195, with a window of 512 65.7 -> 61.8; whole steps over caches in turn, with 128 rows
// in more launches: those chunks 113.1 -> 110.0, with the window 71.3 -> 68.7, 8 prompts of 2 560 366.7 -> 352.0.  Few rows behind long contexts lost: prefill_deep.)
// Such a load cannot pad rows, but it may bring any piece to any lane.  A tile is groups of 4 rows (head_dim 64: 8), 1 KiB and
// a pad of 16 (32) bytes each.  In a group pieces of 64 bytes - four lanes, 64 bytes of one row's, as the memory system likes
// them - lie row behind row, then the next 64 bytes of all rows:
//     offset = (column / 4) * (64 * rows) + row * 64 + (column % 4) * 16      (columns of 16 bytes; head_dim 64: column ^ 1 in rows 4-7)
// What the score MFMAs read at once (one column of 16 rows) then lies in 16 different sixteenths of the 64 banks, and so do
// the 32-byte pieces of four rows of a transposing load; and a lane's pieces are at constant distances.
template <int D> struct PfDirect {
    static constexpr int kRows = 512 / D, kGroups = 32 / kRows;           // rows of a group; groups of a tile
    static constexpr int kGroup = 1024 + (D == 128 ? 16 : 32);            // bytes from group to group
    static constexpr int kTile = kGroups * kGroup;                        // bytes of a tile (of 32 query rows, too)
    // the row of its group and the column that lane l of a load brings
    static __device__ __forceinline__ int load_row(int l) { return (l >> 2) & (kRows - 1); }
    static __device__ __forceinline__ int load_col(int l)
    {
        return D == 128 ? (l >> 4) * 4 + (l & 3) : (l >> 5) * 4 + ((l & 3) ^ ((l >> 4) & 1));
    }
    // byte offset of dims 8 * h2 .. +7 of a row, and from there to the dims 16m further on
    static __device__ __forceinline__ int row_at(int row, int h2)
    {
        return D == 128 ? (row >> 2) * kGroup + (row & 3) * 64 + h2 * 16
                        : (row >> 3) * kGroup + (row & 7) * 64 + (h2 ^ ((row >> 2) & 1)) * 16;
    }
    static constexpr int dims_at(int m) { return (m >> 1) * 64 * kRows + (m & 1) * 32; }
    // byte offset of what lane s16 of 16 addresses in a transposing load of keys 4 * h2 .. +3, dims 16 * dhalf .. +15, and
    // from there to the keys 8 * k8 and the dims 32 * db further on
    static __device__ __forceinline__ int keys_at(int s16, int dhalf, int h2)
    {
        return D == 128 ? h2 * kGroup + (s16 >> 2) * 64 + dhalf * 32 + (s16 & 3) * 8
                        : (4 * h2 + (s16 >> 2)) * 64 + dhalf * 32 + (((s16 & 3) >> 1) ^ h2) * 16 + (s16 & 1) * 8;
    }
    static constexpr int further(int k8, int db) { return k8 * (8 / kRows) * kGroup + db * 64 * kRows; }

    // DEEP: a key group's LDS holds kDeepBuffers buffers of a K and a V tile each.  The waves' query rows lie behind K and V of the first
    // tile and K of the second, where nothing is loaded before they have been read; the output rows, after the walk, from the
    // beginning on (two groups: behind what they exchange).
    static constexpr int kDeepBuffers = 4, kRowsAt = 3 * kTile;
    static constexpr int group_bytes(int group_waves)
    {
        const int tiles = 2 * kDeepBuffers * kTile, rows = kRowsAt + group_waves * PfTile<D>::kWaveBytes;
        return tiles > rows ? tiles : rows;
    }
    static constexpr int exchange_bytes(int waves, int groups) { return groups == 1 ? 0 : waves * 64 * (D / 64 * 4 * 16 + 8); }
    static constexpr int deep_lds_bytes(int waves, int groups)
    {
        const int walk = groups * group_bytes(waves / groups), out = exchange_bytes(waves, groups) + waves * PfTile<D>::kWaveBytes;
        return walk > out ? walk : out;
    }
};

// One such load, to LDS address `lds` (wave-uniform) on; from a wave-uniform base and lane offsets, or from lane addresses.
// In assembly because the compiler, which does not know which buffer a load writes, would have every later read of LDS wait
// for it; wait_direct() comes before the barrier that publishes the tile.  (m0 is an operand, which the compiler sets: it is a
// reserved register, and a statement that writes it by itself is not one that the compiler allows for.  The s_nop is the wait
// state between that and the load.)
__device__ __forceinline__ void load_direct(uint32_t lds, const unsigned char* base, uint32_t lane_off)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "{m0}"(lds), "v"(lane_off), "s"(base) : "memory");
}
__device__ __forceinline__ void load_direct(uint32_t lds, const unsigned char* lane_addr)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "{m0}"(lds), "v"(lane_addr) : "memory");
}
// (non-temporal: what is read once, see stream_load16)
__device__ __forceinline__ void stream_direct(uint32_t lds, const unsigned char* base, uint32_t lane_off)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" :: "{m0}"(lds), "v"(lane_off), "s"(base) : "memory");
}
template <int NEWER = 0> __device__ __forceinline__ void wait_direct() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(NEWER) : "memory"); }

template <int DT> __device__ __forceinline__ uint32_t pack2(float lo, float hi) { return narrow2<DT>(lo, hi); }

typedef float f32x16 __attribute__((ext_vector_type(16)));
// v_mfma_f32_32x32x16: A lane (row L % 32, k-slab L / 32) holds k = 8 * slab .. + 7, B likewise
// for its column; C / D lane (column L % 32, half L / 32) holds rows 8i + 4 * half + j in
// element 4i + j (i, j = 0..3).
template <int DT> __device__ __forceinline__ f32x16 mfma32(uint4 a, uint4 b, f32x16 c);
template <> __device__ __forceinline__ f32x16 mfma32<kF16>(uint4 a, uint4 b, f32x16 c)
{
    typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x16 mfma32<kBF16>(uint4 a, uint4 b, f32x16 c)
{
    typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// what this wave wrote to LDS is there for its other lanes (LDS instructions of a wave complete in order; the compiler
// keeps theirs across this)
__device__ __forceinline__ void wave_lds_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <int DT> struct PfSoftmax;
template <> struct PfSoftmax<kF16> {
    static constexpr float kThreshold = 14.f, kHeadroom = 2.f;
    static constexpr bool kSplitWeights = false;
};
template <> struct PfSoftmax<kBF16> {
    static constexpr float kThreshold = kRescaleThreshold, kHeadroom = kRescaleHeadroom;
    static constexpr bool kSplitWeights = true;
};

}  // namespace optgqa
