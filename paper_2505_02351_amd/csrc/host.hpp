// What the library's host sources share: argument checks, launches, facts about the device.
#pragma once
#include <hip/hip_runtime.h>

#include <cmath>
#include <tuple>
#include <utility>

#include "common.hpp"
#include "optgqa.h"

namespace optgqa {

inline bool dtype_ok(int dt) { return dt == OPTGQA_F16 || dt == OPTGQA_BF16; }
inline bool head_dim_ok(int d) { return d == 64 || d == 128; }
inline bool block_size_ok(int bs) { return bs == 16 || bs == 32 || bs == 64; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Workgroups of so many threads that one dimension of a launch may have: fewer than 2^32 threads.
constexpr int64_t most_workgroups(int threads) { return 0xffffffffLL / threads; }

// Launch through the call that reports THIS launch's own status (hipLaunchKernel): an error
// some earlier work of the caller left behind in the runtime's "last error" slot is neither
// reported as ours nor cleared.
template <typename... KArgs, typename... Args>
int launch(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t lds_bytes, hipStream_t st, Args&&... args)
{
    static_assert(sizeof...(KArgs) == sizeof...(Args), "argument count does not match the kernel");
    // (the runtime takes a dimension of 2^32 threads and more without a word, and runs what is left of it modulo 2^32)
    if ((uint64_t)grid.x * block.x >> 32 || (uint64_t)grid.y * block.y >> 32 || (uint64_t)grid.z * block.z >> 32) return OPTGQA_ERR_LAUNCH;
    std::tuple<std::decay_t<KArgs>...> vals(std::forward<Args>(args)...);
    void* ptrs[sizeof...(KArgs)];
    std::apply([&](auto&... v) { int i = 0; ((ptrs[i++] = static_cast<void*>(&v)), ...); }, vals);
    return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, ptrs, lds_bytes, st) == hipSuccess
               ? OPTGQA_OK : OPTGQA_ERR_LAUNCH;
}

// Compute units of the current device, asked once (every GPU of a box is the same part); 256,
// the MI355X count, where no device answers (the sizing calls also work on a GPU-less host).
inline int num_cus()
{
    static const int cus = [] {
        int dev = 0, n = 0;
        if (hipGetDevice(&dev) != hipSuccess ||
            hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0)
            return 256;
        return n;
    }();
    return cus;
}

// Scales of 8-bit (E4M3) caches: one pair per tensor (k, v), or - k_heads / v_heads set, device
// arrays of num_kv_heads values each - one pair per KV head.
struct KvScales {
    float k, v;
    const float* k_heads;
    const float* v_heads;
    bool per_head() const { return k_heads != nullptr; }
    bool valid() const
    {
        if (per_head()) return v_heads != nullptr;           // contents live on the device: not checked here
        return k > 0.f && v > 0.f && k <= 3e38f && v <= 3e38f;
    }
};

// The tiled prefill kernel carries the tile-invariant part of the ALiBi term inside the score
// accumulator as slope / scale, so it cannot take a score scale of exactly zero.  Magnitudes
// below 2^-64 (zero included) are evaluated as +-2^-64: the scores then differ from the exact
// ones by |q.k| * 2^-64, far below fp32 resolution of the bias they are added to.
inline float prefill_scale2(float scale)
{
    const float tiny = 0x1p-64f;
    const float s = std::fabs(scale) < tiny ? std::copysign(tiny, scale) : scale;
    return s * kLog2e;
}

}  // namespace optgqa
