// Element types and small device helpers of the policy operators (linear recurrence, log probabilities, orthogonalised
// update): arrays are fp32, bf16 or fp16, arithmetic is fp32.
#pragma once
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qnet_internal.h"

namespace marl {

constexpr int kWave = 64;

template <typename T>
__device__ __forceinline__ float to_f32(T v) { return (float)v; }

// Rounds to nearest even; fp32 stays as it is.
template <typename T>
__device__ __forceinline__ T from_f32(float v) { return (T)v; }

__host__ __device__ __forceinline__ int element_bytes(int dtype) { return dtype == MARL_DTYPE_F32 ? 4 : 2; }

inline bool known_dtype(int dtype) { return dtype == MARL_DTYPE_F32 || dtype == MARL_DTYPE_BF16 || dtype == MARL_DTYPE_F16; }

// A launch has fewer than 2^32 threads.
inline bool fits_a_launch(int64_t groups, int threads) { return groups * threads < (int64_t)1 << 32; }

inline bool aligned_to(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Calls f with a value of the element type of `dtype`.
template <typename F>
inline int with_dtype(int dtype, F &&f)
{
    switch (dtype) {
    case MARL_DTYPE_F32: return f(float{});
    case MARL_DTYPE_BF16: return f(__bf16{});
    default: return f(_Float16{});
    }
}

// What a launch left behind, as a status of the C ABI.
inline int launched(const char *what)
{
    const hipError_t err = hipGetLastError();
    return err == hipSuccess ? MARL_OK : report_device_error(err, what);
}

}  // namespace marl
