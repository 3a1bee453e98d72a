// Shared by the operators of scd_lm.h: real types, 16-byte vectors of them, index arrays, argument checks.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "scd_lm_shape.h"

namespace scd {

int report_hip(hipError_t e);  // keeps the code for scd_last_hip_error; SCD_EHIP

namespace lm {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));

constexpr int kWave = 64;
constexpr int64_t kMaxDim = 0x7FFFFFFF;

inline bool real_ok(int dt) { return dt == SCD_REAL_F32 || dt == SCD_REAL_BF16 || dt == SCD_REAL_F16; }
inline size_t real_bytes(int dt) { return dt == SCD_REAL_F32 ? 4 : 2; }
inline bool index_ok(int bytes) { return bytes == 4 || bytes == 8; }
inline bool dim_ok(int64_t d) { return d >= 1 && d <= kMaxDim; }
inline bool rows_ok(int64_t d) { return d >= 0 && d <= kMaxDim; }
inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
// A launch has fewer than 2^32 threads along x.
inline bool grid_ok(int64_t groups, int64_t threads) { return groups >= 1 && groups <= (int64_t)0xFFFFFFFF / threads; }

// 16 bytes of a real type.
template <typename T>
struct Vec {
    static constexpr int N = 16 / sizeof(T);
    typedef T V __attribute__((ext_vector_type(16 / sizeof(T))));
};

template <typename T>
__device__ __forceinline__ float to_f32(T x)
{
    return (float)x;
}

// The one rounding of a result to its type.  The value is pinned in a 32-bit register first: a product folded into the
// conversion (f16 has such instructions) would round otherwise in one form of a kernel than in another.
template <typename T>
__device__ __forceinline__ T round_to(float x)
{
    if constexpr (sizeof(T) < 4) asm("" : "+v"(x));
    return (T)x;
}

__device__ __forceinline__ int64_t index_at(const void* p, int bytes, int64_t i)
{
    return bytes == 4 ? (int64_t)((const int32_t*)p)[i] : ((const int64_t*)p)[i];
}

// f(T{}) for the type of dt (checked before).
template <typename F>
inline auto with_real(int dt, F&& f)
{
    if (dt == SCD_REAL_F32) return f(float{});
    if (dt == SCD_REAL_BF16) return f(__bf16{});
    return f(_Float16{});
}

}  // namespace lm
}  // namespace scd
