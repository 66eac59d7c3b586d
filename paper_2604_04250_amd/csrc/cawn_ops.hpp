// What the operators beside the scan share (gfx950 only): element types, loads and stores that widen and round, host checks.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cawn.h"

namespace cawn {
namespace ops {

using bf16 = __bf16;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <typename T, int N> struct alignas(sizeof(T) * N) Pack { T v[N]; };

// N adjacent elements as fp32, one access; p is aligned to N elements
template <typename T, int N> __device__ inline void load_n(const T *p, float (&x)[N])
{
    const Pack<T, N> a = *reinterpret_cast<const Pack<T, N> *>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (float)a.v[i];
}
// ... and back, rounded to nearest even
template <typename T, int N> __device__ inline void store_n(T *p, const float (&x)[N])
{
    Pack<T, N> a;
#pragma unroll
    for (int i = 0; i < N; ++i) a.v[i] = (T)x[i];
    *reinterpret_cast<Pack<T, N> *>(p) = a;
}

inline bool aligned_to(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
inline int launched() { return hipGetLastError() == hipSuccess ? CAWN_OK : CAWN_ELAUNCH; }
inline long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

} // namespace ops
} // namespace cawn
