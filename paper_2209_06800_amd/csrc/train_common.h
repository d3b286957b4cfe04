// Loads, stores and reductions shared by the kernels for training (lookup.hip, grouped.hip, distill.hip).
#pragma once

#include <hip/hip_runtime.h>

#include "mgg_internal.h"

namespace mgg {
namespace train {

constexpr int kWave = 64;

// bf16 values as raw bits: a type of its own, so that templates tell them from 16-bit integers
struct Bf16 { uint16_t bits; };

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(Bf16 x) { return __uint_as_float(static_cast<uint32_t>(x.bits) << 16); }

// two values to bf16, nearest even, in one instruction
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const f32x2 f = {lo, hi};
    union { bf16x2 b; uint32_t u; } r;
    r.b = __builtin_convertvector(f, bf16x2);
    return r.u;
}
__device__ __forceinline__ void from_f32(float f, float &out) { out = f; }
__device__ __forceinline__ void from_f32(float f, Bf16 &out) { out.bits = static_cast<uint16_t>(pack_bf16(f, 0.f)); }

// N consecutive elements at any element boundary (the hardware takes 16 bytes at any address; where the address is a
// multiple of 16 it is one request)
template <int N>
__device__ __forceinline__ void load_n(const float *p, float (&v)[N]) { __builtin_memcpy(v, __builtin_assume_aligned(p, 4), sizeof v); }
template <int N>
__device__ __forceinline__ void load_n(const Bf16 *p, float (&v)[N])
{
    if constexpr (N == 1) {
        v[0] = to_f32(*p);
    } else {
        uint32_t u[N / 2];
        __builtin_memcpy(u, __builtin_assume_aligned(p, 2), sizeof u);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            v[2 * i] = __uint_as_float(u[i] << 16);
            v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
}
template <int N>
__device__ __forceinline__ void store_n(float *p, const float (&v)[N]) { __builtin_memcpy(__builtin_assume_aligned(p, 4), v, sizeof v); }
template <int N>
__device__ __forceinline__ void store_n(Bf16 *p, const float (&v)[N])
{
    if constexpr (N == 1) {
        from_f32(v[0], *p);
    } else {
        uint32_t u[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) u[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
        __builtin_memcpy(__builtin_assume_aligned(p, 2), u, sizeof u);
    }
}

inline int ceil_log2(int64_t v)
{
    int b = 0;
    while ((static_cast<int64_t>(1) << b) < v) ++b;
    return b;
}
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
// a launch has fewer than 2^31 blocks and 2^32 threads along its first axis
inline bool launchable(int64_t blocks, int threads) { return blocks <= INT32_MAX && blocks * threads <= static_cast<int64_t>(UINT32_MAX); }
inline size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

}  // namespace train
}  // namespace mgg
