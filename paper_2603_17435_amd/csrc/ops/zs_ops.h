// What the kernels of the 8-bit products and of the embedding operators share: unaligned vector
// access, BF16 conversion, and the host's argument helpers.
#ifndef ZS_OPS_H
#define ZS_OPS_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

#include "zipserv.h"

namespace zs_ops {

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(8))) int32_t i32x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

// Vectors at any element's address: rows of odd length or stride start where no vector is aligned.
// The hardware takes such an address for a global access of any width.
template <typename V, typename T>
__device__ __forceinline__ V load_any(const T *p)
{
    V v;
    __builtin_memcpy(&v, p, sizeof v);
    return v;
}
template <typename V, typename T>
__device__ __forceinline__ void store_any(T *p, V v)
{
    __builtin_memcpy(p, &v, sizeof v);
}

__device__ __forceinline__ float bf16_value(uint32_t bits) { return __builtin_bit_cast(float, bits << 16); }

// Nearest BF16 number, ties to even; NaN stays NaN.
__device__ __forceinline__ uint16_t bf16_bits(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi)
{
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)lo, (__bf16)hi});
}

// N consecutive values of a row of BF16 patterns or floats as they lie there; those at and behind `left` are zero.
template <typename T, int N>
struct Values {
    uint32_t w[N * sizeof(T) / 4];
    __device__ __forceinline__ float operator[](int i) const // i is a constant
    {
        const uint32_t v = w[i * (int)sizeof(T) / 4];
        return __builtin_bit_cast(float, sizeof(T) == 4 ? v : i % 2 ? v & 0xFFFF0000u : v << 16);
    }
};
template <int N, typename T>
__device__ __forceinline__ Values<T, N> fetch(const T *p, int64_t left)
{
    if (left >= N) return load_any<Values<T, N>>(p);
    Values<T, N> v = {};
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < left) {
            if constexpr (sizeof(T) == 2) v.w[i / 2] |= (uint32_t)p[i] << (16 * (i % 2));
            else v.w[i] = __builtin_bit_cast(uint32_t, p[i]);
        }
    return v;
}

inline bool aligned(const void *p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
inline int launched() { return hipGetLastError() == hipSuccess ? ZS_OK : ZS_ERR_HIP; }
// Lets a kernel use up to `bytes` of dynamic LDS on the current device.  The attribute stays with (kernel, device):
// `done` has a bit for each device that it was set on.
template <auto Kernel>
inline int allow_lds(size_t bytes)
{
    static std::atomic<uint64_t> done{0};
    int device = 0;
    if (hipGetDevice(&device) != hipSuccess || device < 0 || device >= 64) return ZS_ERR_HIP;
    if (done.load(std::memory_order_acquire) >> device & 1u) return ZS_OK;
    if (hipFuncSetAttribute(reinterpret_cast<const void *>(Kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != hipSuccess)
        return ZS_ERR_HIP;
    done.fetch_or(1ull << device, std::memory_order_release);
    return ZS_OK;
}
// A launch counts its threads along x in 32 bits: kernels whose work could exceed that stride over it.
inline unsigned grid_for(int64_t wgs, int64_t most = 1 << 20) { return (unsigned)(wgs < most ? wgs : most); }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

} // namespace zs_ops
#endif
