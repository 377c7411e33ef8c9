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

// Eight consecutive values of a row of BF16 patterns or floats as they lie there; those at and behind `left` are zero.
template <typename T>
struct Eight {
    u32x4 w[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ Eight<T> fetch8(const T *p, int64_t left)
{
    if (left >= 8) return load_any<Eight<T>>(p);
    Eight<T> e = {};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) {
            if constexpr (sizeof(T) == 2) e.w[0][i / 2] |= (uint32_t)p[i] << (16 * (i % 2));
            else e.w[i / 4][i % 4] = __builtin_bit_cast(uint32_t, p[i]);
        }
    return e;
}
template <typename T>
__device__ __forceinline__ float value8(const Eight<T> &e, int i) // i is a constant
{
    const uint32_t w = sizeof(T) == 2 ? e.w[0][i / 2] : e.w[(i / 4) % (sizeof(T) / 2)][i % 4];
    return __builtin_bit_cast(float, sizeof(T) == 4 ? w : i % 2 ? w & 0xFFFF0000u : w << 16);
}
template <typename T>
__device__ __forceinline__ void load8(const T *p, int64_t left, float v[8])
{
    const Eight<T> e = fetch8(p, left);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = value8(e, i);
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
