// zs_fp8_quantize: BF16 or FP32 values to OCP E4M3 codes with one power-of-two scale for each block of
// 1 x 128 or 128 x 128 along the rows of the result, which is the matrix itself or its transpose.
//
// For the largest finite magnitude a of a block the scale is the smallest 2^e >= 2^-126 with
// a <= 448 * 2^e (1 where a = 0).  A division by a power of two is exact, so a code is the E4M3 number
// nearest to x / scale after a single rounding, whoever computes it.  448 = 1.75 * 2^8: e follows from the bits of a.
#include "zs_ops.h"

using namespace zs_ops;

namespace {

constexpr int kBlock = 128;

__device__ __forceinline__ uint32_t finite_magnitude(float x)
{
    const uint32_t a = __builtin_bit_cast(uint32_t, x) & 0x7FFFFFFFu;
    return a < 0x7F800000u ? a : 0u;
}

// Bits of the scale 2^e and of 2^-e for a block whose largest finite magnitude has the bits a.
__device__ __forceinline__ uint32_t scale_bits(uint32_t a)
{
    const int e = (int)(a >> 23) - 8 + ((a & 0x7FFFFFu) > 0x600000u ? 1 : 0); // e + 127
    return a == 0 ? 127u << 23 : (uint32_t)(e < 1 ? 1 : e) << 23;
}
__device__ __forceinline__ float inverse_of(uint32_t scale) { return __builtin_bit_cast(float, (254u << 23) - scale); }

// The codes of four values, lowest byte first (nearest, ties to even; Inf and NaN give NaN).
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

__device__ __forceinline__ uint32_t max_over(uint32_t a, int lanes) // of `lanes` neighbouring lanes
{
    for (int d = 1; d < lanes; d *= 2) a = max(a, (uint32_t)__shfl_xor((int)a, d));
    return a;
}

// Blocks of 1 x 128, not transposed: sixteen lanes to a block, eight values to a lane.  Bound by memory, or a launch: 200 x 14336
// BF16 values take 4 us, 4096 x 14336 41 us (4.3 TB/s), FP32 values 54 us (5.4).
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T *X, int64_t R, int64_t C, int64_t ldx, uint8_t *Q, int64_t ldq,
                                                            float *S, int64_t lds, int64_t k_blocks)
{
    const int64_t blocks = R * k_blocks, step = (int64_t)gridDim.x * 16;
    for (int64_t b = (int64_t)blockIdx.x * 16 + threadIdx.x / 16; b < blocks; b += step) {
        const int64_t r = b / k_blocks, kb = b - r * k_blocks, c = kb * kBlock + 8 * (threadIdx.x % 16);
        const Values<T, 8> v = fetch<8>(X + r * ldx + c, C - c);
        uint32_t a = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) a = max(a, finite_magnitude(v[i]));
        const uint32_t s = scale_bits(max_over(a, 16));
        const float inv = inverse_of(s);
        if (c < (C + 15) / 16 * 16)
            *reinterpret_cast<u32x2 *>(Q + r * ldq + c) = u32x2{codes4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv),
                                                                codes4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv)};
        if (threadIdx.x % 16 == 0) S[kb * lds + r] = __builtin_bit_cast(float, s);
    }
}

// Tiles of 128 x 128 of X, a workgroup each: a thread holds eight rows of eight columns.  ROWS: 1 or 128, the
// height of a block of the result.  With TRANSPOSE the codes of a column's eight rows are packed together and go
// through LDS, from where they leave as rows of the result (chunks of 16 bytes by column: without bank conflicts; rows padded by 16
// bytes had eightfold ones, 26 instead of 20 us).  Bound by memory: BF16 2051 x 14336 transposed 20 us, 28672 x 4096 in square blocks 66 us
// (5.3 TB/s), transposed 70.
template <typename T, int ROWS, bool TRANSPOSE>
__global__ __launch_bounds__(256) void quantize_tiles_kernel(const T *X, int64_t R, int64_t C, int64_t ldx, uint8_t *Q, int64_t ldq,
                                                             float *S, int64_t lds, int64_t c_tiles, int64_t tiles)
{
    __shared__ uint32_t peak[4][kBlock]; // by wave: of each column, or [0] of everything
    __shared__ __attribute__((aligned(16))) uint8_t turned[TRANSPOSE ? kBlock * kBlock : 16]; // chunk c of column j at c ^ (j / 8 % 8)
    const int tid = threadIdx.x, wave = tid / 64, cg = tid % 16, rg = tid / 16;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t rt = tile / c_tiles, ct = tile - rt * c_tiles;
        const int64_t r0 = rt * kBlock + 8 * rg, c0 = ct * kBlock + 8 * cg;
        Values<T, 8> raw[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) raw[i] = r0 + i < R ? fetch<8>(X + (r0 + i) * ldx + c0, C - c0) : Values<T, 8>{};
        auto value = [&](int i, int j) { return raw[i][j]; };
        uint32_t a[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            a[j] = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) a[j] = max(a[j], finite_magnitude(value(i, j)));
        }
        float inv[8];
        if constexpr (ROWS == kBlock) {
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) m = max(m, a[j]);
            m = max_over(m, 64);
            if (tid % 64 == 0) peak[wave][0] = m;
            __syncthreads();
            const uint32_t s = scale_bits(max(max(peak[0][0], peak[1][0]), max(peak[2][0], peak[3][0])));
#pragma unroll
            for (int j = 0; j < 8; ++j) inv[j] = inverse_of(s);
            if (tid == 0) S[TRANSPOSE ? rt * lds + ct : ct * lds + rt] = __builtin_bit_cast(float, s);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                a[j] = max(a[j], (uint32_t)__shfl_xor((int)a[j], 16));
                a[j] = max(a[j], (uint32_t)__shfl_xor((int)a[j], 32));
                if (tid % 64 < 16) peak[wave][8 * cg + j] = a[j];
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = 8 * cg + j;
                const uint32_t s = scale_bits(max(max(peak[0][c], peak[1][c]), max(peak[2][c], peak[3][c])));
                inv[j] = inverse_of(s);
                if (rg == 0 && c0 + j < C) S[rt * lds + c0 + j] = __builtin_bit_cast(float, s);
            }
        }
        if constexpr (TRANSPOSE) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                auto q = [&](int i) { return codes4(value(i, j) * inv[j], value(i + 1, j) * inv[j], value(i + 2, j) * inv[j], value(i + 3, j) * inv[j]); };
                *reinterpret_cast<u32x2 *>(turned + (8 * cg + j) * kBlock + 16 * ((rg / 2) ^ (cg % 8)) + 8 * (rg % 2)) = u32x2{q(0), q(4)};
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = 32 * i + tid / 8, at = 16 * (tid % 8);
                if (ct * kBlock + c < C && rt * kBlock + at < R)
                    *reinterpret_cast<u32x4 *>(Q + (ct * kBlock + c) * ldq + rt * kBlock + at) =
                        *reinterpret_cast<const u32x4 *>(turned + c * kBlock + 16 * ((tid % 8) ^ (c / 8 % 8)));
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                auto q = [&](int j) { return codes4(value(i, j) * inv[j], value(i, j + 1) * inv[j + 1], value(i, j + 2) * inv[j + 2], value(i, j + 3) * inv[j + 3]); };
                if (r0 + i < R && c0 < (C + 15) / 16 * 16) *reinterpret_cast<u32x2 *>(Q + (r0 + i) * ldq + c0) = u32x2{q(0), q(4)};
            }
        }
        __syncthreads(); // peak and turned are written again
    }
}

template <typename T>
int launch(const T *X, int64_t R, int64_t C, int64_t ldx, int block_rows, int transpose, uint8_t *Q, int64_t ldq, float *S, int64_t lds,
           hipStream_t s)
{
    const int64_t r_tiles = ceil_div(R, kBlock), c_tiles = ceil_div(C, kBlock);
    if (block_rows == 1 && !transpose) {
        hipLaunchKernelGGL(quantize_rows_kernel<T>, dim3(grid_for(ceil_div(R * c_tiles, 16))), dim3(256), 0, s, X, R, C, ldx, Q, ldq, S, lds,
                           c_tiles);
        return launched();
    }
    const dim3 grid(grid_for(r_tiles * c_tiles)), wg(256);
    if (block_rows == 1)
        hipLaunchKernelGGL((quantize_tiles_kernel<T, 1, true>), grid, wg, 0, s, X, R, C, ldx, Q, ldq, S, lds, c_tiles, r_tiles * c_tiles);
    else if (transpose)
        hipLaunchKernelGGL((quantize_tiles_kernel<T, kBlock, true>), grid, wg, 0, s, X, R, C, ldx, Q, ldq, S, lds, c_tiles, r_tiles * c_tiles);
    else
        hipLaunchKernelGGL((quantize_tiles_kernel<T, kBlock, false>), grid, wg, 0, s, X, R, C, ldx, Q, ldq, S, lds, c_tiles, r_tiles * c_tiles);
    return launched();
}

} // namespace

extern "C" int zs_fp8_quantize(const void *X_dev, int x_type, int64_t R, int64_t C, int64_t ldx, int block_rows, int transpose,
                               uint8_t *Q_dev, int64_t ldq, float *S_dev, int64_t lds, void *hip_stream)
{
    if (!X_dev || !Q_dev || !S_dev) return ZS_ERR_ARG;
    if (x_type != ZS_TYPE_BF16 && x_type != ZS_TYPE_F32) return ZS_ERR_CONFIG;
    if (block_rows != 1 && block_rows != kBlock) return ZS_ERR_CONFIG;
    if (!aligned(X_dev, x_type == ZS_TYPE_BF16 ? 2 : 4) || !aligned(Q_dev, 16) || !aligned(S_dev, 4)) return ZS_ERR_ARG;
    if (R < 1 || C < 1 || R > INT32_MAX || C > INT32_MAX || ldx < C) return ZS_ERR_SHAPE;
    const int64_t rows = transpose ? C : R, cols = transpose ? R : C;
    if (ldq < cols || ldq % 16 || lds < ceil_div(rows, block_rows)) return ZS_ERR_SHAPE;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (x_type == ZS_TYPE_BF16) return launch(static_cast<const uint16_t *>(X_dev), R, C, ldx, block_rows, transpose, Q_dev, ldq, S_dev, lds, s);
    return launch(static_cast<const float *>(X_dev), R, C, ldx, block_rows, transpose, Q_dev, ldq, S_dev, lds, s);
}
