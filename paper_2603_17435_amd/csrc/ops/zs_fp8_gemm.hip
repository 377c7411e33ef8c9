// zs_fp8_gemm: C[m,n] = sum over blocks b of 128 along K of SA[b,m] SW[b,n / w_rows] sum_{k in b} A[m,k] W[n,k]
// on E4M3 codes.  The products of one block of K are summed by the matrix cores; the sum is scaled once and added to an
// FP32 accumulator.
#include "zs_ops.h"

#include <algorithm>
#include <type_traits>

using namespace zs_ops;

namespace {

constexpr int kBlock = 128;
constexpr int64_t kMaxLd = (int64_t)1 << 23;
constexpr int64_t kMaxTiles = (int64_t)1 << 22; // of one launch: its threads are counted in 32 bits

struct Product {
    const uint8_t *A, *W;
    const float *SA, *SW;
    int64_t lda, ldsa, ldw, ldsw, ldc;
    int64_t M, N, K, k_blocks;
    int w_rows;
};

// Eight codes as FP16 numbers, which hold every one of them exactly; v_mfma_f32_16x16x32_f16 then sums whole products in
// FP32.  (The 8-bit matrix instructions cut each product at 2^-13 of the largest of its group of eight.)
__device__ __forceinline__ f16x8 widened(uint32_t lo, uint32_t hi)
{
    const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true);
    const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true);
    return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ void store4(float *p, f32x4 v, int64_t left)
{
    if (left >= 4) {
        *reinterpret_cast<f32x4 *>(p) = v;
        return;
    }
    for (int i = 0; i < 4; ++i)
        if (i < left) p[i] = v[i];
}
__device__ __forceinline__ void store4(uint16_t *p, f32x4 v, int64_t left)
{
    if (left >= 4) {
        *reinterpret_cast<u32x2 *>(p) = u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
        return;
    }
    for (int i = 0; i < 4; ++i)
        if (i < left) p[i] = bf16_bits(v[i]);
}

// ---- few tokens: the weights are read once ----------------------------------------------------
// A workgroup computes 16 RT features x 16 MT tokens; its NW waves take the blocks of K in turn, each with D blocks
// requested ahead, and add their sums up in LDS, always in the same order.  W is the first operand, so a lane
// holds four features of one token.  A lane takes the chunks of 16 bytes `part` and `part` + 4 of its row, so that a
// load covers 64 contiguous bytes of sixteen rows.
template <int MT, int RT, int NW, int D, bool W1, typename OUT>
__global__ __launch_bounds__(64 * NW) void stream_kernel(Product p, OUT *C)
{
    constexpr int kTiles = MT * RT;
    __shared__ f32x4 sums[NW][kTiles][64];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), row = lane % 16, part = lane / 16;
    const int64_t n0 = (int64_t)blockIdx.x * (16 * RT), m0 = (int64_t)blockIdx.y * (16 * MT);
    const int m_last = (int)min(p.M - 1 - m0, (int64_t)16 * MT - 1), n_last = (int)min(p.N - 1 - n0, (int64_t)16 * RT - 1);
    const uint8_t *const a_base = p.A + m0 * p.lda, *const w_base = p.W + n0 * p.ldw;
    const float *const sa_base = p.SA + m0, *const sw_base = p.SW + n0 / p.w_rows;
    uint32_t a_row[MT], w_row[RT];
#pragma unroll
    for (int i = 0; i < MT; ++i) a_row[i] = (uint32_t)min(16 * i + row, m_last);
#pragma unroll
    for (int j = 0; j < RT; ++j) w_row[j] = (uint32_t)min(16 * j + row, n_last) * (uint32_t)p.ldw;

    struct Block {
        u32x4 w[RT][2], a[MT][2];
        float sa[MT];
        f32x4 sw[W1 ? RT : 1];
    };
    auto load = [&](Block &b, int64_t kb) {
        const uint32_t k = (uint32_t)kb * kBlock;
#pragma unroll
        for (int h = 0; h < 2; ++h) { // (chunks behind a row's end repeat its last one)
            const uint32_t w_k = min(k + 16 * part + 64 * h, (uint32_t)p.ldw - 16), a_k = min(k + 16 * part + 64 * h, (uint32_t)p.lda - 16);
#pragma unroll
            for (int j = 0; j < RT; ++j) b.w[j][h] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(w_base + (w_row[j] + w_k)));
#pragma unroll
            for (int i = 0; i < MT; ++i) b.a[i][h] = *reinterpret_cast<const u32x4 *>(a_base + (a_row[i] * (uint32_t)p.lda + a_k));
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) b.sa[i] = sa_base[kb * p.ldsa + a_row[i]];
        if constexpr (W1) {
#pragma unroll
            for (int j = 0; j < RT; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) b.sw[j][e] = sw_base[kb * p.ldsw + min(16 * j + 4 * part + e, n_last)];
        } else {
            b.sw[0][0] = sw_base[kb * p.ldsw];
        }
    };
    f32x4 acc[MT][RT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < RT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](Block &b, int64_t kb) {
        if ((kb + 1) * kBlock > p.K) { // codes behind K
            const int keep = (int)(p.K - kb * kBlock);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int left = keep - (16 * part + 64 * h + 4 * e);
                    const uint32_t mask = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
#pragma unroll
                    for (int j = 0; j < RT; ++j) b.w[j][h][e] &= mask;
#pragma unroll
                    for (int i = 0; i < MT; ++i) b.a[i][h][e] &= mask;
                }
        }
        f16x8 a[MT][4];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) a[i][e] = widened(b.a[i][e / 2][2 * (e % 2)], b.a[i][e / 2][2 * (e % 2) + 1]);
#pragma unroll
        for (int j = 0; j < RT; ++j) {
            f16x8 w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = widened(b.w[j][e / 2][2 * (e % 2)], b.w[j][e / 2][2 * (e % 2) + 1]);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int e = 0; e < 4; ++e) sum = __builtin_amdgcn_mfma_f32_16x16x32_f16(w[e], a[i][e], sum, 0, 0, 0);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = __builtin_fmaf(sum[e], b.sa[i] * (W1 ? b.sw[W1 ? j : 0][e] : b.sw[0][0]), acc[i][j][e]);
            }
        }
    };

    Block b[D];
#pragma unroll
    for (int d = 0; d < D; ++d)
        if (wave + d * NW < p.k_blocks) load(b[d], wave + d * NW);
    for (int64_t kb = wave; kb < p.k_blocks; kb += D * NW)
#pragma unroll
        for (int d = 0; d < D; ++d) {
            const int64_t now = kb + d * NW, next = now + D * NW;
            if (now < p.k_blocks) multiply(b[d], now);
            if (next < p.k_blocks) load(b[d], next);
        }

#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < RT; ++j) sums[wave][i * RT + j][lane] = acc[i][j];
    __syncthreads();
    for (int t = wave; t < kTiles; t += NW) {
        f32x4 sum = sums[0][t][lane];
#pragma unroll
        for (int w = 1; w < NW; ++w) sum += sums[w][t][lane];
        const int64_t m = m0 + 16 * (t / RT) + row, n = n0 + 16 * (t % RT) + 4 * part;
        if (m < p.M && n < p.N) store4(C + m * p.ldc + n, sum, p.N - n);
    }
}

template <int MT, int RT, int NW, int D, typename OUT>
int run_stream(const Product &p, OUT *C, hipStream_t s)
{
    const dim3 grid((unsigned)ceil_div(p.N, 16 * RT), (unsigned)ceil_div(p.M, 16 * MT)), wg(64 * NW);
    if (grid.x > kMaxTiles) return ZS_ERR_SHAPE;
    if (p.w_rows == 1) hipLaunchKernelGGL((stream_kernel<MT, RT, NW, D, true, OUT>), grid, wg, 0, s, p, C);
    else hipLaunchKernelGGL((stream_kernel<MT, RT, NW, D, false, OUT>), grid, wg, 0, s, p, C);
    return launched();
}

// ---- tiles through LDS ---------------------------------------------------------------------
// A workgroup of WM x WN waves computes (16 TM WM) tokens x (16 TN WN) features over the blocks [kb0, kb1) of K.  Each
// block's codes and scales go from memory straight to LDS (two buffers: block b + 1 is under way while b is
// multiplied, one barrier a block).  A row's eight chunks of 16 bytes lie in the order chunk ^ (row % 8), so that
// the sixteen rows of an operand are read without bank conflicts.
constexpr int kRowBytes = 128;

// 64 lanes x 16 (or 4) bytes from base + at to the 1 KB (256 bytes) of LDS at `to`.  Not tracked by the compiler: arrived().
__device__ __forceinline__ void fetch16(const void *base, uint32_t at, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(at), "s"(base), "s"(to) : "memory", "m0");
}
__device__ __forceinline__ void fetch4(const void *base, uint32_t at, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(at), "s"(base), "s"(to) : "memory", "m0");
}
__device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

typedef const __attribute__((address_space(3))) u32x4 *LdsU32x4;
typedef const __attribute__((address_space(3))) f32x4 *LdsF32x4;
typedef const __attribute__((address_space(3))) float *LdsF32;
typedef __attribute__((address_space(3))) uint8_t *LdsU8;

struct Tiling {
    int64_t n_tiles, tiles; // of the result
    int64_t per_split;      // blocks of K of one split
    int splits;
    int64_t part_ld;        // row length of the partial results (splits > 1)
};

template <int TM, int TN, int WM, int WN, bool W1, bool EXACT, typename OUT>
__global__ __launch_bounds__(64 * WM * WN) void tiles_kernel(Product p, Tiling g, OUT *C, float *parts)
{
    constexpr int kWaves = WM * WN, BM = 16 * TM * WM, BN = 16 * TN * WN, kRows = BM + BN;
    constexpr uint32_t kStage = kRows * kRowBytes, kScales = 2 * kStage, kScaleStage = kRows * 4;
    constexpr int kFetches = kRows / 8 / kWaves;
    static_assert(kRows % (8 * kWaves) == 0 && kRows % 64 == 0 && kRows / 64 <= kWaves && BM % 64 == 0, "whole fetches");
    __shared__ __attribute__((aligned(1024))) uint8_t smem[kScales + 2 * kScaleStage];
    const uint32_t lds = (uint32_t)(uintptr_t)(LdsU8)smem;

    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), row = lane % 16, part = lane / 16;
    const int wm = wave % WM, wn = wave / WM;
    // workgroups go round over the eight XCDs: each XCD takes a contiguous range of the tiles
    const uint32_t wgs = gridDim.x, xcd = blockIdx.x % 8, in_xcd = blockIdx.x / 8, base = wgs / 8, more = wgs % 8;
    const uint32_t job = xcd * base + min(xcd, more) + in_xcd;
    const uint32_t split = job / (uint32_t)g.tiles, tile = job - split * (uint32_t)g.tiles;
    // tiles in bands of eight along the tokens, so that a range of them shares rows of both operands
    const uint32_t n_tiles = (uint32_t)g.n_tiles, m_tiles = (uint32_t)(g.tiles / g.n_tiles), band = tile / (8 * n_tiles);
    const uint32_t in_band = tile - band * 8 * n_tiles, height = min(8u, m_tiles - 8 * band);
    const int64_t m0 = (int64_t)(8 * band + in_band % height) * BM, n0 = (int64_t)(in_band / height) * BN;
    const int64_t kb0 = split * g.per_split, kb1 = min(kb0 + g.per_split, p.k_blocks);

    const uint8_t *const a_base = p.A + m0 * p.lda, *const w_base = p.W + n0 * p.ldw;
    const int m_last = (int)min(p.M - 1 - m0, (int64_t)BM - 1), n_last = (int)min(p.N - 1 - n0, (int64_t)BN - 1);
    uint32_t at[kFetches]; // this lane's offset of each fetch: rows behind the last repeat it
#pragma unroll
    for (int j = 0; j < kFetches; ++j) {
        const int r = 8 * (wave * kFetches + j) + lane / 8; // of the tile: tokens, then features
        const uint32_t chunk = 16 * ((lane % 8) ^ (lane / 8));
        at[j] = (r < BM ? (uint32_t)min(r, m_last) * (uint32_t)p.lda : (uint32_t)min(r - BM, n_last) * (uint32_t)p.ldw) + chunk;
    }
    const bool a_scales = 64 * wave < BM;
    const int64_t w_row0 = n0 / p.w_rows;
    const uint32_t scale_at = 4 * (a_scales ? (uint32_t)min(64 * wave + lane, m_last)
                                            : (uint32_t)((n0 + min(64 * wave + lane - BM, n_last)) / p.w_rows - w_row0));
    const float *const scale_base = a_scales ? p.SA + m0 : p.SW + w_row0;
    const int64_t scale_step = a_scales ? p.ldsa : p.ldsw;

    auto fetch = [&](int64_t kb) {
        const uint32_t buf = (uint32_t)(kb & 1);
        const bool last = kb == p.k_blocks - 1;
#pragma unroll
        for (int j = 0; j < kFetches; ++j) {
            const int g8 = wave * kFetches + j;
            const bool of_a = 8 * g8 < BM;
            uint32_t off = at[j];
            if (last) { // chunks behind the row's end repeat its last one
                const int32_t room = (int32_t)((of_a ? p.lda : p.ldw) - kb * kBlock) - 16;
                const int32_t chunk = 16 * ((lane % 8) ^ (lane / 8));
                off -= (uint32_t)max(0, chunk - room);
            }
            fetch16((of_a ? a_base : w_base) + kb * kBlock, off, lds + buf * kStage + 1024u * g8);
        }
        if (64 * wave < kRows) fetch4(scale_base + kb * scale_step, scale_at, lds + kScales + buf * kScaleStage + 256u * wave);
    };

    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    const uint32_t frag = row * kRowBytes + 16 * ((2 * part) ^ (row % 8));
    const uint32_t a_at = lds + wm * (16 * TM * kRowBytes) + frag, w_at = lds + BM * kRowBytes + wn * (16 * TN * kRowBytes) + frag;
    const uint32_t sa_at = lds + kScales + 4 * (wm * 16 * TM + row), sw_at = lds + kScales + 4 * (BM + wn * 16 * TN + 4 * part);

    fetch(kb0);
    for (int64_t kb = kb0; kb < kb1; ++kb) {
        const uint32_t buf = (uint32_t)(kb & 1), stage = buf * kStage, scales = buf * kScaleStage;
        arrived();
        barrier(); // block kb is there, and nobody reads the other buffer any more
        if (kb + 1 < kb1) fetch(kb + 1);
        if ((kb + 1) * kBlock > p.K) { // codes behind K
            const int keep = (int)(p.K - kb * kBlock);
            for (uint32_t i = threadIdx.x; i < kRows * 8; i += 64 * kWaves) {
                const uint32_t r = i / 8, chunk = (i % 8) ^ (r % 8);
                __attribute__((address_space(3))) uint32_t *w = (__attribute__((address_space(3))) uint32_t *)(lds + stage + 16 * i);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int left = keep - (int)(16 * chunk + 4 * e);
                    if (left <= 0) w[e] = 0;
                    else if (left < 4) w[e] &= (1u << (8 * left)) - 1u;
                }
            }
            barrier();
        }
        auto load = [&](uint32_t a) {
            const u32x4 lo = *(LdsU32x4)a, hi = *(LdsU32x4)(a ^ 16u);
            return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
        };
        i32x8 a[TM];
        float s[TM];
        [[maybe_unused]] const float sw = W1 ? 0.f : *(LdsF32)(sw_at + scales);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            a[i] = load(a_at + stage + 16 * kRowBytes * i);
            s[i] = *(LdsF32)(sa_at + scales + 64 * i);
            if constexpr (!W1) s[i] *= sw;
        }
        if constexpr (EXACT) {
            f16x8 aw[TM][4];
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) aw[i][e] = widened(a[i][2 * e], a[i][2 * e + 1]);
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const i32x8 w = load(w_at + stage + 16 * kRowBytes * j);
                [[maybe_unused]] f32x4 s4;
                if constexpr (W1) s4 = *(LdsF32x4)(sw_at + scales + 64 * j);
                f16x8 ww[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) ww[e] = widened(w[2 * e], w[2 * e + 1]);
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum = __builtin_amdgcn_mfma_f32_16x16x32_f16(ww[e], aw[i][e], sum, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] = __builtin_fmaf(sum[e], W1 ? s[i] * s4[e] : s[i], acc[i][j][e]);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const i32x8 w = load(w_at + stage + 16 * kRowBytes * j);
                [[maybe_unused]] f32x4 s4;
                if constexpr (W1) s4 = *(LdsF32x4)(sw_at + scales + 64 * j);
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    const f32x4 sum = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, a[i], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] = __builtin_fmaf(sum[e], W1 ? s[i] * s4[e] : s[i], acc[i][j][e]);
                }
            }
        }
    }

#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t m = m0 + 16 * (TM * wm + i) + row;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t n = n0 + 16 * (TN * wn + j) + 4 * part;
            if (m >= p.M || n >= p.N) continue;
            if (g.splits > 1) store4(parts + ((int64_t)split * p.M + m) * g.part_ld + n, acc[i][j], p.N - n);
            else store4(C + m * p.ldc + n, acc[i][j], p.N - n);
        }
    }
}

// The partial results of the splits, added in their order.
template <typename OUT>
__global__ __launch_bounds__(256) void join_kernel(const float *parts, int splits, int64_t part_ld, OUT *C, int64_t ldc, int64_t M, int64_t N)
{
    const int64_t row_units = part_ld / 4, units = M * row_units, step = M * part_ld;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < units; u += (int64_t)gridDim.x * 256) {
        const int64_t m = u / row_units, n = 4 * (u - m * row_units);
        const float *q = parts + m * part_ld + n;
        f32x4 sum = *reinterpret_cast<const f32x4 *>(q);
        for (int i = 1; i < splits; ++i) sum += *reinterpret_cast<const f32x4 *>(q + i * step);
        store4(C + m * ldc + n, sum, N - n);
    }
}

template <int TM, int TN, int WM, int WN, bool EXACT, typename OUT>
int run_tiles(const Product &p, OUT *C, void *workspace, size_t workspace_bytes, hipStream_t s)
{
    constexpr int BM = 16 * TM * WM, BN = 16 * TN * WN;
    Tiling g;
    g.n_tiles = ceil_div(p.N, BN);
    g.tiles = g.n_tiles * ceil_div(p.M, BM);
    if (g.tiles > kMaxTiles) return ZS_ERR_SHAPE;
    g.part_ld = (p.N + 3) / 4 * 4;
    const int64_t cus = zs_compute_units();
    int64_t splits = g.tiles >= cus ? 1 : cus / g.tiles;
    splits = std::min(splits, p.k_blocks / 4); // at least four blocks each
    splits = std::min(splits, workspace ? (int64_t)(workspace_bytes / (4 * (size_t)p.M * (size_t)g.part_ld)) : 0);
    g.per_split = ceil_div(p.k_blocks, splits > 1 ? splits : 1);
    g.splits = (int)ceil_div(p.k_blocks, g.per_split);
    float *parts = static_cast<float *>(workspace);
    const dim3 grid((unsigned)(g.tiles * g.splits)), wg(64 * WM * WN);
    if (p.w_rows == 1) hipLaunchKernelGGL((tiles_kernel<TM, TN, WM, WN, true, EXACT, OUT>), grid, wg, 0, s, p, g, C, parts);
    else hipLaunchKernelGGL((tiles_kernel<TM, TN, WM, WN, false, EXACT, OUT>), grid, wg, 0, s, p, g, C, parts);
    if (g.splits > 1)
        hipLaunchKernelGGL(join_kernel<OUT>, dim3(grid_for(ceil_div(p.M * g.part_ld / 4, 256))), dim3(256), 0, s, parts, g.splits, g.part_ld, C,
                           p.ldc, p.M, p.N);
    return launched();
}

template <typename OUT>
int run(const uint8_t *A, int64_t lda, const float *SA, int64_t ldsa, const uint8_t *W, int64_t ldw, const float *SW, int64_t ldsw, int w_rows,
        OUT *C, int64_t ldc, int64_t M, int64_t N, int64_t K, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!A || !SA || !W || !SW || !C) return ZS_ERR_ARG;
    if (!aligned(A, 16) || !aligned(W, 16) || !aligned(C, 16) || !aligned(SA, 4) || !aligned(SW, 4) || !aligned(workspace, 256)) return ZS_ERR_ARG;
    if (w_rows != 1 && w_rows != kBlock) return ZS_ERR_CONFIG;
    if (M < 1 || N < 1 || K < 1 || M > INT32_MAX || N > INT32_MAX || K > INT32_MAX) return ZS_ERR_SHAPE;
    if (lda < K || lda % 16 || ldw < K || ldw % 16 || ldc < N || ldc % 4 || ldsa < M || ldsw < ceil_div(N, w_rows)) return ZS_ERR_SHAPE;
    if (lda > kMaxLd || ldw > kMaxLd) return ZS_ERR_SHAPE; // offsets inside a tile are 32 bits wide
    const Product p = {A, W, SA, SW, lda, ldsa, ldw, ldsw, ldc, M, N, K, ceil_div(K, kBlock), w_rows};
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (M > 32) {
        if (M <= 64) return run_tiles<4, 2, 1, 4, true>(p, C, workspace, workspace_bytes, stream);
        constexpr bool kExact = std::is_same_v<OUT, float>;
        if constexpr (kExact) return run_tiles<4, 4, 4, 2, true>(p, C, workspace, workspace_bytes, stream);
        else return run_tiles<4, 8, 4, 2, false>(p, C, workspace, workspace_bytes, stream);
    }
    if (M > 16) return run_stream<2, 1, 8, 4>(p, C, stream);
    return run_stream<1, 1, 8, 4>(p, C, stream);
}

} // namespace

extern "C" int zs_fp8_gemm(const uint8_t *A_dev, int64_t lda, const float *SA_dev, int64_t ldsa, const uint8_t *W_dev, int64_t ldw,
                           const float *SW_dev, int64_t ldsw, int w_rows, float *C_dev, int64_t ldc, int64_t M, int64_t N, int64_t K,
                           void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    return run(A_dev, lda, SA_dev, ldsa, W_dev, ldw, SW_dev, ldsw, w_rows, C_dev, ldc, M, N, K, workspace_dev, workspace_bytes, hip_stream);
}

extern "C" int zs_fp8_gemm_bf16(const uint8_t *A_dev, int64_t lda, const float *SA_dev, int64_t ldsa, const uint8_t *W_dev, int64_t ldw,
                                const float *SW_dev, int64_t ldsw, int w_rows, uint16_t *C_dev, int64_t ldc, int64_t M, int64_t N,
                                int64_t K, void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    return run(A_dev, lda, SA_dev, ldsa, W_dev, ldw, SW_dev, ldsw, w_rows, C_dev, ldc, M, N, K, workspace_dev, workspace_bytes, hip_stream);
}
