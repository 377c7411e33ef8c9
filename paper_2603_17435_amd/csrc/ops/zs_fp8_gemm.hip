// zs_fp8_gemm: C[m,n] = sum over blocks b of 128 along K of SA[b,m] SW[b,n / w_rows] sum_{k in b} A[m,k] W[n,k]
// on E4M3 codes.  The products of one block of K are summed by the matrix cores; the sum is scaled once and added to an
// FP32 accumulator.
#include "zs_ops.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

using namespace zs_ops;

namespace {

constexpr int kBlock = 128;
constexpr int64_t kMaxLd = (int64_t)1 << 23;

struct Product {
    const uint8_t *A, *W;
    const float *SA, *SW;
    int64_t lda, ldsa, ldw, ldsw, ldc;
    int64_t M, N, K, k_blocks;
    int w_rows;
};

// Eight codes as FP16 numbers, which hold every one of them exactly; v_mfma_f32_16x16x32_f16 then sums whole products in
// FP32.  (The 8-bit matrix instructions run at twice the rate, but of each group of eight products they drop what lies below 2^-13
// of the largest before they sum: 448 * 448 - 448 * 448 + 1 gives 0.)
__device__ __forceinline__ f16x8 widened(uint32_t lo, uint32_t hi)
{
    const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true);
    const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true);
    return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ i32x8 joined(u32x4 lo, u32x4 hi)
{
    return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// Mask of a word of four codes of which `left` lie before K.
__device__ __forceinline__ uint32_t kept(int left) { return left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1u; }

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
// A workgroup keeps the codes of all M <= 16 tokens in LDS and multiplies them by one tile of 16 features after
// another.  Its NW waves share a tile's blocks of 128 along K and add their sums up in LDS, always in the same order.
// Each wave requests its blocks of W, of this tile and the next ones, D ahead, straight into operand registers: a lane
// takes the chunks of 16 bytes `part` and `part` + 4 of its row, so that a load covers 64 contiguous bytes
// of sixteen rows.  W is the first operand, so a lane holds four features of one token.  Bound by the weights' way from
// memory: FP32 results of 28672 x 4096 take 25 us for one token (4.7 TB/s) and 28 us for sixteen, whose codes in LDS save 6 us
// over fetching them from the L2 for every tile; below 10 MB of weights by latency (4096 features of 1024 codes: 3.6 to 4.4 us, 1024 of 4096: 5.2 to 5.8).
constexpr size_t kLds = 160 * 1024;
constexpr size_t stream_sums(int waves) { return (size_t)2 * waves * 1024; }
constexpr size_t stream_block(int rows) { return (size_t)rows * (kBlock + 4); } // a block's codes and scales

template <int NW, int D, bool W1, typename OUT>
__global__ __launch_bounds__(64 * NW) void stream_kernel(Product p, OUT *C)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), row = lane % 16, part = lane / 16;
    const int blocks = (int)p.k_blocks, rows = (int)p.M;
    const int64_t n_tiles = (p.N + 15) / 16;
    const int tiles = (int)((n_tiles - blockIdx.x + gridDim.x - 1) / gridDim.x); // of this workgroup: its own number, and so on in steps of the grid
    f32x4 *const sums = reinterpret_cast<f32x4 *>(smem);                         // [2][NW][64]
    uint8_t *const codes = smem + stream_sums(NW);                               // [blocks][rows][128], chunk c of a row at c ^ (row % 8)
    float *const scales = reinterpret_cast<float *>(codes + (size_t)blocks * rows * kBlock); // [blocks][rows]

    struct Block {
        u32x4 w[2];
        f32x4 sw;
    };
    const int per_tile = (blocks - wave + NW - 1) / NW; // blocks of this wave in a tile: wave, wave + NW, ...
    Block b[D];
    int at_tile = 0, at_block = 0; // of the next request
    auto request = [&](Block &to) {
        if (at_tile >= tiles) return;
        const int64_t n0 = 16 * (blockIdx.x + (int64_t)at_tile * gridDim.x), kb = wave + at_block * NW;
        const int n_last = (int)min(p.N - 1 - n0, (int64_t)15);
        const uint8_t *base = p.W + n0 * p.ldw + kb * kBlock;
        const uint32_t room = (uint32_t)min(p.ldw - kb * kBlock - 16, (int64_t)112), at = (uint32_t)min(row, n_last) * (uint32_t)p.ldw;
#pragma unroll
        for (int h = 0; h < 2; ++h) // (chunks behind the row's end repeat its last one)
            to.w[h] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(base + (at + min((uint32_t)(16 * part + 64 * h), room))));
        const float *sw = p.SW + kb * p.ldsw;
        if constexpr (W1) {
#pragma unroll
            for (int e = 0; e < 4; ++e) to.sw[e] = sw[n0 + min(4 * part + e, n_last)];
        } else {
            to.sw[0] = sw[n0 / kBlock];
        }
        if (++at_block >= per_tile) {
            at_block = 0;
            ++at_tile;
        }
    };
    if (per_tile > 0)
#pragma unroll
        for (int d = 0; d < D; ++d) request(b[d]);

    for (int i = threadIdx.x; i < blocks * rows * 8; i += 64 * NW) {
        const int chunk = i % 8, r = i / 8 % rows, kb = i / 8 / rows;
        const int64_t k = (int64_t)kb * kBlock + 16 * chunk;
        u32x4 v = {0, 0, 0, 0};
        if (k < p.K) v = *reinterpret_cast<const u32x4 *>(p.A + r * p.lda + k);
        if (k + 16 > p.K) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] &= kept((int)(p.K - (k + 4 * e)));
        }
        *reinterpret_cast<u32x4 *>(codes + (size_t)(kb * rows + r) * kBlock + 16 * (chunk ^ (r % 8))) = v;
    }
    for (int i = threadIdx.x; i < blocks * rows; i += 64 * NW) scales[i] = p.SA[i / rows * p.ldsa + i % rows];
    __syncthreads();

    const int r = min(row, rows - 1);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](Block &v, int block) {
        if ((int64_t)(block + 1) * kBlock > p.K) { // codes behind K
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) v.w[h][e] &= kept((int)(p.K - ((int64_t)block * kBlock + 16 * part + 64 * h + 4 * e)));
        }
        const uint8_t *c = codes + (size_t)(block * rows + r) * kBlock;
        const u32x4 a[2] = {*reinterpret_cast<const u32x4 *>(c + 16 * (part ^ (r % 8))), *reinterpret_cast<const u32x4 *>(c + 16 * ((part + 4) ^ (r % 8)))};
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 4; ++e)
            sum = __builtin_amdgcn_mfma_f32_16x16x32_f16(widened(v.w[e / 2][2 * (e % 2)], v.w[e / 2][2 * (e % 2) + 1]),
                                                         widened(a[e / 2][2 * (e % 2)], a[e / 2][2 * (e % 2) + 1]), sum, 0, 0, 0);
        const float sa = scales[block * rows + r];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(sum[e], sa * v.sw[W1 ? e : 0], acc[e]);
    };
    int tile = 0, block = 0;
    auto finish = [&] { // the tile is done: its sums of all waves, added by one of them
        f32x4 *const mine = sums + (tile % 2) * (NW * 64);
        mine[wave * 64 + lane] = acc;
        __syncthreads();
        if (tile % NW == wave) {
            f32x4 sum = mine[lane];
#pragma unroll
            for (int w = 1; w < NW; ++w) sum += mine[w * 64 + lane];
            const int64_t n = 16 * (blockIdx.x + (int64_t)tile * gridDim.x) + 4 * part;
            if (row < rows && n < p.N) store4(C + row * p.ldc + n, sum, p.N - n);
        }
        acc = f32x4{0.f, 0.f, 0.f, 0.f};
        block = 0;
        ++tile;
    };
    if (per_tile <= 0) { // fewer blocks than waves: only the barriers and the sums
        while (tile < tiles) finish();
        return;
    }
    while (tile < tiles) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            if (tile < tiles) {
                multiply(b[d], wave + block * NW);
                request(b[d]);
                if (++block == per_tile) finish();
            }
        }
    }
}

// ---- tiles through LDS ---------------------------------------------------------------------
// A workgroup of WM x WN waves computes (16 TM WM) tokens x (16 TN WN) features over the blocks [kb0, kb1) of K.  Each
// block's codes and scales go from memory straight to LDS; STAGES - 1 blocks are under way while one is
// multiplied, and there is one barrier a block.  A row's eight chunks of 16 bytes lie in the order chunk ^ (row % 8), so that
// the sixteen rows of an operand are read without bank conflicts.  4096 tokens, 28672 x 4096, BF16 results: 827 to 930 us (1.03 to 1.16
// PFLOP/s); FP32 results 6144 x 4096 x 5003, w_rows 1: 249 to 269 us (0.94 to 1.01).  Bound by the matrix instructions (the library's BF16 product
// takes 645 us of the former) with the conversions to FP16 (two to a matrix instruction in tiles of 256 x 128) and the scaling FMAs beside them.
constexpr int kRowBytes = 128;

// 64 lanes x 16 (or 4) bytes from base + at to the 1 KB (256 bytes) of LDS at `to`.  Not tracked by the compiler: arrived() waits for them.
__device__ __forceinline__ void fetch16(const void *base, uint32_t at, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(at), "s"(base), "s"(to) : "memory", "m0");
}
__device__ __forceinline__ void fetch4(const void *base, uint32_t at, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(at), "s"(base), "s"(to) : "memory", "m0");
}
template <int LEFT> // all fetches of this wave but the youngest LEFT
__device__ __forceinline__ void arrived()
{
    static_assert(LEFT < 64, "vmcnt is a 6-bit counter");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory");
}
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

// A wave's 16 TM x 16 TN results to memory.  A lane holds four features of one token, so that direct stores would leave
// in pieces of 32 or 64 bytes of sixteen rows; through LDS, sixteen tokens at a time, they leave as whole rows of the tile.
// 4096 x 8192 x 128, FP32 results: 57 -> 36 us.  `room`: LDS of this wave alone.
template <int TM, int TN, typename T>
__device__ __forceinline__ void store_tile(T *to, int64_t ld, const f32x4 (&acc)[TM][TN], uint32_t room, int lane, int64_t rows, int64_t cols)
{
    constexpr int kRow = 16 * TN * (int)sizeof(T), kChunks = kRow / 16, kPerChunk = 16 / (int)sizeof(T); // a chunk c lies at c ^ (row % kChunks)
    const int row = lane % 16, part = lane / 16;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            if constexpr (sizeof(T) == 4) {
                *(__attribute__((address_space(3))) f32x4 *)(room + row * kRow + 16 * ((4 * j + part) ^ (row % kChunks))) = acc[i][j];
            } else {
                const f32x4 v = acc[i][j];
                *(__attribute__((address_space(3))) u32x2 *)(room + row * kRow + 16 * ((2 * j + part / 2) ^ (row % kChunks)) + 8 * (part % 2)) =
                    u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int k = 0; k < kChunks / 4; ++k) {
            const int r = (64 * k + lane) / kChunks, c = (64 * k + lane) % kChunks;
            const u32x4 v = *(LdsU32x4)(room + r * kRow + 16 * (c ^ (r % kChunks)));
            const int64_t left = cols - kPerChunk * c;
            T *const q = to + (16 * i + r) * ld + kPerChunk * c;
            if (16 * i + r >= rows || left <= 0) continue;
            if (left >= kPerChunk) {
                store_any(q, v);
            } else {
#pragma unroll
                for (int e = 0; e < kPerChunk; ++e)
                    if (e < left) {
                        if constexpr (sizeof(T) == 4) q[e] = __builtin_bit_cast(f32x4, v)[e];
                        else q[e] = (uint16_t)(v[e / 2] >> (16 * (e % 2)));
                    }
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); // (read before the next sixteen tokens are written)
    }
}

// The tile that a workgroup computes.  Workgroups go round over the eight XCDs, each with an L2 of its own: an XCD
// takes a contiguous range of the tiles, which lie in bands of eight along the tokens, so that the range shares rows
// of both operands.
struct TilePlace {
    uint32_t split, m, n;
};
__device__ __forceinline__ TilePlace place_of(uint32_t wg, uint32_t wgs, const Tiling &g)
{
    const uint32_t xcd = wg % 8, job = xcd * (wgs / 8) + min(xcd, wgs % 8) + wg / 8;
    const uint32_t tiles = (uint32_t)g.tiles, n_tiles = (uint32_t)g.n_tiles, m_tiles = tiles / n_tiles;
    TilePlace at;
    at.split = job / tiles;
    const uint32_t tile = job - at.split * tiles, band = tile / (8 * n_tiles), in_band = tile - band * 8 * n_tiles;
    const uint32_t height = min(8u, m_tiles - 8 * band);
    at.m = 8 * band + in_band % height;
    at.n = in_band / height;
    return at;
}

// Waves that a SIMD has to hold, so that two workgroups share a compute unit whose LDS has room for both.  BF16 results with w_rows 1 take 129
// registers for a tile of 128 x 128 if the compiler is not told, one too many; FP32 results take 128, and told they would spill.
template <int TM, int TN, int WM, int WN, int STAGES, typename OUT>
constexpr int kWavesPerSimd = sizeof(OUT) == 2 && 2 * STAGES * 16 * (TM * WM + TN * WN) * (kRowBytes + 4) <= (int)kLds ? 2 * WM * WN / 4 : 1;

template <int TM, int TN, int WM, int WN, int STAGES, bool W1, typename OUT>
__global__ __launch_bounds__(64 * WM * WN, (kWavesPerSimd<TM, TN, WM, WN, STAGES, OUT>)) void tiles_kernel(Product p, Tiling g, OUT *C, float *parts)
{
    constexpr int kWaves = WM * WN, BM = 16 * TM * WM, BN = 16 * TN * WN, kRows = BM + BN;
    constexpr uint32_t kStage = kRows * (kRowBytes + 4), kScales = kRows * kRowBytes;
    constexpr int kFetches = kRows / 8 / kWaves;
    static_assert(kRows % (8 * kWaves) == 0 && kRows % 64 == 0 && kRows / 64 <= kWaves && BM % 64 == 0, "whole fetches");
    __shared__ __attribute__((aligned(1024))) uint8_t smem[STAGES * kStage];
    const uint32_t lds = (uint32_t)(uintptr_t)(LdsU8)smem;

    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), row = lane % 16, part = lane / 16;
    const int wm = wave % WM, wn = wave / WM;
    const TilePlace place = place_of(blockIdx.x, gridDim.x, g);
    const uint32_t split = place.split;
    const int64_t m0 = (int64_t)place.m * BM, n0 = (int64_t)place.n * BN;
    const int kb0 = (int)(split * (uint32_t)g.per_split), kb1 = min(kb0 + (int)g.per_split, (int)p.k_blocks);

    const uint8_t *const a_base = p.A + m0 * p.lda, *const w_base = p.W + n0 * p.ldw;
    const int m_last = (int)min(p.M - 1 - m0, (int64_t)BM - 1), n_last = (int)min(p.N - 1 - n0, (int64_t)BN - 1);
    uint32_t at[kFetches]; // this lane's offset of each fetch: rows behind the last repeat it
#pragma unroll
    for (int j = 0; j < kFetches; ++j) {
        const int r = 8 * (wave * kFetches + j) + lane / 8; // of the tile: tokens, then features
        const uint32_t chunk = 16 * ((lane % 8) ^ (lane / 8));
        at[j] = (r < BM ? (uint32_t)min(r, m_last) * (uint32_t)p.lda : (uint32_t)min(r - BM, n_last) * (uint32_t)p.ldw) + chunk;
    }
    const int sw_wave = wave % (kRows / 64); // every wave fetches scales, so that all count the same
    const bool a_scales = 64 * sw_wave < BM;
    const int64_t w_row0 = n0 / p.w_rows;
    const uint32_t scale_at = 4 * (a_scales ? (uint32_t)min(64 * sw_wave + lane, m_last)
                                            : (uint32_t)((n0 + min(64 * sw_wave + lane - BM, n_last)) / p.w_rows - w_row0));
    const float *const scale_base = a_scales ? p.SA + m0 : p.SW + w_row0;
    const int64_t scale_step = a_scales ? p.ldsa : p.ldsw;

    const int k_last = (int)p.k_blocks - 1;
    const uint8_t *a_block, *w_block;
    const float *scale_block;
    // Each XCD begins at an eighth of its own of the blocks and comes round.  If all began at the first one, they would read the same few columns of all rows
    // at a time, which lie in few of the memory's channels if a row is a power of two long.  16 tokens x 28672 x 4096 31.3 -> 28.6 us, 64 tokens 33.9 -> 30.2,
    // 32 x 32768 x 8192 63.1 -> 57.4; with 512 tokens or more within 1 %.
    const int blocks = kb1 - kb0, first = (int)(blockIdx.x % 8 * (uint32_t)blocks / 8);
    int coming = kb0 + first; // block of the next fetches; behind the last one they take some again, so that all waits count the same
    bool cut = false;
    auto aim = [&] {
        if (cut != (coming == k_last)) { // in the last block chunks behind the row's end repeat its last one
            const int chunk = 16 * ((lane % 8) ^ (lane / 8));
            const int a_over = max(0, chunk + 16 - (int)(p.lda - (int64_t)k_last * kBlock)), w_over = max(0, chunk + 16 - (int)(p.ldw - (int64_t)k_last * kBlock));
#pragma unroll
            for (int j = 0; j < kFetches; ++j) {
                const int over = 8 * (wave * kFetches + j) < BM ? a_over : w_over;
                at[j] += cut ? over : -over;
            }
            cut = !cut;
        }
        a_block = a_base + (int64_t)coming * kBlock;
        w_block = w_base + (int64_t)coming * kBlock;
        scale_block = scale_base + coming * scale_step;
        coming = coming + 1 == kb1 ? kb0 : coming + 1;
    };
    auto fetch = [&](int from, int to, uint32_t stage) { // pieces of this wave's kFetches of codes and one of scales
#pragma unroll
        for (int j = 0; j <= kFetches; ++j) {
            if (j < from || j >= to) continue;
            const int g8 = wave * kFetches + j;
            if (j < kFetches) fetch16(8 * g8 < BM ? a_block : w_block, at[j], lds + stage + 1024u * g8);
            else fetch4(scale_block, scale_at, lds + stage + kScales + 256u * sw_wave);
        }
    };

    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    // a lane takes the chunks `part` and `part` + 4 of its row
    const uint32_t frag = row * kRowBytes + 16 * (part ^ (row % 8));
    const uint32_t a_at = lds + wm * (16 * TM * kRowBytes) + frag, w_at = lds + BM * kRowBytes + wn * (16 * TN * kRowBytes) + frag;
    const uint32_t sa_at = lds + kScales + 4 * (wm * 16 * TM + row), sw_at = lds + kScales + 4 * (BM + wn * 16 * TN + 4 * part);

#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) {
        aim();
        fetch(0, kFetches + 1, i * kStage);
    }
    uint32_t stage = 0, ahead = (STAGES - 1) * kStage; // where this block is, and where the one STAGES - 1 after it goes
    int kb = kb0 + first;
    for (int i = 0; i < blocks; ++i, kb = kb + 1 == kb1 ? kb0 : kb + 1, stage = stage == (STAGES - 1) * kStage ? 0 : stage + kStage,
             ahead = ahead == (STAGES - 1) * kStage ? 0 : ahead + kStage) {
        arrived<(STAGES - 2) * (kFetches + 1)>();
        barrier(); // this block is there, and nobody reads the one before any more
        aim();
        if (kb == k_last && p.K % kBlock) { // codes behind K
            const int keep = (int)(p.K % kBlock);
            for (uint32_t i = threadIdx.x; i < kRows * 8; i += 64 * kWaves) {
                const uint32_t r = i / 8, chunk = (i % 8) ^ (r % 8);
                __attribute__((address_space(3))) uint32_t *w = (__attribute__((address_space(3))) uint32_t *)(lds + stage + 16 * i);
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] &= kept(keep - (int)(16 * chunk + 4 * e));
            }
            barrier();
        }
        const uint32_t a_lo = a_at + stage, a_hi = (a_at ^ 64u) + stage, w_lo = w_at + stage, w_hi = (w_at ^ 64u) + stage;
        auto codes = [&](uint32_t lo, uint32_t hi, int tile) {
            return joined(*(LdsU32x4)(lo + 16 * kRowBytes * tile), *(LdsU32x4)(hi + 16 * kRowBytes * tile));
        };
        // A sum is scaled and added while the matrix cores work on the next ones.  The fetches go out during the first half of the
        // block, not all of them behind the barrier (28672 x 4096 with 4096 tokens, BF16 results: 850 instead of 860 us; 4096 x 8192 x 8192, FP32: 474
        // instead of 462).
        auto fetch_part = [&](int j) {
            constexpr int kPer = 2 * kFetches / TN;
            fetch(j * kPer, j == TN - 1 ? kFetches + 1 : (j + 1) * kPer, ahead);
        };
        i32x8 a[TM], w[2];
        f32x4 s4[2];
        float s[TM];
        w[0] = codes(w_lo, w_hi, 0);
#pragma unroll
        for (int i = 0; i < TM; ++i) a[i] = codes(a_lo, a_hi, i);
        const float sw = W1 ? 1.f : *(LdsF32)(sw_at + stage);
#pragma unroll
        for (int i = 0; i < TM; ++i) s[i] = *(LdsF32)(sa_at + stage + 64 * i) * sw;
        auto add = [&](f32x4 sum, int i, int j) {
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] = __builtin_fmaf(sum[e], W1 ? s[i] * s4[j % 2][e] : s[i], acc[i][j][e]);
            asm volatile("" : "+v"(acc[i][j])); // here, and not behind the next barrier
        };
        f16x8 aw[TM][4], ww[4];
        f32x4 sum[2][TM];
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) aw[i][e] = widened(a[i][2 * e], a[i][2 * e + 1]);
#pragma unroll
        for (int j = 0; j <= TN; ++j) {
            if (j < TN) {
                fetch_part(j);
#pragma unroll
                for (int e = 0; e < 4; ++e) ww[e] = widened(w[j % 2][2 * e], w[j % 2][2 * e + 1]);
                if (j + 1 < TN) w[(j + 1) % 2] = codes(w_lo, w_hi, j + 1);
                if constexpr (W1) s4[j % 2] = *(LdsF32x4)(sw_at + stage + 64 * j);
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int i = 0; i < TM; ++i)
                        sum[j % 2][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ww[e], aw[i][e], e ? sum[j % 2][i] : f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
            }
            if (j > 0) {
#pragma unroll
                for (int i = 0; i < TM; ++i) add(sum[(j + 1) % 2][i], i, j - 1);
            }
        }
    }

    arrived<0>();
    barrier(); // LDS holds results from here on
    const int64_t m = m0 + 16 * TM * wm, n = n0 + 16 * TN * wn;
    const uint32_t room = lds + wave * (kStage * STAGES / kWaves / 1024 * 1024);
    if (g.splits > 1) store_tile<TM, TN>(parts + ((int64_t)split * p.M + m) * g.part_ld + n, g.part_ld, acc, room, lane, p.M - m, p.N - n);
    else store_tile<TM, TN>(C + m * p.ldc + n, p.ldc, acc, room, lane, p.M - m, p.N - n);
}

// The partial results of the splits, added in their order.  Bound by memory, or a launch: 200 x 4096 in four parts takes 4 us.
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

constexpr int kStreamWaves = 16;
// Dynamic LDS of the kernel for few tokens.
size_t stream_lds(const Product &p) { return stream_sums(kStreamWaves) + stream_block((int)p.M) * (size_t)p.k_blocks; }

// Its estimated time (us), or more than any if it cannot take the product.
double stream_time(const Product &p)
{
    if (p.M > 16 || stream_lds(p) > kLds) return HUGE_VAL;
    const double tiles = (double)ceil_div(ceil_div(p.N, 16), zs_compute_units()); // of a workgroup
    return 2.8 + tiles * (0.37 + (double)p.k_blocks * (0.0956 + 0.00125 * (double)p.M));
}

template <bool W1, typename OUT>
int run_stream(const Product &p, OUT *C, hipStream_t s)
{
    const int rc = allow_lds<stream_kernel<kStreamWaves, 2, W1, OUT>>(kLds);
    if (rc != ZS_OK) return rc;
    const dim3 grid((unsigned)std::min(ceil_div(p.N, 16), (int64_t)zs_compute_units()));
    hipLaunchKernelGGL((stream_kernel<kStreamWaves, 2, W1, OUT>), grid, dim3(64 * kStreamWaves), stream_lds(p), s, p, C);
    return launched();
}

// Tile shapes and what a round of them takes (us), with one workgroup to a compute unit (`alone`) or two: `start` for its
// first loads and its results, `block` for each block of 128 along K (0: LDS holds one).  For 2242 products of 17 to 6144 tokens (N 1000 to 32768, K 1000 to
// 14336, half of them with each type of results), timed with each shape and up to 16 splits, the ones chosen take 0.7 % longer than the
// fastest on the average, 16 % at most (254 x 4096 x 4096, BF16 results: 22.8 against 19.6 us).
struct RoundTime {
    float start, block;
};
struct TileShape {
    int tokens, features;
    RoundTime alone, two;
};
constexpr TileShape kShapes[] = {{64, 128, {2.05f, 0.74f}, {3.25f, 1.05f}}, {128, 128, {2.7f, 1.05f}, {2.85f, 1.70f}}, {256, 128, {4.25f, 1.52f}, {}}};

// The shape and number of splits along K with the least estimated time: rounds of workgroups times their blocks, no less than
// the operands' way from memory, which gives less to few workgroups, and for splits a second kernel (the partial results there and back at 7
// TB/s: they stay in the last cache).
struct TilePlan {
    int shape;
    double time;
    Tiling g;
};
TilePlan plan_tiles(const Product &p, size_t workspace_bytes)
{
    constexpr int kN = sizeof kShapes / sizeof *kShapes;
    const double cus = zs_compute_units(), operands = ((double)p.N + (double)p.M) * (double)p.K / 6.3e6;
    const int64_t part_ld = (p.N + 3) / 4 * 4;
    const uint32_t k_blocks = (uint32_t)p.k_blocks;
    int64_t n_tiles[kN], tiles[kN];
    for (int i = 0; i < kN; ++i) {
        n_tiles[i] = ceil_div(p.N, kShapes[i].features);
        tiles[i] = n_tiles[i] * ceil_div(p.M, kShapes[i].tokens);
    }
    TilePlan best{-1, 0, {}};
    for (uint32_t splits = 1; splits <= 16; ++splits) {
        const uint32_t per_split = (k_blocks + splits - 1) / splits;
        double join = 0;
        if (splits > 1) {
            if (per_split < 4) break;
            if ((k_blocks + per_split - 1) / per_split != splits || workspace_bytes / 4 / splits / (size_t)p.M < (size_t)part_ld) continue;
            join = 2.45 + 0.33 * splits + (double)splits * (double)p.M * (double)part_ld * 8 / 7e6;
        }
        for (int i = 0; i < kN; ++i) {
            const RoundTime &alone = kShapes[i].alone, &two = kShapes[i].two;
            const double wgs = (double)tiles[i] * splits;
            if (splits > 1 && wgs > 4 * cus) continue;
            const double one = alone.start + per_split * alone.block, pair = two.start + per_split * two.block;
            const bool pairs = two.block != 0.f;
            const double slots = pairs ? 2 * cus : cus, full = std::floor(wgs / slots), rest = wgs - full * slots;
            double time = full * (pairs ? pair : one) + (rest > cus ? pair : rest > 0 ? one : 0.0);
            double traffic = operands;
            if (wgs < 2 * cus) traffic /= std::sqrt(std::sqrt(std::sqrt(std::sqrt(wgs / (2 * cus)))));
            time = std::max(time, traffic) + 0.1 * time + join; // (of those that wait for memory, the one with less to do)
            if (best.shape < 0 || time < best.time) best = {i, time, {n_tiles[i], tiles[i], (int64_t)per_split, (int)splits, part_ld}};
        }
    }
    return best;
}

template <int TM, int TN, int WM, int WN, int STAGES, typename OUT>
int run_tiles(const Product &p, const Tiling &g, OUT *C, void *workspace, hipStream_t s)
{
    if (g.tiles * g.splits * (64 * WM * WN) > UINT32_MAX) return ZS_ERR_SHAPE; // (results of half a terabyte and more)
    float *parts = static_cast<float *>(workspace);
    const dim3 grid((unsigned)(g.tiles * g.splits)), wg(64 * WM * WN);
    if (p.w_rows == 1) hipLaunchKernelGGL((tiles_kernel<TM, TN, WM, WN, STAGES, true, OUT>), grid, wg, 0, s, p, g, C, parts);
    else hipLaunchKernelGGL((tiles_kernel<TM, TN, WM, WN, STAGES, false, OUT>), grid, wg, 0, s, p, g, C, parts);
    if (g.splits > 1)
        hipLaunchKernelGGL(join_kernel<OUT>, dim3(grid_for(ceil_div(p.M * g.part_ld / 4, 256))), dim3(256), 0, s, parts, g.splits, g.part_ld, C,
                           p.ldc, p.M, p.N);
    return launched();
}

template <typename OUT>
int run_tiled(const Product &p, const TilePlan &plan, OUT *C, void *workspace, hipStream_t s)
{
    if (plan.shape == 0) return run_tiles<4, 2, 1, 4, 3>(p, plan.g, C, workspace, s);
    if (plan.shape == 1) return run_tiles<2, 4, 4, 2, 2>(p, plan.g, C, workspace, s);
    return run_tiles<4, 4, 4, 2, 2>(p, plan.g, C, workspace, s);
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
    if (!workspace) workspace_bytes = 0;
    // The kernel for few tokens, where it is estimated to be faster (for few tokens tiles take a fifth longer than their plan says, a tenth where BF16
    // results halve what they write).  For 930 products of 1 to 16 tokens (N 1000 to 32768, K 1000 to 14336) this takes 0.5 % longer than the fastest of
    // all on the average, 14 % at most.  It is the one for rows of more than 1024 codes or so: one token x 28672 x 8192, FP32 results, 44 us against 54 in
    // tiles, sixteen tokens x 28672 x 4096 28.1 against 30.8, but 1 x 32768 x 1024 13.2 against 10.5, and its ends of a tile tell.
    const double few = stream_time(p), tiles_take = std::is_same_v<OUT, float> ? 1.2 : 1.1;
    TilePlan plan{};
    if (few < 8 || few <= (plan = plan_tiles(p, workspace_bytes)).time * tiles_take)
        return w_rows == 1 ? run_stream<true>(p, C, stream) : run_stream<false>(p, C, stream);
    return run_tiled(p, plan, C, workspace, stream);
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
