// Embedding operators: rows of a table by token ids, times a scale (zs_embed out of a compressed blob,
// zs_dense_embed out of a BF16 matrix), and the gradient of the table (zs_embed_grad).
#include "zs_device.h"
#include "zs_ops.h"

#include <algorithm>

using namespace zs_ops;

namespace {

// A token id, or -1 where it names no row of the table.
__device__ __forceinline__ int64_t id_at(const void *ids, int id_bytes, int64_t t, int64_t N)
{
    const int64_t id = id_bytes == 8 ? static_cast<const int64_t *>(ids)[t] : static_cast<const int32_t *>(ids)[t];
    return id >= 0 && id < N ? id : -1;
}

// ---- rows of the compressed table --------------------------------------------------------
// A wave decodes one token's 64 weights of one BlockTile.  Lane f first stands for FragTile f: where the
// row's bytes of a FragTile start in H is the number of in-window elements before them, which a prefix sum of the popcounts
// over the lanes gives.  Then lane c stands for the row's column c and fetches the three
// plane bytes and the start of the FragTile that holds it.  Per BlockTile 39 to 64 FragTiles' planes of 24 bytes and 64 to 128
// bytes of the row are read: 5000 frequent and rare tokens of 128256 x 4096 take 81 us for 425 MB, of which about a
// third comes from the caches.  Few tokens are bound by latency (32: 2.9 us).
struct Blob {
    const uint8_t *bitmaps;
    const u32x2 *offsets;
    const uint8_t *H;
    const uint8_t *L;
    uint64_t h_last, l_last; // offsets of the last byte of H and the last halfword of L: no read goes behind them
    int32_t base_exp;
    int32_t k_blocks;
};

template <int U> // BlockTiles whose planes a wave requests at a time
__global__ __launch_bounds__(256) void embed_kernel(Blob b, int64_t N, const void *ids, int id_bytes, int64_t T, float scale, uint16_t *Y,
                                                    int64_t ldy)
{
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), j = lane % 8;
    for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
        const int64_t id = id_at(ids, id_bytes, t, N);
        const int64_t first = id < 0 ? 0 : id / ZS_BT_DIM * b.k_blocks;
        const uint32_t row = (uint32_t)(id & (ZS_BT_DIM - 1)), r = row % 8;
        // column `lane`: FragTile column lane / 8, which lies in TensorCoreTile column lane / 32
        const uint32_t f_row = row / 16 * ZS_FT_PER_TT + row / 8 % 2;
        const uint32_t f = lane / 32 * (4 * ZS_FT_PER_TT) + lane / 8 % 4 * 2 + f_row, f_last = 4 * ZS_FT_PER_TT + 6 + f_row;
        const uint64_t below = (1ull << (8 * r)) - 1; // of a FragTile, the rows above this one
        for (uint32_t kb0 = (blockIdx.y * 4 + wave) * U; kb0 < (uint32_t)b.k_blocks; kb0 += gridDim.y * 4 * U) {
            uint16_t *const out = Y + t * ldy + ZS_BT_DIM * (int64_t)kb0 + lane;
            if (id < 0) {
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (kb0 + u < (uint32_t)b.k_blocks) out[ZS_BT_DIM * u] = 0;
                continue;
            }
            u32x2 p[U][3], starts[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t bt = first + min(kb0 + u, (uint32_t)b.k_blocks - 1);
                const u32x2 *planes = reinterpret_cast<const u32x2 *>(b.bitmaps + bt * ZS_BT_BITMAP_BYTES) + 3 * lane;
#pragma unroll
                for (int i = 0; i < 3; ++i) p[u][i] = lane <= f_last ? planes[i] : u32x2{0, 0}; // (those behind the row's last one do not matter)
                starts[u] = b.offsets[bt];
            }
            uint32_t value[U], code[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t lo = p[u][0].x | p[u][1].x | p[u][2].x, hi = p[u][0].y | p[u][1].y | p[u][2].y;
                const uint32_t count = __popc(lo) + __popc(hi);
                const uint32_t start = zs::wave_inclusive_scan(count) - count + __popc(lo & (uint32_t)below) + __popc(hi & (uint32_t)(below >> 32));
                const uint32_t at = 8 * (r % 4);
                auto byte = [&](u32x2 v) { return (r < 4 ? v.x : v.y) >> at & 0xFFu; };
                const uint32_t bytes = byte(p[u][0]) | byte(p[u][1]) << 8 | byte(p[u][2]) << 16;
                const uint32_t w = (uint32_t)__shfl((int)bytes, (int)f), m = (w | w >> 8 | w >> 16) & 0xFFu;
                const uint32_t h_at = (uint32_t)__shfl((int)start, (int)f) + __popc(m & ((1u << j) - 1u));
                code[u] = (w >> j & 1u) | (w >> (j + 8) & 1u) << 1 | (w >> (j + 16) & 1u) << 2;
                if (code[u]) {
                    value[u] = b.H[min(16 * (uint64_t)starts[u].x + h_at, b.h_last)];
                } else {
                    const uint32_t l_at = 64 * f + 8 * r + j - h_at;
                    value[u] = *reinterpret_cast<const uint16_t *>(b.L + min(16 * (uint64_t)starts[u].y + 2 * l_at, b.l_last));
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t h = value[u];
                const uint32_t bits = code[u] ? (h & 0x80u) << 8 | ((uint32_t)(b.base_exp + (int)code[u]) & 0xFFu) << 7 | (h & 0x7Fu) : h;
                if (kb0 + u < (uint32_t)b.k_blocks) out[ZS_BT_DIM * u] = bf16_bits(bf16_value(bits) * scale);
            }
        }
    }
}

// ---- rows of a BF16 table ------------------------------------------------------------------
// A thread takes eight columns of one token.  Bound by memory: 16384 tokens of 128256 x 4096 take 48 us (268 MB both ways, 5.6 TB/s).
__global__ __launch_bounds__(256) void dense_embed_kernel(const uint16_t *W, int64_t N, int64_t K, int64_t ldw, const void *ids, int id_bytes,
                                                          int64_t units, int64_t row_units, float scale, uint16_t *Y, int64_t ldy)
{
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < units; u += (int64_t)gridDim.x * 256) {
        const int64_t t = u / row_units, c = 8 * (u - t * row_units), left = K - c;
        const int64_t id = id_at(ids, id_bytes, t, N);
        const Values<uint16_t, 8> v = id >= 0 ? fetch<8>(W + id * ldw + c, left) : Values<uint16_t, 8>{};
        uint16_t *const out = Y + t * ldy + c;
        const float s = id >= 0 ? scale : 0.f;
        if (left >= 8) {
            store_any(out, u32x4{bf16_pair(v[0] * s, v[1] * s), bf16_pair(v[2] * s, v[3] * s), bf16_pair(v[4] * s, v[5] * s),
                                 bf16_pair(v[6] * s, v[7] * s)});
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) out[i] = bf16_bits(v[i] * s);
        }
    }
}

int check_lookup(const void *ids, int id_bytes, int64_t T, const void *Y, int64_t ldy, int64_t K)
{
    if (id_bytes != 4 && id_bytes != 8) return ZS_ERR_CONFIG;
    if (T < 0 || T > INT32_MAX || ldy < K) return ZS_ERR_SHAPE;
    if (T > 0 && (!ids || !Y || !aligned(ids, id_bytes) || !aligned(Y, 2))) return ZS_ERR_ARG;
    return ZS_OK;
}

// ---- gradient of the table -------------------------------------------------------------------
// The (id, position) pairs of the tokens are sorted, so that a row's tokens lie next to each other in the order
// of the batch.  The sorted list is cut into chunks of equal length, however often a token occurs; a wave sums
// a chunk's rows of dY over a slice of the columns.  A run of one id that lies inside a chunk is finished
// there; one that crosses a boundary leaves a partial sum for each chunk in the workspace, and these are added in order.
// Every sum has one fixed order: the result is the same from run to run.
constexpr int kTile = 1024; // pairs sorted by one workgroup, a thread each
constexpr int kFan = 16;    // sorted lists merged at a time
constexpr uint32_t kNoRow = 0x7FFFFFFFu; // (a table has fewer rows)

typedef uint64_t Pair; // id << 32 | position: all different, so that a pair's place is a count of smaller ones

typedef f32x4 __attribute__((aligned(4))) f32x4_any;

// Zeros for `rows` rows of `cols` elements (a dW without gaps is one row), by `wgs` workgroups of which this is `wg`.
// Non-temporal: the sums behind it do not wait for 256 MB of dirty lines (128256 x 4096: 77 -> 52 us).
struct Zeros {
    float *p;
    int64_t rows, cols, ld;
};
// A workgroup has a store of 16 bytes for each thread: a part of a row, or several short rows side by side.  With stores in a loop
// 2 GB take 440 to 570 us (1024 to 8192 workgroups of 256 threads) instead of 300.
struct Clearing {
    int64_t units, across, side, wgs; // stores to a row, workgroups across a row, rows side by side, workgroups for everything
};
__host__ __device__ __forceinline__ Clearing clearing(const Zeros &z, int threads)
{
    Clearing c;
    c.units = (z.cols + 3) / 4;
    c.across = (c.units + threads - 1) / threads;
    c.side = z.rows > 1 && c.units < threads ? threads / c.units : 1;
    c.wgs = c.side > 1 ? (z.rows + c.side - 1) / c.side : z.rows * c.across;
    return c;
}
template <int THREADS>
__device__ __forceinline__ void clear(const Zeros &z, int64_t wg, int64_t wgs)
{
    const Clearing plan = clearing(z, THREADS);
    uint32_t at = threadIdx.x, beside = 0;
    if (plan.side > 1) {
        beside = at / (uint32_t)plan.units;
        at -= beside * (uint32_t)plan.units;
        if (beside >= plan.side) return;
    }
    for (; wg < plan.wgs; wg += wgs) {
        const int64_t row = z.rows == 1 ? 0 : plan.across == 1 ? wg * plan.side + beside : wg / plan.across;
        const int64_t u = plan.across == 1 ? at : at + (wg - row * plan.across) * THREADS;
        if (row >= z.rows || u >= plan.units) continue;
        float *q = z.p + row * z.ld + 4 * u;
        if (4 * u + 4 <= z.cols) __builtin_nontemporal_store(f32x4{0.f, 0.f, 0.f, 0.f}, reinterpret_cast<f32x4_any *>(q));
        else
            for (int64_t i = 0; i < z.cols - 4 * u; ++i) q[i] = 0.f;
    }
}

// Up to kCounted pairs: a pair's place is the number of smaller ones.  Sixteen lanes to a pair, which compare it with four ids each at
// a time, in the first `wgs` workgroups; the others clear dW meanwhile.  Bound by latency for few pairs, then by the T^2 comparisons.  Whole calls with
// 1024 BF16 columns added to dW, counted against sorted and merged, us: 64 tokens 9.5 and 13.8, 2048 17 and 23, 4096 28 and 30, 6000 33 and 32.
constexpr int kCounted = 4096;
__global__ __launch_bounds__(256) void count_kernel(const void *ids, int id_bytes, int T, int64_t N, Pair *out, int wgs, Zeros z)
{
    extern __shared__ __attribute__((aligned(16))) uint32_t keys[];
    if ((int)blockIdx.x >= wgs) {
        clear<256>(z, blockIdx.x - wgs, gridDim.x - wgs);
        return;
    }
    const int blocks = (T + 63) / 64, tid = threadIdx.x, lane = tid % kFan;
    for (int i = tid; i < 64 * blocks; i += 256) {
        uint32_t key = ~0u; // behind the last: larger than any
        if (i < T) {
            const int64_t id = id_at(ids, id_bytes, i, N);
            key = id < 0 ? kNoRow : (uint32_t)id;
        }
        keys[i] = key;
    }
    __syncthreads();
    const int t = blockIdx.x * (256 / kFan) + tid / kFan, own = blockIdx.x * (256 / kFan) / 64; // the block of 64 ids with this workgroup's pairs
    const uint32_t mine = keys[t];
    int smaller = 0;
    auto ids_of = [&](int b) { return *reinterpret_cast<const u32x4 *>(keys + 64 * b + 4 * lane); };
#pragma unroll 4
    for (int b = 0; b < own; ++b) { // earlier positions
        const u32x4 v = ids_of(b);
#pragma unroll
        for (int e = 0; e < 4; ++e) smaller += v[e] <= mine;
    }
    const u32x4 v = ids_of(own);
#pragma unroll
    for (int e = 0; e < 4; ++e) smaller += v[e] < mine + (64 * own + 4 * lane + e < t);
#pragma unroll 4
    for (int b = own + 1; b < blocks; ++b) {
        const u32x4 w = ids_of(b);
#pragma unroll
        for (int e = 0; e < 4; ++e) smaller += w[e] < mine;
    }
    for (int d = 1; d < kFan; d *= 2) smaller += __shfl_xor(smaller, d);
    if (lane == 0 && t < T) out[smaller] = (Pair)mine << 32 | (uint32_t)t;
}

// The value of the lane whose number differs in bit d (a constant): within a row of sixteen lanes by moves of the
// vector unit where it has one, else through the LDS crossbar.
__device__ __forceinline__ uint32_t partner(uint32_t x, int d)
{
    switch (d) {
    case 1: return __builtin_amdgcn_update_dpp(0u, x, 0xB1, 0xf, 0xf, false);  // quad_perm 1, 0, 3, 2
    case 2: return __builtin_amdgcn_update_dpp(0u, x, 0x4E, 0xf, 0xf, false);  // quad_perm 2, 3, 0, 1
    case 4: return (uint32_t)__builtin_amdgcn_ds_swizzle((int)x, 0x101F);      // xor 4
    case 8: return __builtin_amdgcn_update_dpp(0u, x, 0x128, 0xf, 0xf, false); // row_ror:8
    case 16: return (uint32_t)__builtin_amdgcn_ds_swizzle((int)x, 0x401F);     // xor 16
    default: return (uint32_t)__shfl_xor((int)x, 32);
    }
}

// Sorts kTile pairs in each of the first `tiles` workgroups; the others clear their part of dW meanwhile.  The sorting is bound by
// the latency of the network's 55 steps, ten of them through LDS (7.5 us).
__global__ __launch_bounds__(kTile) void sort_tiles_kernel(const void *ids, int id_bytes, int64_t T, int64_t N, Pair *out, int tiles, Zeros z)
{
    __shared__ Pair keys[kTile];
    const int tid = threadIdx.x;
    if ((int)blockIdx.x >= tiles) {
        clear<kTile>(z, blockIdx.x - tiles, gridDim.x - tiles);
        return;
    }
    const int64_t t = (int64_t)blockIdx.x * kTile + tid;
    Pair mine = ~0ull;
    if (t < T) {
        const int64_t id = id_at(ids, id_bytes, t, N);
        mine = (Pair)(id < 0 ? kNoRow : (uint32_t)id) << 32 | (uint32_t)t;
    }
    // bitonic sorting network: partners less than a wave apart meet in registers, the others in LDS
#pragma unroll
    for (int size = 2; size <= kTile; size *= 2)
#pragma unroll
        for (int d = size / 2; d > 0; d /= 2) {
            Pair other;
            if (d < 64) {
                other = (Pair)partner((uint32_t)(mine >> 32), d) << 32 | partner((uint32_t)mine, d);
            } else {
                keys[tid] = mine;
                __syncthreads();
                other = keys[tid ^ d];
                __syncthreads();
            }
            const bool low = (tid & d) == 0, up = (tid & size) == 0;
            mine = (low == up) ? min(mine, other) : max(mine, other);
        }
    if (t < T) out[t] = mine;
}

// Sorted lists of `run` pairs (a power of two) become lists of run * kFan: a pair's place is its own index plus the
// number of smaller pairs in each of the other lists of its group.  Sixteen lanes to a pair, each searches one list.
// (One lane to a pair, which searched all lists, kept few waves busy for long: 43 us for 15920 pairs, and the call 72 instead of 40.)
__device__ __forceinline__ void merge(const Pair *in, Pair *out, int64_t T, int64_t run, int64_t t, int lane)
{
    const Pair mine = in[t];
    const int64_t group = t / (run * kFan) * (run * kFan), list = group + lane * run;
    int64_t smaller = 0;
    for (int64_t step = run; step > 0; step /= 2) {
        const int64_t to = list + smaller + step;
        if (smaller + step <= run && to <= T && in[to - 1] < mine) smaller += step;
    }
    for (int d = 1; d < kFan; d *= 2) smaller += __shfl_xor((long long)smaller, d);
    if (lane == 0) out[group + smaller] = mine;
}

// Merges in the first `wgs` workgroups; the others clear their part of dW meanwhile.
__global__ __launch_bounds__(256) void merge_kernel(const Pair *in, Pair *out, int64_t T, int64_t run, int wgs, Zeros z)
{
    if ((int)blockIdx.x >= wgs) {
        clear<256>(z, blockIdx.x - wgs, gridDim.x - wgs);
        return;
    }
    for (int64_t t = (int64_t)blockIdx.x * (256 / kFan) + threadIdx.x / kFan; t < T; t += (int64_t)wgs * (256 / kFan))
        merge(in, out, T, run, t, threadIdx.x % kFan);
}

struct Runs {
    const Pair *pairs; // sorted
    int64_t T, K, slices, chunks;
    int chunk;
    float *heads, *tails; // [chunks, K]: sums of a run that began before the chunk / that goes on behind it
    __device__ uint32_t id(int64_t i) const { return (uint32_t)(pairs[i] >> 32); }
    __device__ uint32_t id_before(int64_t chunk_at) const { return chunk_at == 0 ? kNoRow : id(chunk_at - 1); }
    __device__ uint32_t id_behind(int64_t end) const { return end >= T ? kNoRow : id(end); }
};

constexpr int kCols = 4; // columns of a lane: a wave's sums are whole lines

__device__ __forceinline__ void put(float *p, f32x4 v, int64_t left, float scale, bool add)
{
    if (left >= kCols) {
        f32x4 a = {v[0] * scale, v[1] * scale, v[2] * scale, v[3] * scale};
        if (add) a += load_any<f32x4>(p);
        store_any(p, a);
        return;
    }
#pragma unroll
    for (int i = 0; i < kCols; ++i)
        if (i < left) p[i] = add ? p[i] + v[i] * scale : v[i] * scale;
}

// Sums of a chunk.  Bound by memory with many tokens: 16384 of 4096 BF16 columns take 53 us (134 MB read, a row of dW written for each id); by the
// latency of one round of loads with few (509 tokens of 1024 columns: 4 us).
template <typename T>
__global__ __launch_bounds__(64) void sum_kernel(Runs g, const T *dY, int64_t lddy, float scale, float *dW, int64_t ldw, int add)
{
    constexpr int kAhead = 16; // rows of dY requested at a time
    for (int64_t task = blockIdx.x; task < g.chunks * g.slices; task += gridDim.x) {
        const int64_t chunk = task / g.slices, c = ((task - chunk * g.slices) * 64 + threadIdx.x) * kCols, left = g.K - c;
        const int64_t begin = chunk * g.chunk;
        const int size = (int)min((int64_t)g.chunk, g.T - begin);
        // the chunk's pairs, one to a lane, and the ids on both sides; tokens without a row are the last ones
        const Pair mine = g.pairs[begin + min((int)threadIdx.x, size - 1)];
        const uint32_t before = g.id_before(begin), behind = g.id_behind(begin + size);
        const int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64((int)threadIdx.x < size && (uint32_t)(mine >> 32) != kNoRow));
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        for (int i0 = 0; i0 < n; i0 += kAhead) {
            Values<T, kCols> v[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int64_t t = (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)mine, min(i0 + i, n - 1));
                v[i] = fetch<kCols>(dY + t * lddy + c, left);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int at = i0 + i;
                if (at >= n) break;
                const uint32_t id = (uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), at);
#pragma unroll
                for (int j = 0; j < kCols; ++j) acc[j] += v[i][j];
                const uint32_t next = at + 1 < n ? (uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), at + 1) : behind;
                if (at + 1 < n && next == id) continue;
                // the run's sum over this chunk
                if (id == before) put(g.heads + chunk * g.K + c, acc, left, 1.f, false);
                else if (id == next) put(g.tails + chunk * g.K + c, acc, left, 1.f, false);
                else put(dW + (int64_t)id * ldw + c, acc, left, scale, add);
                acc = f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
    }
}

// Runs over several chunks: what the chunks behind its first one left is added up in their order.  A wave takes the run
// that begins in one chunk, if any does; a workgroup has the runs of eight neighbouring chunks, of which one at most is
// longer than sixteen, and its waves share that one: each adds sixteen chunks in turn, then the waves are added in order.
// (A wave by itself for each run: 112 instead of 78 us for a call with 16384 tokens of one id, K = 4096, and the same for others.)
constexpr int kJoinWaves = 8, kJoinAhead = 16;

__device__ __forceinline__ void add_heads(f32x4 &acc, const Runs &g, int64_t from, int n, int64_t c, int64_t left)
{
    Values<float, kCols> v[kJoinAhead];
#pragma unroll
    for (int i = 0; i < kJoinAhead; ++i) v[i] = fetch<kCols>(g.heads + (from + min(i, n - 1)) * g.K + c, left);
#pragma unroll
    for (int i = 0; i < kJoinAhead; ++i)
        if (i < n)
#pragma unroll
            for (int j = 0; j < kCols; ++j) acc[j] += v[i][j];
}

__global__ __launch_bounds__(64 * kJoinWaves) void join_kernel(Runs g, float scale, float *dW, int64_t ldw, int add)
{
    __shared__ f32x4 sums[kJoinWaves][64];
    __shared__ int shared_run; // the wave that found the run for all of them
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int64_t groups = (g.chunks - 1 + kJoinWaves - 1) / kJoinWaves;
    for (int64_t task = blockIdx.x; task < groups * g.slices; task += gridDim.x) {
        const int64_t group = task / g.slices, first = group * kJoinWaves, c = ((task - group * g.slices) * 64 + lane) * kCols, left = g.K - c;
        auto tail = [&](int64_t chunk) {
            const Values<float, kCols> v = fetch<kCols>(g.tails + chunk * g.K + c, left);
            return f32x4{v[0], v[1], v[2], v[3]};
        };
        auto inside = [&](int64_t k, uint32_t id) { // of the chunks from k on, how many begin inside the run (up to kJoinAhead + 1)
            const uint64_t begin = __builtin_amdgcn_ballot_w64(lane <= kJoinAhead && k + lane < g.chunks && g.id(min(k + lane, g.chunks - 1) * g.chunk) == id);
            return (int)__builtin_ctzll(~begin);
        };
        if (threadIdx.x == 0) shared_run = -1;
        __syncthreads();
        const int64_t chunk = first + wave;
        if (chunk + 1 < g.chunks) {
            const int64_t begin = chunk * g.chunk, end = begin + g.chunk;
            const uint32_t id = g.id(end - 1);
            if (id != kNoRow && id == g.id(end) && id != g.id_before(begin)) {
                const int n = inside(chunk + 1, id);
                if (n > kJoinAhead) {
                    if (lane == 0) shared_run = wave;
                } else {
                    f32x4 acc = tail(chunk);
                    add_heads(acc, g, chunk + 1, n, c, left);
                    put(dW + (int64_t)id * ldw + c, acc, left, scale, add);
                }
            }
        }
        __syncthreads();
        const int run = __builtin_amdgcn_readfirstlane(shared_run);
        if (run < 0) continue;
        const uint32_t id = g.id((first + run + 1) * g.chunk - 1);
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        if (wave == 0) acc = tail(first + run);
        for (int64_t k = first + run + 1 + kJoinAhead * wave;; k += kJoinAhead * kJoinWaves) {
            const int n = min(inside(k, id), kJoinAhead);
            if (n > 0) add_heads(acc, g, k, n, c, left);
            if (n < kJoinAhead) break;
        }
        sums[wave][lane] = acc;
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int w = 1; w < kJoinWaves; ++w) acc += sums[w][lane];
            put(dW + (int64_t)id * ldw + c, acc, left, scale, add);
        }
        __syncthreads();
    }
}

struct GradPlan {
    int chunk; // tokens
    int64_t chunks, slices;
    size_t pairs_bytes, sums_bytes, total;
};
GradPlan plan_grad(int64_t T, int64_t K)
{
    GradPlan p;
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    p.slices = ceil_div(K, 64 * kCols);
    // Small chunks make more waves, and more partial sums.  With 8, 16 and 32 tokens, us: 256 tokens x 4096 columns 14, 16, 22;
    // 512 17, 19, 25; 4096 55, 54, 58; 16384 137, 127, 121 (frequent ids) or 102, 84, 78 (one id).
    p.chunk = T * K <= 1 << 21 ? 8 : T * K < 1 << 25 ? 16 : 32;
    p.chunks = ceil_div(T, p.chunk);
    p.pairs_bytes = up(8 * (size_t)T);
    p.sums_bytes = up(4 * (size_t)p.chunks * (size_t)K);
    p.total = 2 * p.pairs_bytes + 2 * p.sums_bytes;
    return p;
}

bool grad_shape_ok(int64_t T, int64_t N, int64_t K)
{
    return T >= 0 && T <= INT32_MAX && N >= 1 && N <= INT32_MAX && K >= 1 && K <= INT32_MAX;
}

} // namespace

extern "C" int zs_embed(const zs_desc *d, const void *blob_dev, const void *ids_dev, int id_bytes, int64_t T, float scale, uint16_t *Y_dev,
                        int64_t ldy, void *hip_stream)
{
    if (!d) return ZS_ERR_ARG;
    int rc = zs_desc_validate(d);
    if (rc != ZS_OK) return rc;
    if (!blob_dev || !aligned(blob_dev, ZS_SECTION_ALIGN)) return ZS_ERR_ARG;
    if ((rc = check_lookup(ids_dev, id_bytes, T, Y_dev, ldy, d->K)) != ZS_OK || T == 0) return rc;
    const uint8_t *base = static_cast<const uint8_t *>(blob_dev);
    Blob b;
    b.bitmaps = base + d->off_bitmaps;
    b.offsets = reinterpret_cast<const u32x2 *>(base + d->off_offsets);
    b.H = d->h_bytes ? base + d->off_H : base; // (an empty section may lie at the blob's end)
    b.L = d->l_bytes ? base + d->off_L : base;
    b.h_last = d->h_bytes ? d->h_bytes - 1 : 0;
    b.l_last = d->l_bytes ? d->l_bytes - 2 : 0;
    b.base_exp = d->base_exp;
    b.k_blocks = (int32_t)(d->K / ZS_BT_DIM);
    // Four BlockTiles to a wave, or one while that leaves fewer than 8192 waves.  K = 4096, one against four, us: 32 tokens 2.9
    // and 3.9, 256 8.8 and 9.2, 512 14.9 and 14.5, 2048 45 and 43; 5000 of which many are cached 106 and 81, 8192 of which few are 144 and 157.
    const int u = T * b.k_blocks >= 4 * 8192 ? 4 : 1;
    const dim3 grid(grid_for(T), (unsigned)std::min(ceil_div(b.k_blocks, 4 * u), (int64_t)1024));
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (u == 4) hipLaunchKernelGGL(embed_kernel<4>, grid, dim3(256), 0, s, b, d->N, ids_dev, id_bytes, T, scale, Y_dev, ldy);
    else hipLaunchKernelGGL(embed_kernel<1>, grid, dim3(256), 0, s, b, d->N, ids_dev, id_bytes, T, scale, Y_dev, ldy);
    return launched();
}

extern "C" int zs_dense_embed(const uint16_t *W_dev, int64_t N, int64_t K, int64_t ldw, const void *ids_dev, int id_bytes, int64_t T,
                              float scale, uint16_t *Y_dev, int64_t ldy, void *hip_stream)
{
    if (!W_dev || !aligned(W_dev, 2)) return ZS_ERR_ARG;
    if (N < 1 || K < 1 || N > INT32_MAX || K > INT32_MAX || ldw < K) return ZS_ERR_SHAPE;
    const int rc = check_lookup(ids_dev, id_bytes, T, Y_dev, ldy, K);
    if (rc != ZS_OK || T == 0) return rc;
    const int64_t row_units = ceil_div(K, 8), units = T * row_units;
    hipLaunchKernelGGL(dense_embed_kernel, dim3(grid_for(ceil_div(units, 256))), dim3(256), 0, static_cast<hipStream_t>(hip_stream), W_dev, N, K,
                       ldw, ids_dev, id_bytes, units, row_units, scale, Y_dev, ldy);
    return launched();
}

extern "C" size_t zs_embed_grad_workspace(int64_t T, int64_t N, int64_t K)
{
    return grad_shape_ok(T, N, K) ? plan_grad(T, K).total : 0;
}

extern "C" int zs_embed_grad(const void *ids_dev, int id_bytes, int64_t T, const void *dY_dev, int dy_type, int64_t lddy, float scale,
                             float *dW_dev, int64_t N, int64_t K, int64_t lddw, int accumulate, void *workspace_dev, size_t workspace_bytes,
                             void *hip_stream)
{
    if (id_bytes != 4 && id_bytes != 8) return ZS_ERR_CONFIG;
    if (dy_type != ZS_TYPE_BF16 && dy_type != ZS_TYPE_F32) return ZS_ERR_CONFIG;
    if (!grad_shape_ok(T, N, K) || lddy < K || lddw < K) return ZS_ERR_SHAPE;
    if (!dW_dev || !aligned(dW_dev, 4)) return ZS_ERR_ARG;
    if (T > 0 && (!ids_dev || !dY_dev || !workspace_dev || !aligned(ids_dev, id_bytes) || !aligned(dY_dev, dy_type == ZS_TYPE_BF16 ? 2 : 4) ||
                  !aligned(workspace_dev, 256)))
        return ZS_ERR_ARG;
    const GradPlan plan = plan_grad(T, K);
    if (workspace_bytes < plan.total) return ZS_ERR_SIZE;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    // dW is cleared by workgroups beside those that count or sort.  Where there is a merge most of it goes there, and beside the sorting what that
    // hides: 128256 x 4096 with nothing, 2^22, 2^24, 2^26 elements and half of it there takes 378, 376, 372, 378, 388 us (whole lines: a
    // part that begins inside one costs 120 us more).
    constexpr int64_t kBesideSort = 1 << 24;
    const bool whole = lddw == K, counted = T <= kCounted;
    const int64_t rows = accumulate ? 0 : whole ? 1 : N, cols = whole ? N * K : K;
    Zeros first = {dW_dev, rows, cols, lddw}, second = {dW_dev, 0, cols, lddw};
    if (!counted && rows == 1) {
        first.cols = std::min(cols / 2, kBesideSort) / 1024 * 1024;
        second = {dW_dev + first.cols, 1, cols - first.cols, lddw};
    } else if (!counted) {
        first.rows = std::min(rows / 2, kBesideSort / K);
        second = {dW_dev + first.rows * lddw, rows - first.rows, cols, lddw};
    }
    const Zeros none = {dW_dev, 0, cols, lddw};
    auto with = [](int64_t wgs, const Zeros &z, int threads) { return dim3((unsigned)wgs + grid_for(clearing(z, threads).wgs, (1 << 28) / threads)); };
    uint8_t *ws = static_cast<uint8_t *>(workspace_dev);
    Pair *from = reinterpret_cast<Pair *>(ws), *to = reinterpret_cast<Pair *>(ws + plan.pairs_bytes);
    if (counted) {
        const int wgs = (int)ceil_div(T, 256 / kFan);
        if (T > 0 || rows > 0)
            hipLaunchKernelGGL(count_kernel, with(wgs, first, 256), dim3(256), 4 * 64 * ceil_div(T, 64), s, ids_dev, id_bytes, (int)T, N, from, wgs, first);
    } else {
        const int tiles = (int)ceil_div(T, kTile);
        hipLaunchKernelGGL(sort_tiles_kernel, with(tiles, first, kTile), dim3(kTile), 0, s, ids_dev, id_bytes, T, N, from, tiles, first);
        for (int64_t run = kTile; run < T; run *= kFan) {
            const Zeros &z = run == kTile ? second : none;
            const int wgs = (int)grid_for(ceil_div(T, 256 / kFan));
            hipLaunchKernelGGL(merge_kernel, with(wgs, z, 256), dim3(256), 0, s, from, to, T, run, wgs, z);
            Pair *const swap = from;
            from = to;
            to = swap;
        }
    }
    if (T == 0) return launched();
    Runs g;
    g.pairs = from;
    g.T = T;
    g.K = K;
    g.slices = plan.slices;
    g.chunks = plan.chunks;
    g.chunk = plan.chunk;
    g.heads = reinterpret_cast<float *>(ws + 2 * plan.pairs_bytes);
    g.tails = reinterpret_cast<float *>(ws + 2 * plan.pairs_bytes + plan.sums_bytes);
    const dim3 grid(grid_for(g.chunks * g.slices));
    if (dy_type == ZS_TYPE_BF16)
        hipLaunchKernelGGL(sum_kernel<uint16_t>, grid, dim3(64), 0, s, g, static_cast<const uint16_t *>(dY_dev), lddy, scale, dW_dev, lddw, accumulate);
    else
        hipLaunchKernelGGL(sum_kernel<float>, grid, dim3(64), 0, s, g, static_cast<const float *>(dY_dev), lddy, scale, dW_dev, lddw, accumulate);
    if (g.chunks > 1) hipLaunchKernelGGL(join_kernel, dim3(grid_for(ceil_div(g.chunks - 1, kJoinWaves) * g.slices)), dim3(64 * kJoinWaves), 0, s, g, scale, dW_dev, lddw, accumulate);
    return launched();
}
