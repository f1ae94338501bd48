// The tiles that the worker's matrix products are made of: R = P Q^T summed over k, P with a row for each row of the result, Q with a
// row for each column of it.  An operand lies in memory by rows (its k adjacent) or by k (its rows adjacent: a transposed matrix).
//
// A block makes a tile of the result.  Tiles of the operands go through LDS as rows of 128 bytes of k (64 16-bit values, 32 floats), in
// eight chunks of 16 bytes; chunk c of row r lies at place c ^ (r & 7), so that eight lanes that read one chunk of eight rows meet all banks.
//
// The matrix instructions take Q as their first operand: a lane then holds four neighbouring columns of one row of the result, 8 or 16 bytes that
// it loads and stores at once.  For floats a lane reads a chunk of four k and feeds them to four instructions; which k stand together
// in one does not matter as long as both operands agree.
#pragma once
#include "../../include/dblp_layers.h"
#include "worker_common.h"

typedef float f4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// The sum over the 16 bytes of k that each of the four groups of 16 lanes holds of 16 rows of Q (a) and of P (b).
template <class T> __device__ __forceinline__ f4 mfma(u4v a, u4v b, f4 c);
template <> __device__ __forceinline__ f4 mfma<BF16>(u4v a, u4v b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f4 mfma<F16>(u4v a, u4v b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f4 mfma<F32>(u4v a, u4v b, f4 c) {
    const f4 x = __builtin_bit_cast(f4, a), y = __builtin_bit_cast(f4, b);
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
    return c;
}
// 16 bytes of ones: a product with them is a sum over k.
template <class T> __device__ __forceinline__ u4v ones();
template <> __device__ __forceinline__ u4v ones<BF16>() { return (u4v)(0x3F803F80u); }
template <> __device__ __forceinline__ u4v ones<F16>() { return (u4v)(0x3C003C00u); }
template <> __device__ __forceinline__ u4v ones<F32>() { return (u4v)(0x3F800000u); }

// One operand of a batch of products: element (row, k) at row * stride + k, or at k * stride + row where it lies by k.
struct Operand { const void* p; u64 stride, step; };

// What a launch computes: rows x cols results of sums over `depth` k, of which block z takes part z % parts of matrix z / parts.
struct Product {
    Operand P, Q;
    u32 rows, cols, depth, tile_cols, part, parts;   // part: k of one part, a multiple of 64; tile_cols: tiles of a row of tiles
    u64 tile0;                                       // first tile of this launch
};

#define TILE_THREADS 256

// A tile of BT rows and 128 bytes of k in registers, chunk by chunk, on its way to LDS.
template <class T, int BT, bool BY_K>
struct Staged {
    typedef typename T::elem elem;
    static constexpr int E = 16 / sizeof(elem), N = BT * 8 / TILE_THREADS;        // elements of a chunk, chunks of a thread
    typedef Vec<T, E> V;
    u4v v[N];

    // BY_K: a chunk is E neighbouring rows of one k; otherwise E neighbouring k of one row.  Rows past the end are any row's, k past it zeros.
    __device__ __forceinline__ void load(const elem* p, u64 stride, u32 row0, u32 rows, u32 k0, u32 depth) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const u32 q = threadIdx.x + i * TILE_THREADS;
            if (BY_K) {
                const u32 k = k0 + q / (BT / E), r = row0 + q % (BT / E) * E;
                v[i] = (u4v)(0u);
                if (k < depth && r < rows) {
                    const elem* at = p + (u64)k * stride + r;
                    v[i] = __builtin_bit_cast(u4v, r + E <= rows ? V::load(at) : V::some(at, rows - r));
                }
            } else {
                const u32 r = row0 + q / 8 < rows ? row0 + q / 8 : rows - 1, k = k0 + q % 8 * E;
                v[i] = (u4v)(0u);
                if (k < depth) {
                    const elem* at = p + (u64)r * stride + k;
                    v[i] = __builtin_bit_cast(u4v, k + E <= depth ? V::load(at) : V::some(at, depth - k));
                }
            }
        }
    }
    __device__ __forceinline__ void store(uint8_t* tile) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const u32 q = threadIdx.x + i * TILE_THREADS;
            if (BY_K) {
                const u32 k = q / (BT / E), r = q % (BT / E) * E;
                typedef elem chunk __attribute__((ext_vector_type(E)));
                const chunk c = __builtin_bit_cast(chunk, v[i]);
#pragma unroll
                for (int e = 0; e < E; ++e) *(elem*)(tile + (r + e) * 128 + ((k / E) ^ ((r + e) & 7)) * 16 + k % E * sizeof(elem)) = c[e];
            } else {
                const u32 r = q / 8, c = q % 8;
                *(u4v*)(tile + r * 128 + (c ^ (r & 7)) * 16) = v[i];
            }
        }
    }
};

__device__ __forceinline__ u4v chunk_of(const uint8_t* tile, u32 row, u32 chunk) { return *(const u4v*)(tile + row * 128 + (chunk ^ (row & 7)) * 16); }

// Four waves, two by two, each a quarter of a BM x BN tile.  SUMS: of the first column of tiles, also P's own sums over k.  `out` gets the results, four columns of
// a row at a time; `sums` a row's sum.
template <class T, bool P_BY_K, bool Q_BY_K, int BM, int BN, bool SUMS, class Out>
__global__ __launch_bounds__(TILE_THREADS) void tile_products(Product a, Out out) {
    typedef typename T::elem elem;
    constexpr u32 STEP = 128 / sizeof(elem);
    constexpr int NM = BM / 32, NN = BN / 32;
    __shared__ __attribute__((aligned(16))) uint8_t tiles[2][(BM + BN) * 128];
    const u64 tile = a.tile0 + blockIdx.x;
    const u32 m0 = (u32)(tile / a.tile_cols) * BM, n0 = (u32)(tile % a.tile_cols) * BN;
    const u32 matrix = blockIdx.z / a.parts, part = blockIdx.z % a.parts;
    const elem* const p = (const elem*)a.P.p + matrix * a.P.step;
    const elem* const q = (const elem*)a.Q.p + matrix * a.Q.step;
    const u32 lane = threadIdx.x & 63, wave = threadIdx.x >> 6, group = lane >> 4, in_group = lane & 15;
    const u32 wm = (wave >> 1) * (BM / 2), wn = (wave & 1) * (BN / 2);
    const u32 k_first = part * a.part, k_end = a.depth - k_first > a.part ? k_first + a.part : a.depth;
    const bool summing = SUMS && n0 == 0 && wn == 0;
    f4 acc[NM][NN] = {}, sum[NM] = {};
    Staged<T, BM, P_BY_K> sp;
    Staged<T, BN, Q_BY_K> sq;
    const auto load = [&](u32 k) { sp.load(p, a.P.stride, m0, a.rows, k, k_end); sq.load(q, a.Q.stride, n0, a.cols, k, k_end); };
    const auto store = [&](u32 at) { sp.store(tiles[at]); sq.store(tiles[at] + BM * 128); };
    if (k_first < k_end) {
        load(k_first);
        store(0);
    }
    u32 at = 0;
    for (u32 k = k_first; k < k_end; k += STEP, at ^= 1) {
        const bool more = k_end - k > STEP;
        if (more) load(k + STEP);
        __syncthreads();
        const uint8_t *const tp = tiles[at], *const tq = tiles[at] + BM * 128;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            u4v b[NM];
#pragma unroll
            for (int i = 0; i < NM; ++i) b[i] = chunk_of(tp, wm + i * 16 + in_group, kk * 4 + group);
#pragma unroll
            for (int j = 0; j < NN; ++j) {
                const u4v c = chunk_of(tq, wn + j * 16 + in_group, kk * 4 + group);
#pragma unroll
                for (int i = 0; i < NM; ++i) acc[i][j] = mfma<T>(c, b[i], acc[i][j]);
            }
            if (SUMS && summing)
#pragma unroll
                for (int i = 0; i < NM; ++i) sum[i] = mfma<T>(ones<T>(), b[i], sum[i]);
        }
        if (more) store(at ^ 1);
    }
#pragma unroll
    for (int i = 0; i < NM; ++i) {
        const u32 m = m0 + wm + i * 16 + in_group;
        if (m >= a.rows) continue;
        if (SUMS && summing && group == 0) out.sums(matrix, part, m, sum[i][0]);
#pragma unroll
        for (int j = 0; j < NN; ++j) {
            const u32 n = n0 + wn + j * 16 + group * 4;
            if (n < a.cols) out.put(matrix, part, m, n, a.cols, acc[i][j]);
        }
    }
}

// Columns [n, n + 4) of a row, as floats.
template <class T>
__device__ __forceinline__ void get4(const typename T::elem* row, u32 n, u32 cols, float (&v)[4]) {
    typedef Vec<T, 4> V;
    V::open(n + 4 <= cols ? V::load(row + n) : V::some(row + n, cols - n), v);
}

// Launches of a product's tiles: at most 2^20 tiles and 2^15 matrices' parts each (a grid's threads stay below 2^32, its z below 2^16).  Rows
// have a tile even where there is no column: for their own sums.
template <int BM, int BN, class F>
static void each_tiles(u32 rows, u32 cols, u32 parts, u64 matrices, F f) {
    const u64 tile_cols = cols ? (cols + (u64)BN - 1) / BN : 1, tiles = (rows + (u64)BM - 1) / BM * tile_cols;
    for (u64 m = 0; m < matrices; m += 32768 / parts) {
        const u64 here = matrices - m < 32768 / parts ? matrices - m : 32768 / parts;
        for (u64 t = 0; t < tiles; t += 1u << 20)
            f(t, (u32)tile_cols, dim3((u32)(tiles - t < (1u << 20) ? tiles - t : 1u << 20), 1, (u32)here * parts), m);
    }
}
