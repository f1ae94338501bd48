// Rows of a worker's training step on gfx950 (MI355X): dropout, the embedding and its gradient.
// Kernels and the C-ABI declared in include/dblp_worker.h.
//
// All of it is bound by memory: a few operations on each value, read once and written once.  Lanes that follow each other
// hold 16 neighbouring bytes each (8 where a 16-bit matrix meets a float one), and several rows of a thread are in flight.
#include "worker_common.h"

// ------------------------------------------------------------------------------------------
// dropout and embedding
// ------------------------------------------------------------------------------------------
// Units that a thread has in flight.  Dropout: one is fastest (8192 x 768 with a residual 7.4 us, 9.1 with two); four columns take two, whose gates
// lanes share.  Embedding: two, the row's address being a load itself (32768 x 4096 77 us, 84 with one, 95 with four).
template <int W> struct InFlight { static constexpr int N = W == 4 ? 2 : 1; };
#define EMBED_EACH 2
#define FAR_BYTES (256ull << 20)  // matrices that the memory-side cache does not hold are read and written past it

// The gates of a thread's units i, i + 256, ..., as words for `shut`.
template <int W, int N>
__device__ __forceinline__ void gates_of_units(const Mask& m, u64 draw, u64 unit0, u32 (&gate)[N][W / 2]) {
    if constexpr (W == 4) {
#pragma unroll
        for (int j = 0; j < N; j += 2) gates_of_two(m, draw, (unit0 + j * 256) / 2, (unit0 + j * 256 + 256) / 2, gate[j], gate[j + 1]);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const Gates g = gates_of(m, draw, unit0 + j * 256);
#pragma unroll
            for (int k = 0; k < 4; ++k) gate[j][k] = g.w[k];
        }
    }
}

template <class T, int W, bool RES, bool WHOLE, bool FAR>
__global__ __launch_bounds__(256) void dropout_units(Units s, Mask m, const typename T::elem* x, u64 x_stride,
                                                     const typename T::elem* res, u64 res_stride, typename T::elem* y, u64 y_stride) {
    typedef Vec<T, W> V;
    constexpr int N = InFlight<W>::N;
    const u32 i0 = blockIdx.x * (256 * N) + threadIdx.x;
    typename V::raw a[N], b[N];
    u32 c[N], gate[N][W / 2];
    u64 row[N];
    bool mine[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const u32 i = i0 + j * 256, r = s.per_row.of(i);
        c[j] = (i - r * s.per_row.d) * W;
        row[j] = s.row0 + r;
        mine[j] = i < s.n && (WHOLE || c[j] < s.cols);
        if (!mine[j]) continue;
        a[j] = load_cols<V, W, WHOLE, FAR>(x + row[j] * x_stride, c[j], s.cols);
        if (RES) b[j] = load_cols<V, W, WHOLE, FAR>(res + row[j] * res_stride, c[j], s.cols);
    }
    gates_of_units<W, N>(m, draw_of(m), s.row0 * s.per_row.d + i0, gate);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if (!mine[j]) continue;
        float v[W], w[W];
        a[j] = settle_cols<V, W, WHOLE>(a[j], c[j], s.cols);
        V::shut(a[j], gate[j]);
        V::open(a[j], v);
        for (int k = 0; k < W; ++k) v[k] *= m.keep;
        if (RES) {
            V::open(settle_cols<V, W, WHOLE>(b[j], c[j], s.cols), w);
            for (int k = 0; k < W; ++k) v[k] += w[k];
        }
        store_cols<V, W, FAR>(y + row[j] * y_stride, c[j], s.cols, v);
    }
}

template <class S, class T, int W, bool DROP, bool WHOLE, bool FAR>
__global__ __launch_bounds__(256) void embed_units(Units s, Mask m, const int64_t* __restrict__ tokens, const typename S::elem* __restrict__ table, u64 table_stride, u64 vocab,
                                                   float scale, const int64_t* __restrict__ positions, const typename S::elem* __restrict__ pos_table, u64 pos_stride, u64 n_pos,
                                                   typename T::elem* __restrict__ out, u64 out_stride) {
    typedef Vec<S, W> VS;
    typedef Vec<T, W> VT;
    constexpr int N = EMBED_EACH;
    const u32 i0 = blockIdx.x * (256 * N) + threadIdx.x;
    typename VS::raw a[N], b[N];
    u32 c[N], gate[N][W / 2];
    u64 row[N], tok[N], at[N];
    bool mine[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const u32 i = i0 + j * 256, r = s.per_row.of(i);
        c[j] = (i - r * s.per_row.d) * W;
        row[j] = s.row0 + r;
        mine[j] = i < s.n && (WHOLE || c[j] < s.cols);
        tok[j] = mine[j] ? (u64)tokens[row[j]] : vocab;
        at[j] = mine[j] && positions ? (u64)positions[row[j]] : n_pos;
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if (tok[j] < vocab) a[j] = load_cols<VS, W, WHOLE>(table + tok[j] * table_stride, c[j], s.cols);
        if (at[j] < n_pos) b[j] = load_cols<VS, W, WHOLE>(pos_table + at[j] * pos_stride, c[j], s.cols);
    }
    if (DROP) gates_of_units<W, N>(m, draw_of(m), s.row0 * s.per_row.d + i0, gate);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if (!mine[j]) continue;
        float v[W] = {}, w[W];
        if (tok[j] < vocab) {                        // (a select, not a product with zero: scale may be infinite)
            VS::open(settle_cols<VS, W, WHOLE>(a[j], c[j], s.cols), v);
            for (int k = 0; k < W; ++k) v[k] *= scale;
        }
        if (at[j] < n_pos) {
            VS::open(settle_cols<VS, W, WHOLE>(b[j], c[j], s.cols), w);
            for (int k = 0; k < W; ++k) v[k] += w[k];
        }
        if (DROP) {
#pragma unroll
            for (int k = 0; k < W; ++k) {
                const int half = (k & 1) ? (int)gate[j][k >> 1] >> 16 : (int)(gate[j][k >> 1] << 16) >> 16;
                v[k] = __builtin_bit_cast(float, __builtin_bit_cast(int, v[k] * m.keep) & half);
            }
        }
        store_cols<VT, W, FAR>(out + row[j] * out_stride, c[j], s.cols, v);
    }
}

// ------------------------------------------------------------------------------------------
// gradient of the embedding: a table row's gradient is the sum over the places of its token, so the places are sorted by token
// (stably: a row is summed in the order of its places) and the sorted list is cut into pieces of equal length.  Every value of dy is read
// once and every row of the result written once, by whichever launch has the memory idle: the rows without a token are most of the bytes.
// 8192 x 768 16-bit values on a base of 50257 rows: 71 us (sort 47, of which 22 alone, with 263 of the 309 MB beside it; pieces 18, chains 7), 4.5 TB/s where a
// large copy reaches 5.4.  65536 x 1024, no base: 100 us (four launches of sort 38, pieces 52, chains 10), 3.4 TB/s: what is left is that pieces take
// two to four steps of eight rows one after the other, five waves a SIMD of 16-bit values under a mask (six, with registers spilled, 106 us).  Floats take 86 to 137 registers, three to five waves:
// 8192 x 768 on a base 75 us where the bytes take 62, 65536 x 1024 116 where they take 88.
// ------------------------------------------------------------------------------------------
// far: base and gradient are more than the memory-side cache should hold, and lie on multiples of 16 bytes
struct Result { const float* base; u64 base_stride; float* grad; u64 grad_stride; u64 vocab; float scale; bool far; };
typedef Vec<F32, 4> G4;                          // of the gradient and its base

// Rows of the result as they are without a token: FILL_EACH units a thread, NT threads a block.  `present`: a byte a row, whether it has a token and
// is left out; null: all rows are written, those with a token again later.
#define FILL_EACH 2
template <int NT>
__device__ __forceinline__ void fill_block(const Result& out, const Units& s, u32 block, const uint8_t* present) {
    const u32 i0 = block * (NT * FILL_EACH) + threadIdx.x;
    f4v v[FILL_EACH];
    u32 r[FILL_EACH], c[FILL_EACH];
    bool mine[FILL_EACH];
#pragma unroll
    for (int k = 0; k < FILL_EACH; ++k) {
        const u32 i = i0 + k * NT;
        r[k] = s.per_row.of(i);
        c[k] = (i - r[k] * s.per_row.d) * 4;
        mine[k] = i < s.n && c[k] < s.cols;
        v[k] = f4v{0, 0, 0, 0};
    }
    if (present) {
        uint8_t there[FILL_EACH];
#pragma unroll
        for (int k = 0; k < FILL_EACH; ++k) there[k] = mine[k] ? present[s.row0 + r[k]] : 0;
#pragma unroll
        for (int k = 0; k < FILL_EACH; ++k) mine[k] = mine[k] && !there[k];
    }
    if (out.base) {
#pragma unroll
        for (int k = 0; k < FILL_EACH; ++k) {
            if (!mine[k]) continue;
            const float* row = out.base + (s.row0 + r[k]) * out.base_stride;
            v[k] = out.far ? load_cols<G4, 4, true, true>(row, c[k], s.cols) : load_cols<G4, 4, false>(row, c[k], s.cols);
        }
        if (!out.far) {
#pragma unroll
            for (int k = 0; k < FILL_EACH; ++k) if (mine[k]) v[k] = settle_cols<G4, 4, false>(v[k], c[k], s.cols);
        }
    }
#pragma unroll
    for (int k = 0; k < FILL_EACH; ++k) {
        if (!mine[k]) continue;
        const float y[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
        float* row = out.grad + (s.row0 + r[k]) * out.grad_stride;
        if (out.far) store_cols<G4, 4, true>(row, c[k], s.cols, y);
        else store_cols<G4, 4>(row, c[k], s.cols, y);
    }
}
static u32 fill_blocks(const Units& s, u32 nt = 256) { return blocks_of(s.n, nt * FILL_EACH); }

__global__ __launch_bounds__(256) void fill_rows(Units s, Result out) { fill_block<256>(out, s, blockIdx.x, nullptr); }

// Few tokens: one launch.  A block stands for one token place and 64 units of columns.  It compares its token with all of them; the block of
// a token's first place adds up the rows of all its places, a quarter of the places a wave, and the others end.  The launch's other blocks write the rows that have no
// token, each block with a list of which of its rows have one.  (Sorting takes three launches, 17 us for 500 tokens of 768 columns; this one 8.)
#define GRAD_SHORT 512
#define GRAD_DIM_LIMIT (1u << 22)                // so that a block for each place and 256 columns is a grid of fewer than 2^32 threads
#define SHORT_FILL 4                             // units that a thread of a filling block writes

template <class T, bool DROP, bool WHOLE>
__global__ __launch_bounds__(256) void grad_short(const int64_t* __restrict__ tokens, u32 n, u32 cols, u32 units, u32 lead_blocks, Units rows, Result out, Mask m,
                                                  const typename T::elem* __restrict__ dy, u64 dy_stride) {
    typedef Vec<T, 4> V;
    const u32 tid = threadIdx.x;
    if (blockIdx.x >= lead_blocks) {
        __shared__ u32 taken[256 * SHORT_FILL];
        const u32 i0 = (blockIdx.x - lead_blocks) * (256 * SHORT_FILL), i1 = rows.n - i0 < 256 * SHORT_FILL ? rows.n : i0 + 256 * SHORT_FILL;
        const u32 r0 = rows.per_row.of(i0), r1 = rows.per_row.of(i1 - 1);
        for (u32 r = tid; r <= r1 - r0; r += 256) taken[r] = 0;
        __syncthreads();
        for (u32 j = tid; j < n; j += 256) {
            const u64 r = (u64)tokens[j] - rows.row0 - r0;
            if (r <= r1 - r0) taken[r] = 1;
        }
        f4v v[SHORT_FILL];
#pragma unroll
        for (int k = 0; k < SHORT_FILL; ++k) {
            const u32 i = i0 + k * 256 + tid, r = rows.per_row.of(i), c = (i - r * units) * 4;
            v[k] = f4v{0, 0, 0, 0};
            if (i < i1 && c < cols && out.base) v[k] = load_cols<G4, 4, WHOLE>(out.base + (rows.row0 + r) * out.base_stride, c, cols);
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < SHORT_FILL; ++k) {
            const u32 i = i0 + k * 256 + tid, r = rows.per_row.of(i), c = (i - r * units) * 4;
            if (i >= i1 || c >= cols || taken[r - r0]) continue;
            if (out.base) v[k] = settle_cols<G4, 4, WHOLE>(v[k], c, cols);
            const float y[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
            store_cols<G4, 4>(out.grad + (rows.row0 + r) * out.grad_stride, c, cols, y);
        }
        return;
    }
    __shared__ u64 words[GRAD_SHORT / 64];                 // the places of the token, 64 a word
    __shared__ f4v sums[4][64];
    const u32 lane = tid & 63, w = tid >> 6, chunk = blockIdx.x / n, t = blockIdx.x - chunk * n;
    const u32 unit = chunk * 64 + lane, c = unit * 4, n_words = (n + 63) / 64, each = (n_words + 3) / 4;
    const u64 tok = (u64)tokens[t];
    u64 other[GRAD_SHORT / 256];
#pragma unroll
    for (u32 k = 0; k < GRAD_SHORT / 256; ++k) other[k] = k * 256 + tid < n ? (u64)tokens[k * 256 + tid] : ~0ull;
#pragma unroll
    for (u32 k = 0; k < GRAD_SHORT / 256; ++k) {
        const u64 hits = __ballot(other[k] == tok);
        if (lane == 0) words[k * 4 + w] = hits;
    }
    __syncthreads();
    if (tok >= out.vocab) return;
    u64 earlier = 0;
    for (u32 k = 0; k < t / 64; ++k) earlier |= words[k];
    if (earlier || (words[t / 64] & ((1ull << (t & 63)) - 1))) return;
    const bool here = c < cols;
    const u64 draw = DROP ? draw_of(m) : 0, groups = units / 2;
    f4v base = {0, 0, 0, 0};
    if (w == 0 && here && out.base) base = load_cols<G4, 4, WHOLE>(out.base + tok * out.base_stride, c, cols);
    float sum[4] = {0, 0, 0, 0};
    for (u32 k = w * each; k < n_words && k < (w + 1) * each; ++k) {                 // a quarter of the places a wave
        u64 left = (u64)(u32)__builtin_amdgcn_readfirstlane((int)(u32)words[k]) | (u64)(u32)__builtin_amdgcn_readfirstlane((int)(u32)(words[k] >> 32)) << 32;
        while (left) {
            u64 row[8];
            bool there[8];
            typename V::raw v[8] = {};
            u32 gate[8][2];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                there[q] = left != 0;
                row[q] = k * 64 + (left ? (u32)__ffsll((long long)left) - 1 : 0);
                left &= left - 1;
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) if (there[q] && here) v[q] = load_cols<V, 4, WHOLE>(dy + row[q] * dy_stride, c, cols);
#pragma unroll
            for (int q = 0; q < 8; q += 2) {
                if (!there[q]) continue;
                if (DROP) gates_of_two(m, draw, row[q] * groups + unit / 2, row[q + 1] * groups + unit / 2, gate[q], gate[q + 1]);
#pragma unroll
                for (int h = q; h < q + 2; ++h) {
                    float x[4];
                    if (!there[h]) continue;
                    if (here) v[h] = settle_cols<V, 4, WHOLE>(v[h], c, cols);
                    if (DROP) V::shut(v[h], gate[h]);
                    V::open(v[h], x);
                    for (int e = 0; e < 4; ++e) sum[e] += DROP ? x[e] * m.keep : x[e];
                }
            }
        }
    }
    sums[w][lane] = G4::pack(sum);
    __syncthreads();
    if (w || !here) return;
    const f4v all = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
    if (out.base) base = settle_cols<G4, 4, WHOLE>(base, c, cols);
    float y[4];
    for (int e = 0; e < 4; ++e) y[e] = base[e] + out.scale * all[e];
    store_cols<G4, 4>(out.grad + tok * out.grad_stride, c, cols, y);
}

// ---- the sort: least significant digit first, at most nine bits a pass ----
#define BINS 512
#define NO_TOKEN(vocab) ((u32)(vocab))          // key of a place without a token: behind all others

__device__ __forceinline__ u32 key_of(int64_t token, u64 vocab) { return (u64)token < vocab ? (u32)token : NO_TOKEN(vocab); }

// Lanes whose digit is this lane's.
__device__ __forceinline__ u64 same_digit(u32 digit, u32 bits, bool there) {
    u64 m = __ballot(there);
#pragma unroll
    for (u32 b = 0; b < 9; ++b) {
        if (b < bits) {
            const bool one = (digit >> b) & 1;
            const u64 v = __ballot(one);
            m &= one ? v : ~v;
        }
    }
    return m;
}
// Place of this lane's item among its wave's items of the same digit so far, counted up in the wave's own counters.  The counter is
// read by the lane that adds to it, and handed to the others.
__device__ __forceinline__ u32 rank_digit(u32* counts, u32 digit, u32 bits, bool there) {
    const u64 m = same_digit(digit, bits, there);
    const u32 lane = threadIdx.x & 63, first = (u32)__ffsll((long long)m) - 1;
    u32 old = 0;
    if (there && lane == first) old = atomicAdd(&counts[digit], (u32)__popcll(m));
    old = (u32)__shfl((int)old, (int)(there ? first : lane));
    return old + (u32)__popcll(m & ((1ull << lane) - 1));
}
// Exclusive sum over the block's threads (NT a multiple of 64); `part`: one word for each wave.
template <int NT>
__device__ __forceinline__ u32 scan_block(u32 v, u32* part) {
    const u32 lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    u32 s = v;
    for (int d = 1; d < WAVE; d <<= 1) { const u32 o = __shfl_up(s, d); if ((int)lane >= d) s += o; }
    __syncthreads();
    if (lane == 63) part[w] = s;
    __syncthreads();
    u32 before = 0;
    for (u32 i = 0; i < NT / WAVE; ++i) if (i < w) before += part[i];
    return before + s - v;
}

struct SortShape { u32 n, passes, bits; u64 vocab; };        // bits: of a digit
#define KEY_PAD 64                               // entries without a token before the sorted list and behind it

__device__ __forceinline__ void pad_lists(u32* keys, u32* places, u32 n, u64 vocab) {
    if (threadIdx.x < KEY_PAD) {
        keys[(int)threadIdx.x - KEY_PAD] = NO_TOKEN(vocab);
        keys[n + threadIdx.x] = NO_TOKEN(vocab);
        places[n + threadIdx.x] = 0;
    }
}

// All places of a short batch by one block, keys and places in LDS between the passes (8192 places 22 us, as long as four launches of tiles take; 16000 39);
// the launch's other blocks write rows of the result meanwhile (those that have a token are written again later, they are few next to the table).  `present`: marks of the rows that have a token, or null.
#define SORT_BLOCK_ROWS 8
#define SORT_BLOCK_MOST (1024 * SORT_BLOCK_ROWS)
struct SortLds { u32 keys[SORT_BLOCK_MOST]; u16 places[SORT_BLOCK_MOST]; u32 counts[16][BINS]; u32 part[16]; };

__global__ __launch_bounds__(1024) void sort_one_block(SortShape q, const int64_t* __restrict__ tokens, u32* __restrict__ keys_out, u32* __restrict__ places_out, u32* __restrict__ n_chains,
                                                       uint8_t* __restrict__ present, Units s, Result out) {
    __shared__ SortLds L;
    const u32 tid = threadIdx.x;
    if (blockIdx.x) {
        fill_block<1024>(out, s, blockIdx.x - 1, nullptr);
        return;
    }
    const u32 lane = tid & 63, w = tid >> 6;
    const u32 rows = (q.n + 1023) / 1024;                // of 64 places, of each wave
    if (tid == 0) *n_chains = 0;
    pad_lists(keys_out, places_out, q.n, q.vocab);
    if (present) for (u32 i = tid; i < (u32)(q.vocab + 3) / 4; i += 1024) ((u32*)present)[i] = 0;      // (the passes' barriers come before the marks)
    u32 key[SORT_BLOCK_ROWS], place[SORT_BLOCK_ROWS], rank[SORT_BLOCK_ROWS];
#pragma unroll
    for (u32 r = 0; r < SORT_BLOCK_ROWS; ++r) {
        const u32 i = (w * rows + r) * 64 + lane;
        if (r < rows && i < q.n) { key[r] = key_of(tokens[i], q.vocab); place[r] = i; }
    }
    for (u32 pass = 0; pass < q.passes; ++pass) {
        for (u32 i = tid; i < 16 * BINS; i += 1024) (&L.counts[0][0])[i] = 0;
        __syncthreads();
        const u32 shift = pass * q.bits, mask = (1u << q.bits) - 1;
#pragma unroll
        for (u32 r = 0; r < SORT_BLOCK_ROWS; ++r)
            if (r < rows) {
                const bool there = (w * rows + r) * 64 + lane < q.n;
                rank[r] = rank_digit(L.counts[w], (key[r] >> shift) & mask, q.bits, there);
            }
        __syncthreads();
        u32 of_wave[16], sum = 0;
        if (tid < BINS) {
#pragma unroll
            for (u32 i = 0; i < 16; ++i) of_wave[i] = L.counts[i][tid];
#pragma unroll
            for (u32 i = 0; i < 16; ++i) { const u32 c = of_wave[i]; of_wave[i] = sum; sum += c; }
        }
        const u32 before = scan_block<1024>(sum, L.part);
        if (tid < BINS) {
#pragma unroll
            for (u32 i = 0; i < 16; ++i) L.counts[i][tid] = of_wave[i] + before;
        }
        __syncthreads();
        const bool last = pass + 1 == q.passes;
#pragma unroll
        for (u32 r = 0; r < SORT_BLOCK_ROWS; ++r)
            if (r < rows && (w * rows + r) * 64 + lane < q.n) {
                const u32 to = L.counts[w][(key[r] >> shift) & mask] + rank[r];
                if (last) {
                    keys_out[to] = key[r];
                    places_out[to] = place[r];
                    if (present && key[r] != NO_TOKEN(q.vocab)) present[key[r]] = 1;
                }
                else { L.keys[to] = key[r]; L.places[to] = (u16)place[r]; }
            }
        if (last) break;
        __syncthreads();
#pragma unroll
        for (u32 r = 0; r < SORT_BLOCK_ROWS; ++r) {
            const u32 i = (w * rows + r) * 64 + lane;
            if (r < rows && i < q.n) { key[r] = L.keys[i]; place[r] = L.places[i]; }
        }
    }
}

// Longer batches: at most SORT_TILES tiles, two launches a pass (count, move).  The first launch clears the marks of the rows that have a token, the
// second sets them; their other blocks write rows of the result, the later ones only such that have no token.
#define SORT_TILES 64
#define SORT_STEP 1024                           // items that a block of 256 threads moves at once
struct SortFrom { const int64_t* tokens; const u32 *keys, *places; };            // tokens in the first pass, keys and places later

__device__ __forceinline__ u32 key_at(const SortFrom& f, u64 vocab, u32 i) { return f.tokens ? key_of(f.tokens[i], vocab) : f.keys[i]; }

__global__ __launch_bounds__(256) void sort_count(SortShape q, SortFrom from, u32 shift, u32 tile, u32 tiles, u32* __restrict__ hist, u32* __restrict__ n_chains, u32* __restrict__ clear, u32 clear_words,
                                                  Units s, Result out, const uint8_t* __restrict__ present) {
    __shared__ u32 counts[BINS];
    const u32 tid = threadIdx.x;
    if (blockIdx.x >= tiles) {
        for (u32 i = (blockIdx.x - tiles) * 256 + tid; i < clear_words; i += (gridDim.x - tiles) * 256) clear[i] = 0;
        fill_block<256>(out, s, blockIdx.x - tiles, present);
        return;
    }
    if (blockIdx.x == 0 && tid == 0) *n_chains = 0;
    for (u32 b = tid; b < BINS; b += 256) counts[b] = 0;
    __syncthreads();
    const u32 mask = (1u << q.bits) - 1, lo = blockIdx.x * tile, hi = q.n - lo < tile ? q.n : lo + tile;
    for (u32 i = lo + tid; i < hi; i += 256) atomicAdd(&counts[(key_at(from, q.vocab, i) >> shift) & mask], 1u);
    __syncthreads();
    for (u32 b = tid; b < BINS; b += 256) hist[blockIdx.x * BINS + b] = counts[b];
}

__global__ __launch_bounds__(256) void sort_move(SortShape q, SortFrom from, u32 shift, u32 tile, u32 tiles, const u32* __restrict__ hist, u32* __restrict__ keys_to, u32* __restrict__ places_to,
                                                 uint8_t* __restrict__ mark, Units s, Result out, const uint8_t* __restrict__ present) {
    __shared__ u32 counts[4][BINS];
    __shared__ u32 next[BINS];                   // where the next item of a digit goes
    __shared__ u32 part[4];
    const u32 tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    if (blockIdx.x >= tiles) {
        fill_block<256>(out, s, blockIdx.x - tiles, present);
        return;
    }
    if (blockIdx.x == 0) pad_lists(keys_to, places_to, q.n, q.vocab);
    const u32 mask = (1u << q.bits) - 1, lo = blockIdx.x * tile, hi = q.n - lo < tile ? q.n : lo + tile;
    u32 total[2] = {0, 0}, mine[2] = {0, 0};
    for (u32 t0 = 0; t0 < tiles; t0 += 16) {               // sixteen tiles' counts in flight, also where there are fewer
        uint2 c[16];
#pragma unroll
        for (u32 j = 0; j < 16; ++j) c[j] = *(const uint2*)(hist + (t0 + j < tiles ? t0 + j : tiles - 1) * BINS + 2 * tid);
#pragma unroll
        for (u32 j = 0; j < 16; ++j) {
            if (t0 + j < blockIdx.x) { mine[0] += c[j].x; mine[1] += c[j].y; }
            if (t0 + j < tiles) { total[0] += c[j].x; total[1] += c[j].y; }
        }
    }
    const u32 before = scan_block<256>(total[0] + total[1], part);
    next[2 * tid] = before + mine[0];
    next[2 * tid + 1] = before + total[0] + mine[1];
    for (u32 at = lo; at < hi; at += SORT_STEP) {
        for (u32 i = tid; i < 4 * BINS; i += 256) (&counts[0][0])[i] = 0;
        __syncthreads();
        u32 key[4], place[4], rank[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const u32 i = at + (w * 4 + r) * 64 + lane;
            if (i < hi) { key[r] = key_at(from, q.vocab, i); place[r] = from.tokens ? i : from.places[i]; }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) rank[r] = rank_digit(counts[w], (key[r] >> shift) & mask, q.bits, at + (w * 4 + r) * 64 + lane < hi);
        __syncthreads();
        for (u32 b = tid; b < BINS; b += 256) {
            u32 sum = next[b];
            for (int i = 0; i < 4; ++i) { const u32 c = counts[i][b]; counts[i][b] = sum; sum += c; }
            next[b] = sum;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (at + (w * 4 + r) * 64 + lane < hi) {
                const u32 to = counts[w][(key[r] >> shift) & mask] + rank[r];
                keys_to[to] = key[r];
                places_to[to] = place[r];
                if (mark && key[r] != NO_TOKEN(q.vocab)) mark[key[r]] = 1;
            }
        __syncthreads();
    }
}

// ---- the sums over the sorted places ----
// A thread takes four columns of a piece of LEN sorted places.  A run (the places of one token) is summed by the piece it begins in, also where it ends in the next one.
// A run that covers the whole next piece is long: its pieces' sums go to `chain` (two rows a piece: [0] of a run that comes from before, [1] of one that goes on)
// and are added up by the next launch.  The pieces know which it is from the keys at their borders; the list of keys has KEY_PAD entries "none" before it and behind it, so
// that nothing asks where it ends.  PIECE_STEP rows, and those of the base, are in flight together, with the keys behind them.
#define PIECE_STEP 8
template <class T, bool DROP, int LEN, bool WHOLE, bool BASE>
__global__ __launch_bounds__(256) void grad_pieces(const u32* __restrict__ keys, const u32* __restrict__ places, Units s, Result out, Mask m, const typename T::elem* __restrict__ dy, u64 dy_stride,
                                                   float* __restrict__ chain, uint2* __restrict__ chains, u32* __restrict__ n_chains, u32 piece_blocks, Units fill, const uint8_t* __restrict__ present) {
    if (blockIdx.x >= piece_blocks) {
        fill_block<256>(out, fill, blockIdx.x - piece_blocks, present);
        return;
    }
    typedef Vec<T, 4> V;
    constexpr int B = PIECE_STEP;
    const u32 i = blockIdx.x * 256 + threadIdx.x;
    if (i >= s.n) return;                                  // (an even number of threads stays)
    const u32 units = s.per_row.d, local = s.per_row.of(i), unit = i - local * units, c = unit * 4;
    const u32 piece = (u32)s.row0 + local, none = NO_TOKEN(out.vocab);
    const bool here = WHOLE || c < s.cols;
    const u32* const key = keys + (u64)piece * LEN;
    const u32* const place = places + (u64)piece * LEN;
    float* const slot = chain + ((u64)piece * 2 * units + unit) * 4;
    u4v own[LEN / 4], after[LEN / 4], at_k[B / 4], at_p[B / 4];
#pragma unroll
    for (int j = 0; j < LEN / 4; ++j) { own[j] = ((const u4v*)key)[j]; after[j] = ((const u4v*)(key + LEN))[j]; }
#pragma unroll
    for (int j = 0; j < B / 4; ++j) { at_k[j] = own[j]; at_p[j] = ((const u4v*)place)[j]; }
    const u32 before = *(key - 1), far = *(key - LEN - 1), k0 = own[0].x, k1 = own[LEN / 4 - 1].w;
    if (k0 == none) return;
    u32 same0 = 0, same1 = 0;
#pragma unroll
    for (int j = 0; j < LEN; ++j) { same0 += own[j / 4][j % 4] == k0; same1 += after[j / 4][j % 4] == k1; }
    const bool came = before == k0, first_to_chain = came && (far == k0 || k1 == k0);
    const u32 from = came && !first_to_chain ? same0 : 0;
    const bool goes = k1 != none && same1 && !(first_to_chain && k1 == k0), last_to_chain = goes && same1 == LEN;
    const u32 to = goes && !last_to_chain ? LEN + same1 : LEN;
    const u64 draw = DROP ? draw_of(m) : 0, groups = units / 2;
    float sum[4] = {0, 0, 0, 0};
    for (u32 at = 0; at < to; at += B) {
        u32 k[B + 1], p[B];
        typename V::raw v[B] = {};
        f4v base[B];
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const bool mine = at + j >= from && at + j < to;
            k[j] = mine ? at_k[j / 4][j % 4] : none;
            p[j] = at_p[j / 4][j % 4];
        }
        // (past the last step these are read too: the lists go on for KEY_PAD entries)
#pragma unroll
        for (int j = 0; j < B / 4; ++j) { at_k[j] = *(const u4v*)(key + at + B + 4 * j); at_p[j] = *(const u4v*)(place + at + B + 4 * j); }
#pragma unroll
        for (int j = 0; j < B; ++j)
            if (k[j] != none && here) {
                v[j] = load_cols<V, 4, WHOLE, true>(dy + (u64)p[j] * dy_stride, c, s.cols);
                if (BASE) base[j] = load_cols<G4, 4, WHOLE>(out.base + (u64)k[j] * out.base_stride, c, s.cols);
            }
        k[B] = at + B < to ? at_k[0].x : none;
#pragma unroll
        for (int j0 = 0; j0 < B; j0 += 2) {
            if (k[j0] == none && k[j0 + 1] == none) continue;
            u32 gate[2][2];
            if (DROP) gates_of_two(m, draw, (u64)p[j0] * groups + unit / 2, (u64)p[j0 + 1] * groups + unit / 2, gate[0], gate[1]);
#pragma unroll
            for (int j = j0; j < j0 + 2; ++j) {
                if (k[j] == none) continue;
                float x[4];
                if (here) v[j] = settle_cols<V, 4, WHOLE>(v[j], c, s.cols);
                if (DROP) V::shut(v[j], gate[j - j0]);
                else if constexpr (sizeof(typename T::elem) == 2) asm volatile("" : "+v"(v[j]));        // not converted before its turn: the eight rows' floats took 170 registers, and 65536 x 1024 without dropout 176 us
                V::open(v[j], x);
                for (int e = 0; e < 4; ++e) sum[e] += DROP ? x[e] * m.keep : x[e];
                if (k[j + 1] == k[j]) continue;
                if (first_to_chain && k[j] == k0) {
                    G4::store(slot, G4::pack(sum));
                } else if (last_to_chain && k[j] == k1) {
                    G4::store(slot + (u64)units * 4, G4::pack(sum));
                    if (unit == 0) chains[atomicAdd(n_chains, 1u)] = make_uint2(piece, k1);        // in any order: the chains have nothing to do with each other
                } else if (here) {
                    float y[4];
                    if (BASE) base[j] = settle_cols<G4, 4, WHOLE>(base[j], c, s.cols);
                    for (int e = 0; e < 4; ++e) y[e] = (BASE ? base[j][e] : 0.0f) + out.scale * sum[e];
                    store_cols<G4, 4>(out.grad + (u64)k[j] * out.grad_stride, c, s.cols, y);
                }
                for (int e = 0; e < 4; ++e) sum[e] = 0.0f;
            }
        }
    }
}

// The long runs: a block takes a chain and 32 units of columns; 8 threads share its pieces, eight at a time, whose keys and sums are asked for together (the
// sums of pieces past the chain's end are not used).
__global__ __launch_bounds__(256) void grad_chains(const u32* __restrict__ keys, u32 len, u32 pieces, u32 cols, u32 units, Result out, const float* __restrict__ chain, const uint2* __restrict__ chains,
                                                   const u32* __restrict__ n_chains, u32 chain_blocks, Units fill, const uint8_t* __restrict__ present) {
    if (blockIdx.x >= chain_blocks) {
        fill_block<256>(out, fill, blockIdx.x - chain_blocks, present);
        return;
    }
    __shared__ f4v sh[8][32];
    const u32 chunks = (units + 31) / 32, ul = threadIdx.x & 31, strand = threadIdx.x >> 5;
    const u64 work = (u64)*n_chains * chunks;
    for (u64 w = blockIdx.x; w < work; w += chain_blocks) {
        const u32 i = (u32)(w / chunks), unit = (u32)(w - (u64)i * chunks) * 32 + ul;
        const uint2 head = chains[i];
        const u32 piece = head.x, k = head.y;
        const bool here = unit < units, lead = strand == 0 && unit * 4 < cols;
        f4v sum = {0, 0, 0, 0}, base = {0, 0, 0, 0};
        if (here) {
            if (strand == 0) sum = G4::load(chain + (((u64)piece * 2 + 1) * units + unit) * 4);
            if (lead && out.base) base = load_cols<G4, 4, false>(out.base + (u64)k * out.base_stride, unit * 4, cols);
            for (u32 p = piece + 1 + strand;; p += 64) {
                u32 at[8];
                f4v v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const u32 q = p + 8 * j < pieces ? p + 8 * j : pieces - 1;
                    at[j] = keys[(u64)q * len];
                    v[j] = G4::load(chain + ((u64)q * 2 * units + unit) * 4);
                    if (p + 8 * j >= pieces) at[j] = ~k;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) if (at[j] == k) sum += v[j];
                if (at[7] != k) break;
            }
        }
        sh[strand][ul] = sum;
        for (u32 half = 4; half; half >>= 1) {
            __syncthreads();
            if (strand < half) sh[strand][ul] += sh[strand + half][ul];
        }
        if (lead) {
            const f4v all = sh[0][ul];
            if (out.base) base = settle_cols<G4, 4, false>(base, unit * 4, cols);
            float y[4];
            for (int e = 0; e < 4; ++e) y[e] = base[e] + out.scale * all[e];
            store_cols<G4, 4>(out.grad + (u64)k * out.grad_stride, unit * 4, cols, y);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------
// C-ABI
// ------------------------------------------------------------------------------------------
thread_local char worker_err[192] = "";
extern "C" const char* dblp_worker_error(void) { return worker_err; }

extern "C" int dblp_embed(int device, void* stream, const int64_t* d_tokens, uint64_t n_tokens, uint32_t dim,
                          const void* d_table, uint64_t table_stride, uint64_t vocab, int table_type, float scale,
                          const int64_t* d_positions, const void* d_pos_table, uint64_t pos_stride, uint64_t n_positions,
                          const dblp_drop* h_drop, void* d_out, uint64_t out_stride, int out_type) {
    const char* call = "embed";
    REFUSE_IF(bad_type(table_type) || bad_type(out_type), "unknown type");
    REFUSE_IF(dim == 0 || dim >= COUNT_LIMIT || vocab == 0 || vocab >= COUNT_LIMIT || n_tokens >= COUNT_LIMIT, "size out of range");
    REFUSE_IF(n_tokens && (!d_tokens || !d_table || !d_out), "null pointer");
    REFUSE_IF(n_tokens && (d_positions == nullptr) != (d_pos_table == nullptr), "positions and their table go together");
    REFUSE_IF(d_positions && (n_positions == 0 || n_positions >= COUNT_LIMIT), "size of the position table out of range");
    REFUSE_IF(off(d_tokens, 8) || off(d_positions, 8) || off(d_table, type_bytes(table_type)) || off(d_pos_table, type_bytes(table_type)) || off(d_out, type_bytes(out_type)), "misaligned pointer");
    REFUSE_IF(n_tokens > 1 && out_stride < dim, "the output's rows overlap");
    Mask m;
    if (const int rc = take_drop(call, h_drop, &m)) return rc;
    if (n_tokens == 0) return DBLP_OK;
    OnDevice on(device);
    if (on.err != hipSuccess) return no_device(call, on.err);
    Launches launch;
    by_type(table_type, [&](auto st) {
        by_type(out_type, [&](auto tt) {
            typedef decltype(st) S;
            typedef decltype(tt) T;
            constexpr int W = sizeof(typename S::elem) == 4 || sizeof(typename T::elem) == 4 ? 4 : 8;
            const bool far = n_tokens * dim * type_bytes(out_type) > FAR_BYTES / 2;
            each_launch<W>(n_tokens, dim, [&](Units s) {
                const auto pick = [&](auto whole, auto far_out) { return m.on ? embed_units<S, T, W, true, decltype(whole)::value, decltype(far_out)::value> : embed_units<S, T, W, false, decltype(whole)::value, decltype(far_out)::value>; };
                const auto kernel = dim % 8 ? pick(Int<0>(), Int<0>()) : far ? pick(Int<1>(), Int<1>()) : pick(Int<1>(), Int<0>());
                launch(kernel, dim3(blocks_of(s.n, 256 * EMBED_EACH)), 256, (hipStream_t)stream, s, m, d_tokens, (const typename S::elem*)d_table, (u64)table_stride, (u64)vocab, scale,
                                   d_positions, (const typename S::elem*)d_pos_table, (u64)pos_stride, (u64)n_positions, (typename T::elem*)d_out, (u64)out_stride);
            });
        });
    });
    return launched(call, launch);
}

// How the places of a batch are sorted and cut, and where its intermediate results lie in the workspace.
struct GradPlan {
    bool short_batch;            // one launch
    u32 len, pieces, passes, bits, tile, tiles;
    u64 keys[2], places[2], hist, present, chains, n_chains, chain, bytes;
};

#define GRAD_FEW 16384                           // tokens whose pieces are short
static GradPlan grad_plan(u64 n, u64 vocab, u32 dim) {
    GradPlan p = {};
    p.short_batch = n <= GRAD_SHORT;
    p.bytes = 256;
    if (p.short_batch) return p;
    const u64 units = units_per_row<4>(dim);
    u32 bits = 0;
    while ((vocab >> bits) != 0) ++bits;                 // keys run to vocab itself
    p.passes = (bits + 8) / 9;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.len = n <= GRAD_FEW ? 8 : 16;               // few places: enough threads; many: fewer chains (65536 x 1024: 12 us of chains, 18 with 8)
    p.pieces = (u32)((n + p.len - 1) / p.len);
    p.tile = (u32)round_up((n + SORT_TILES - 1) / SORT_TILES, SORT_STEP);
    p.tiles = (u32)((n + p.tile - 1) / p.tile);
    u64 at = 0;
    const auto take = [&](u64 bytes) { const u64 here = at; at += round_up(bytes, 256); return here; };
    for (int i = 0; i < 2; ++i) { p.keys[i] = take(4 * (n + 2 * KEY_PAD)) + 4 * KEY_PAD; p.places[i] = take(4 * (n + KEY_PAD)); }
    p.hist = take(4ull * SORT_TILES * BINS);
    p.present = take(vocab);
    p.chains = take(8ull * p.pieces);
    p.n_chains = take(4);
    p.chain = take((u64)p.pieces * 2 * units * 16);
    p.bytes = at;
    return p;
}

extern "C" uint64_t dblp_embed_grad_workspace(uint64_t n_tokens, uint64_t vocab, uint32_t dim) {
    if (n_tokens >= COUNT_LIMIT || vocab == 0 || vocab >= COUNT_LIMIT || dim == 0 || dim >= GRAD_DIM_LIMIT) return 0;
    const u64 bytes = grad_plan(n_tokens, vocab, dim).bytes, few = n_tokens > GRAD_FEW ? grad_plan(GRAD_FEW, vocab, dim).bytes : 0;
    return bytes > few ? bytes : few;                // (a larger batch's is large enough for a smaller one)
}

// Which rows without a token are written beside which launch.  Sorting, short batches' pieces and chains leave the memory idle for about as long as it takes to
// move these bytes; what is left goes beside the one-block sort, or the pieces of a long batch.  Rows written before the marks are known may be written again.
#define FILL_COUNT (24ull << 20)                 // beside each count of a tiled sort, twice that where a base is read (65536 x 1024 on a base of 50257 rows 151 us, 159 with
#define FILL_MOVE (64ull << 20)                  // 24 beside each launch; 9000 x 768 on a base 79, 88) and beside each move
#define FILL_PIECES (32ull << 20)
#define FILL_CHAINS (12ull << 20)
#define MARK_MOST (1u << 20)                     // rows whose marks one block clears beside its sort

struct Fill {
    u32 dim, per_row;
    u64 row, rows;                               // next row, rows in all
    u64 row_bytes;
    u64 left() const { return (rows - row) * row_bytes; }
    Units take(u64 bytes) {                     // about that many bytes' rows
        const u64 want = (bytes + row_bytes - 1) / row_bytes, n = want < rows - row ? want : rows - row;
        const Units s = {row, (u32)(n * per_row), dim, Divider::by(per_row)};
        row += n;
        return s;
    }
    Units all_but(u64 bytes) { return take(left() > bytes ? left() - bytes : 0); }
};

extern "C" int dblp_embed_grad(int device, void* stream, const int64_t* d_tokens, uint64_t n_tokens, uint32_t dim, uint64_t vocab,
                               float scale, const dblp_drop* h_drop, const void* d_dy, uint64_t dy_stride, int dy_type,
                               const float* d_base, uint64_t base_stride, float* d_grad, uint64_t grad_stride,
                               void* d_workspace, uint64_t workspace_bytes) {
    const char* call = "embed_grad";
    REFUSE_IF(bad_type(dy_type), "unknown type");
    REFUSE_IF(dim == 0 || dim >= GRAD_DIM_LIMIT || vocab == 0 || vocab >= COUNT_LIMIT || n_tokens >= COUNT_LIMIT, "size out of range");
    REFUSE_IF(!d_grad || (n_tokens && (!d_tokens || !d_dy)), "null pointer");
    REFUSE_IF(off(d_tokens, 8) || off(d_dy, type_bytes(dy_type)) || off(d_base, 4) || off(d_grad, 4), "misaligned pointer");
    REFUSE_IF(vocab > 1 && grad_stride < dim, "the gradient's rows overlap");
    REFUSE_IF(d_base == d_grad && vocab > 1 && base_stride != grad_stride, "in place, the strides must be equal");
    REFUSE_IF(!d_workspace || off(d_workspace, 256) || workspace_bytes < dblp_embed_grad_workspace(n_tokens, vocab, dim), "workspace missing, misaligned or too small");
    Mask m;
    if (const int rc = take_drop(call, h_drop, &m)) return rc;
    OnDevice on(device);
    if (on.err != hipSuccess) return no_device(call, on.err);
    Launches launch;
    const hipStream_t st = (hipStream_t)stream;
    // (the hint takes a copy of 154 MB from 55 to 48 us, one of 38 MB from 11 to 14)
    const bool far = vocab * dim * (d_base ? 8 : 4) > FAR_BYTES / 2 && dim % 4 == 0 && !off(d_base, 16) && !off(d_grad, 16) && base_stride % 4 == 0 && grad_stride % 4 == 0;
    const Result out = {d_base, base_stride, d_grad, grad_stride, vocab, scale, far};
    const GradPlan p = grad_plan(n_tokens, vocab, dim);
    const u32 n = (u32)n_tokens, units = units_per_row<4>(dim);
    if (p.short_batch) {
        by_type(dy_type, [&](auto tt) {
            typedef decltype(tt) T;
            const bool whole = dim % 8 == 0;
            const auto kernel = m.on ? (whole ? grad_short<T, true, true> : grad_short<T, true, false>) : (whole ? grad_short<T, false, true> : grad_short<T, false, false>);
            u32 lead = (u32)(n * ((units + 63ull) / 64));
            const auto go = [&](Units s) {
                const u32 fill = blocks_of(s.n, 256 * SHORT_FILL);
                if (lead + fill)
                    launch(kernel, dim3(lead + fill), 256, st, d_tokens, n, dim, units, lead, s, out, m, (const typename T::elem*)d_dy, (u64)dy_stride);
                lead = 0;
            };
            if (d_base == d_grad) go(Units{0, 0, dim, Divider::by(units)});
            else each_launch<4>(vocab, dim, go);
        });
        return launched(call, launch);
    }
    uint8_t* const ws = (uint8_t*)d_workspace;
    u32* const n_chains = (u32*)(ws + p.n_chains);
    uint2* const chains = (uint2*)(ws + p.chains);
    float* const chain = (float*)(ws + p.chain);
    const SortShape q = {n, p.passes, p.bits, vocab};
    const bool one_block = n <= SORT_BLOCK_MOST, in_place = d_base == d_grad;
    // a table whose units do not fit one launch is written before everything else
    const bool beside = !in_place && vocab * units < COUNT_LIMIT;
    if (!in_place && !beside)
        each_launch<4>(vocab, dim, [&](Units s) { launch(fill_rows, dim3(fill_blocks(s)), 256, st, s, out); });
    Fill fill = {dim, units, 0, beside ? vocab : 0, (u64)dim * (d_base ? 8 : 4)};
    uint8_t* const present = beside && (!one_block || vocab <= MARK_MOST) ? ws + p.present : nullptr;
    int at = 0;
    if (one_block) {
        const Units s = fill.all_but(present ? FILL_PIECES + FILL_CHAINS : 0);
        launch(sort_one_block, dim3(1 + fill_blocks(s, 1024)), 1024, st, q, d_tokens, (u32*)(ws + p.keys[0]), (u32*)(ws + p.places[0]), n_chains, present, s, out);
    } else {
        for (u32 pass = 0; pass < p.passes; ++pass, at ^= 1) {
            const SortFrom from = {pass ? nullptr : d_tokens, pass ? (u32*)(ws + p.keys[at ^ 1]) : nullptr, pass ? (u32*)(ws + p.places[at ^ 1]) : nullptr};
            const u32 clear = pass == 0 && present ? (u32)(round_up(vocab, 256) / 4) : 0;
            const Units a = fill.take(d_base ? 2 * FILL_COUNT : FILL_COUNT), b = fill.take(FILL_MOVE);
            const u32 others = fill_blocks(a) + (u32)((clear + 1023) / 1024);
            launch(sort_count, dim3(p.tiles + others), 256, st, q, from, pass * p.bits, p.tile, p.tiles, (u32*)(ws + p.hist), n_chains, (u32*)present, clear, a, out, (const uint8_t*)(pass ? present : nullptr));
            launch(sort_move, dim3(p.tiles + fill_blocks(b)), 256, st, q, from, pass * p.bits, p.tile, p.tiles, (const u32*)(ws + p.hist), (u32*)(ws + p.keys[at]), (u32*)(ws + p.places[at]),
                               pass == 0 ? present : (uint8_t*)nullptr, b, out, (const uint8_t*)(pass ? present : nullptr));
        }
        at ^= 1;
    }
    const u32 *const keys = (u32*)(ws + p.keys[at]), *const places = (u32*)(ws + p.places[at]);
    Units beside_pieces = fill.all_but(FILL_CHAINS);
    by_type(dy_type, [&](auto tt) {
        typedef decltype(tt) T;
        const auto by_len = [&](auto len) {
            constexpr int L = decltype(len)::value;
            const auto pick = [&](auto whole, auto base) { return m.on ? grad_pieces<T, true, L, decltype(whole)::value, decltype(base)::value> : grad_pieces<T, false, L, decltype(whole)::value, decltype(base)::value>; };
            return d_base ? (dim % 8 ? pick(Int<0>(), Int<1>()) : pick(Int<1>(), Int<1>())) : (dim % 8 ? pick(Int<0>(), Int<0>()) : pick(Int<1>(), Int<0>()));
        };
        const auto kernel = p.len == 8 ? by_len(Int<8>()) : by_len(Int<16>());
        each_launch<4>(p.pieces, dim, [&](Units s) {
            const u32 blocks = blocks_of(s.n, 256);
            launch(kernel, dim3(blocks + fill_blocks(beside_pieces)), 256, st, keys, places, s, out, m, (const typename T::elem*)d_dy, (u64)dy_stride, chain, chains, n_chains, blocks, beside_pieces, (const uint8_t*)present);
            beside_pieces.n = 0;
        });
    });
    const u64 most = (u64)p.pieces * ((units + 31) / 32);
    const u32 chain_blocks = most < 4096 ? (u32)most : 4096;
    const Units beside_chains = fill.take(fill.left());
    launch(grad_chains, dim3(chain_blocks + fill_blocks(beside_chains)), 256, st, keys, p.len, p.pieces, dim, units, out, (const float*)chain, (const uint2*)chains, (const u32*)n_chains, chain_blocks, beside_chains, (const uint8_t*)present);
    return launched(call, launch);
}

extern "C" int dblp_dropout(int device, void* stream, uint64_t rows, uint32_t cols, const void* d_x, uint64_t x_stride,
                            const void* d_residual, uint64_t residual_stride, const dblp_drop* h_drop,
                            void* d_y, uint64_t y_stride, int type) {
    const char* call = "dropout";
    REFUSE_IF(bad_type(type), "unknown type");
    REFUSE_IF(cols == 0 || cols >= COUNT_LIMIT || rows >= COUNT_LIMIT, "size out of range");
    REFUSE_IF(!h_drop || (rows && (!d_x || !d_y)), "null pointer");
    REFUSE_IF(off(d_x, type_bytes(type)) || off(d_residual, type_bytes(type)) || off(d_y, type_bytes(type)), "misaligned pointer");
    REFUSE_IF(rows > 1 && y_stride < cols, "the output's rows overlap");
    REFUSE_IF(rows > 1 && ((d_y == d_x && y_stride != x_stride) || (d_y == d_residual && y_stride != residual_stride)), "in place, the strides must be equal");
    Mask m;
    if (const int rc = take_drop(call, h_drop, &m)) return rc;
    if (rows == 0) return DBLP_OK;
    OnDevice on(device);
    if (on.err != hipSuccess) return no_device(call, on.err);
    Launches launch;
    const bool far = rows * cols * type_bytes(type) * (d_residual ? 3 : 2) >= FAR_BYTES;
    by_type(type, [&](auto tt) {
        typedef decltype(tt) T;
        typedef const typename T::elem* in;
        constexpr int W = sizeof(typename T::elem) == 4 ? 4 : 8;
        each_launch<W>(rows, cols, [&](Units s) {
            const auto pick = [&](auto whole, auto past) { return d_residual ? dropout_units<T, W, true, decltype(whole)::value, decltype(past)::value> : dropout_units<T, W, false, decltype(whole)::value, decltype(past)::value>; };
            const auto kernel = cols % 8 ? pick(Int<0>(), Int<0>()) : far ? pick(Int<1>(), Int<1>()) : pick(Int<1>(), Int<0>());
            launch(kernel, dim3(blocks_of(s.n, 256 * InFlight<W>::N)), 256, (hipStream_t)stream, s, m, (in)d_x, (u64)x_stride, (in)d_residual, (u64)residual_stride, (typename T::elem*)d_y, (u64)y_stride);
        });
    });
    return launched(call, launch);
}
