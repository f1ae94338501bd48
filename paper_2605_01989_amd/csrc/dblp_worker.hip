// The two ends of a worker's training step on gfx950 (MI355X): embedding and its gradient, dropout,
// log probabilities and the policy loss.  Kernels and the C-ABI declared in include/dblp_worker.h.
//
// All of it is bound by memory: a few operations on each value, read once and written once.  Kernels are
// organised so that a thread's loads are 16 bytes wide and several of them are in flight.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include "../../include/dblp_worker.h"

typedef unsigned long long u64;
typedef uint32_t u32;
typedef uint16_t u16;

#define WAVE 64
#define LANES8 8                // columns that one thread holds, and one call of the generator serves

// ------------------------------------------------------------------------------------------
// element types
// ------------------------------------------------------------------------------------------
typedef float f4v __attribute__((ext_vector_type(4)));
typedef u32 u4v __attribute__((ext_vector_type(4)));
typedef f4v f4v_a4 __attribute__((aligned(4)));         // 16-byte accesses at an element's alignment
typedef u4v u4v_a2 __attribute__((aligned(2)));
typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef _Float16 h8v __attribute__((ext_vector_type(8)));
typedef float f8v __attribute__((ext_vector_type(8)));

// Each type: `raw`, eight elements as they lie in memory, loaded apart from their conversion so that several loads can be in flight.
struct F32 {
    typedef float elem;
    struct raw { f4v a, b; };
    static __device__ __forceinline__ float get(const float* p) { return *p; }
    static __device__ __forceinline__ void put(float* p, float v) { *p = v; }
    static __device__ __forceinline__ raw load(const float* p) { return {*(const f4v_a4*)p, *(const f4v_a4*)(p + 4)}; }
    static __device__ __forceinline__ raw some(const float* p, u32 n) {
        raw r = {};
        for (u32 i = 0; i < 7; ++i) if (i < n) { if (i < 4) r.a[i] = p[i]; else r.b[i - 4] = p[i]; }
        return r;
    }
    static __device__ __forceinline__ raw down(raw r, u32 by) {           // by 0..7 elements, zeros behind
        float v[8];
        open(r, v);
        for (u32 step = 4; step; step >>= 1)
            for (u32 i = 0; i < 8; ++i) { const float from = i + step < 8 ? v[i + step] : 0.0f; v[i] = (by & step) ? from : v[i]; }
        return {{v[0], v[1], v[2], v[3]}, {v[4], v[5], v[6], v[7]}};
    }
    static __device__ __forceinline__ void open(const raw& r, float (&v)[8]) {
        for (int i = 0; i < 4; ++i) { v[i] = r.a[i]; v[4 + i] = r.b[i]; }
    }
    static __device__ __forceinline__ void put8(float* p, const float (&v)[8]) {
        const f4v a = {v[0], v[1], v[2], v[3]}, b = {v[4], v[5], v[6], v[7]};
        *(f4v_a4*)p = a;
        *(f4v_a4*)(p + 4) = b;
    }
};

template <class E, class V8>
struct Half {
    typedef E elem;
    typedef u4v raw;
    static __device__ __forceinline__ float get(const E* p) { return (float)*p; }
    static __device__ __forceinline__ void put(E* p, float v) { *p = (E)v; }
    static __device__ __forceinline__ raw load(const E* p) { return *(const u4v_a2*)p; }
    static __device__ __forceinline__ raw some(const E* p, u32 n) {
        V8 r = {};
        for (u32 i = 0; i < 7; ++i) if (i < n) r[i] = p[i];
        return __builtin_bit_cast(u4v, r);
    }
    static __device__ __forceinline__ raw down(raw r, u32 by) {
        if (by & 4) r = (u4v){r.z, r.w, 0u, 0u};
        if (by & 2) r = (u4v){r.y, r.z, r.w, 0u};
        if (by & 1) r = (u4v){r.x >> 16 | r.y << 16, r.y >> 16 | r.z << 16, r.z >> 16 | r.w << 16, r.w >> 16};
        return r;
    }
    static __device__ __forceinline__ void open(const raw& r, float (&v)[8]) {
        const f8v f = __builtin_convertvector(__builtin_bit_cast(V8, r), f8v);
        for (int i = 0; i < 8; ++i) v[i] = f[i];
    }
    static __device__ __forceinline__ void put8(E* p, const float (&v)[8]) {
        const f8v f = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
        *(u4v_a2*)p = __builtin_bit_cast(u4v, __builtin_convertvector(f, V8));
    }
};
typedef Half<__bf16, bf8v> BF16;
typedef Half<_Float16, h8v> F16;

// Columns [c, c + 8) of a row of `cols`; those past the end read as zero and are not written.  WHOLE: cols is a multiple of eight.
// Otherwise the last group of a row is read from the row's last eight elements and shifted down in registers: one load for every
// group, without a branch that would have to wait for it (rows of fewer than eight elements apart).
template <class T, bool WHOLE>
__device__ __forceinline__ typename T::raw load_raw(const typename T::elem* row, u32 c, u32 cols) {
    if (WHOLE) return T::load(row + c);
    if (cols < 8) return T::some(row, cols);
    const u32 at = c + 8 <= cols ? c : cols - 8;
    return T::down(T::load(row + at), c - at);
}
template <class T>
__device__ __forceinline__ void load_group(const typename T::elem* row, u32 c, u32 cols, float (&v)[8]) { T::open(load_raw<T, false>(row, c, cols), v); }
template <class T>
__device__ __forceinline__ void store_group(typename T::elem* row, u32 c, u32 cols, const float (&v)[8]) {
    if (c + 8 <= cols) { T::put8(row + c, v); return; }
    for (u32 i = 0; i < 8; ++i) if (c + i < cols) T::put(row + c + i, v[i]);
}

// ------------------------------------------------------------------------------------------
// division of 32-bit numbers by one that a launch keeps: floor(n / d) as the high half of a product
// (Granlund and Montgomery, PLDI 1994), d >= 1
// ------------------------------------------------------------------------------------------
struct Divider {
    u32 d, mul, shift;
    __host__ static Divider by(u32 d) {
        Divider r = {d, 0, 0};
        while (((u64)1 << r.shift) < d) ++r.shift;
        r.mul = (u32)((((u64)1 << 32) * (((u64)1 << r.shift) - d)) / d + 1);
        return r;
    }
    __device__ __forceinline__ u32 of(u32 n) const {
        const u32 h = __umulhi(n, mul);
        return d == 1 ? n : (h + ((n - h) >> 1)) >> (shift - 1);
    }
};

// ------------------------------------------------------------------------------------------
// dropout masks: Philox4x32, ten rounds (Salmon et al., SC 2011)
// ------------------------------------------------------------------------------------------
struct Mask { u64 seed, draw; const u64* d_draw; u32 limit; float keep; };

// Eight gates of group g: v[i] = field i < limit ? +0 : v[i] * keep.  A select, so that what is dropped is zero also where
// it was infinite or NaN.
// Ten rounds are 20 products of 32 x 32 bits for eight values: at a quarter of the vector rate less than half of the
// time that reading and writing eight 16-bit values takes.
__device__ __forceinline__ void gate8(const Mask& m, u64 draw, u64 g, float (&v)[8]) {
    u32 a = (u32)g, b = (u32)(g >> 32), c = (u32)draw, d = (u32)(draw >> 32), k0 = (u32)m.seed, k1 = (u32)(m.seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const u64 p = (u64)a * 0xD2511F53u, q = (u64)c * 0xCD9E8D57u;
        a = (u32)(q >> 32) ^ b ^ k0;
        b = (u32)q;
        c = (u32)(p >> 32) ^ d ^ k1;
        d = (u32)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    const u32 w[4] = {a, b, c, d};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const u32 field = (i & 1) ? w[i >> 1] >> 16 : w[i >> 1] & 0xFFFFu;
        v[i] = field < m.limit ? 0.0f : v[i] * m.keep;
    }
}
__device__ __forceinline__ u64 draw_of(const Mask& m) { return m.draw + (m.d_draw ? *m.d_draw : 0); }

// ------------------------------------------------------------------------------------------
// dropout and embedding: a thread takes eight columns of a row; groups of eight are numbered through the matrix
// ------------------------------------------------------------------------------------------
struct Groups { u64 row0; u32 n, cols; Divider per_row; };     // groups of this launch (below 2^31), first row of it
#define GROUPS_EACH 2           // groups that a thread has in flight

template <class T, bool RES, bool WHOLE>
__global__ __launch_bounds__(256) void dropout_groups(Groups s, Mask m, const typename T::elem* x, u64 x_stride,
                                                      const typename T::elem* res, u64 res_stride, typename T::elem* y, u64 y_stride) {
    const u32 i0 = blockIdx.x * (256 * GROUPS_EACH) + threadIdx.x;
    typename T::raw a[GROUPS_EACH], b[GROUPS_EACH];
    u32 c[GROUPS_EACH];
    u64 row[GROUPS_EACH];
#pragma unroll
    for (int j = 0; j < GROUPS_EACH; ++j) {
        const u32 i = i0 + j * 256, r = s.per_row.of(i);
        c[j] = (i - r * s.per_row.d) * 8;
        row[j] = s.row0 + r;
        if (i >= s.n) continue;
        a[j] = load_raw<T, WHOLE>(x + row[j] * x_stride, c[j], s.cols);
        if (RES) b[j] = load_raw<T, WHOLE>(res + row[j] * res_stride, c[j], s.cols);
    }
    const u64 draw = draw_of(m);
#pragma unroll
    for (int j = 0; j < GROUPS_EACH; ++j) {
        const u32 i = i0 + j * 256;
        if (i >= s.n) continue;
        float v[8], w[8];
        T::open(a[j], v);
        gate8(m, draw, s.row0 * s.per_row.d + i, v);
        if (RES) {
            T::open(b[j], w);
            for (int k = 0; k < 8; ++k) v[k] += w[k];
        }
        store_group<T>(y + row[j] * y_stride, c[j], s.cols, v);
    }
}

template <class S, class T, bool DROP, bool WHOLE>
__global__ __launch_bounds__(256) void embed_groups(Groups s, Mask m, const int64_t* __restrict__ tokens, const typename S::elem* __restrict__ table, u64 table_stride, u64 vocab,
                                                    float scale, const int64_t* __restrict__ positions, const typename S::elem* __restrict__ pos_table, u64 pos_stride, u64 n_pos,
                                                    typename T::elem* __restrict__ out, u64 out_stride) {
    const u32 i0 = blockIdx.x * (256 * GROUPS_EACH) + threadIdx.x;
    typename S::raw a[GROUPS_EACH], b[GROUPS_EACH];
    u32 c[GROUPS_EACH];
    u64 row[GROUPS_EACH], tok[GROUPS_EACH], at[GROUPS_EACH];
#pragma unroll
    for (int j = 0; j < GROUPS_EACH; ++j) {
        const u32 i = i0 + j * 256, r = s.per_row.of(i);
        c[j] = (i - r * s.per_row.d) * 8;
        row[j] = s.row0 + r;
        tok[j] = i < s.n ? (u64)tokens[row[j]] : vocab;
        at[j] = i < s.n && positions ? (u64)positions[row[j]] : n_pos;
    }
#pragma unroll
    for (int j = 0; j < GROUPS_EACH; ++j) {
        if (tok[j] < vocab) a[j] = load_raw<S, WHOLE>(table + tok[j] * table_stride, c[j], s.cols);
        if (at[j] < n_pos) b[j] = load_raw<S, WHOLE>(pos_table + at[j] * pos_stride, c[j], s.cols);
    }
    const u64 draw = DROP ? draw_of(m) : 0;
#pragma unroll
    for (int j = 0; j < GROUPS_EACH; ++j) {
        const u32 i = i0 + j * 256;
        if (i >= s.n) continue;
        float v[8] = {0, 0, 0, 0, 0, 0, 0, 0}, w[8];
        if (tok[j] < vocab) {
            S::open(a[j], v);
            for (int k = 0; k < 8; ++k) v[k] *= scale;
        }
        if (at[j] < n_pos) {
            S::open(b[j], w);
            for (int k = 0; k < 8; ++k) v[k] += w[k];
        }
        if (DROP) gate8(m, draw, s.row0 * s.per_row.d + i, v);
        store_group<T>(out + row[j] * out_stride, c[j], s.cols, v);
    }
}

// ------------------------------------------------------------------------------------------
// gradient of the embedding: a table row's gradient is the sum over the places of its token, so the places are sorted by token
// (stably: a row is summed in the order of its places) and the sorted list is cut into pieces of equal length
// ------------------------------------------------------------------------------------------
// Eight columns of a row of the result: base (or zero) + scale * sum.
__device__ __forceinline__ void put_row(const float* base, u64 base_stride, float* grad, u64 grad_stride, u64 row, u32 c, u32 cols, float scale, const float (&sum)[8]) {
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (base) load_group<F32>(base + row * base_stride, c, cols, v);
    for (int e = 0; e < 8; ++e) v[e] += scale * sum[e];
    store_group<F32>(grad + row * grad_stride, c, cols, v);
}

struct Result { const float* base; u64 base_stride; float* grad; u64 grad_stride; u64 vocab; float scale; };

// Group i of those rows of the result that have no token (`present` says which have one; null: all rows alike).
__device__ __forceinline__ void fill_group(const Result& out, const Groups& s, u32 i, const uint8_t* present) {
    const u32 r = s.per_row.of(i), c = (i - r * s.per_row.d) * 8;
    const u64 row = s.row0 + r;
    if (present && present[row]) return;
    const float z[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    put_row(out.base, out.base_stride, out.grad, out.grad_stride, row, c, s.cols, 0.0f, z);
}
__global__ __launch_bounds__(256) void fill_rows(Groups s, Result out, const uint8_t* __restrict__ present) {
    const u32 i = blockIdx.x * 256 + threadIdx.x;
    if (i < s.n) fill_group(out, s, i, present);
}

// Few tokens: one launch.  A wave stands for one token place and 64 groups of columns.  It compares its token with all of them; the wave of
// a token's first place adds up the rows of all its places, in order, and the others end.  The launch's other blocks write the rows that have no
// token, each block with a list of which of its rows have one.
#define GRAD_SHORT 512
#define FILL_EACH 4                              // groups that a thread of a filling block writes

template <class T, bool DROP, bool WHOLE>
__global__ __launch_bounds__(256) void grad_short(const int64_t* __restrict__ tokens, u32 n, u32 cols, u32 groups, u32 lead_blocks, Groups rows, Result out, Mask m,
                                                  const typename T::elem* __restrict__ dy, u64 dy_stride) {
    const u32 tid = threadIdx.x;
    if (blockIdx.x >= lead_blocks) {
        __shared__ u32 taken[256 * FILL_EACH + 1];
        const u32 i0 = (blockIdx.x - lead_blocks) * (256 * FILL_EACH), i1 = rows.n - i0 < 256 * FILL_EACH ? rows.n : i0 + 256 * FILL_EACH;
        const u32 r0 = rows.per_row.of(i0), r1 = rows.per_row.of(i1 - 1);
        for (u32 r = tid; r <= r1 - r0; r += 256) taken[r] = 0;
        __syncthreads();
        for (u32 j = tid; j < n; j += 256) {
            const u64 r = (u64)tokens[j] - rows.row0 - r0;
            if (r <= r1 - r0) taken[r] = 1;
        }
        __syncthreads();
        F32::raw v[FILL_EACH];
#pragma unroll
        for (int k = 0; k < FILL_EACH; ++k) {
            const u32 i = i0 + k * 256 + tid, r = rows.per_row.of(i), c = (i - r * groups) * 8;
            v[k] = F32::raw{};
            if (i < i1 && out.base) v[k] = load_raw<F32, WHOLE>(out.base + (rows.row0 + r) * out.base_stride, c, cols);
        }
#pragma unroll
        for (int k = 0; k < FILL_EACH; ++k) {
            const u32 i = i0 + k * 256 + tid, r = rows.per_row.of(i), c = (i - r * groups) * 8;
            if (i >= i1 || taken[r - r0]) continue;
            float y[8];
            F32::open(v[k], y);
            store_group<F32>(out.grad + (rows.row0 + r) * out.grad_stride, c, cols, y);
        }
        return;
    }
    const u32 lane = tid & 63, unit = blockIdx.x * 4 + (tid >> 6), chunk = unit / n, t = unit - chunk * n;
    const u32 c = (chunk * 64 + lane) * 8;
    if (chunk * 64 >= groups) return;
    const u64 tok = (u64)tokens[t];
    if (tok >= out.vocab) return;
    u64 hits[GRAD_SHORT / 64];
#pragma unroll
    for (u32 k = 0; k < GRAD_SHORT / 64; ++k) {
        const u32 j = k * 64 + lane;
        hits[k] = __ballot(j < n && (u64)tokens[j < n ? j : 0] == tok);
    }
    u64 earlier = 0;
#pragma unroll
    for (u32 k = 0; k < GRAD_SHORT / 64; ++k) earlier |= k < t / 64 ? hits[k] : k == t / 64 ? hits[k] & ((1ull << (t & 63)) - 1) : 0;
    if (earlier) return;
    const bool here = c < cols;
    const u64 draw = DROP ? draw_of(m) : 0;
    F32::raw base = {};
    if (here && out.base) base = load_raw<F32, WHOLE>(out.base + tok * out.base_stride, c, cols);
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (u32 k = 0; k < GRAD_SHORT / 64; ++k)
        for (u64 left = hits[k]; left;) {
            u64 row[8];
            bool there[8];
            typename T::raw v[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                there[q] = left != 0;
                row[q] = k * 64 + (left ? (u32)__ffsll((long long)left) - 1 : 0);
                left &= left - 1;
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) if (there[q] && here) v[q] = load_raw<T, WHOLE>(dy + row[q] * dy_stride, c, cols);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                if (!there[q] || !here) continue;
                float x[8];
                T::open(v[q], x);
                if (DROP) gate8(m, draw, row[q] * groups + c / 8, x);
                for (int e = 0; e < 8; ++e) sum[e] += x[e];
            }
        }
    if (!here) return;
    float y[8];
    F32::open(base, y);
    for (int e = 0; e < 8; ++e) y[e] += out.scale * sum[e];
    store_group<F32>(out.grad + tok * out.grad_stride, c, cols, y);
}

// ---- the sort: least significant digit first, at most nine bits a pass ----
#define BINS 512
#define NO_TOKEN(vocab) ((u32)(vocab))          // key of a place without a token: behind all others

__device__ __forceinline__ u32 key_of(int64_t token, u64 vocab) { return (u64)token < vocab ? (u32)token : NO_TOKEN(vocab); }

// Lanes whose digit is this lane's.
__device__ __forceinline__ u64 same_digit(u32 digit, u32 bits, bool there) {
    u64 m = __ballot(there);
    for (u32 b = 0; b < bits; ++b) {
        const bool one = (digit >> b) & 1;
        const u64 v = __ballot(one);
        m &= one ? v : ~v;
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

// All places of a short batch by one block, keys and places in LDS between the passes; the launch's other blocks write the result's rows
// meanwhile (all of them: rows with a token are written again, they are few next to the table).
#define SORT_BLOCK_ROWS 16
#define SORT_BLOCK_MOST (1024 * SORT_BLOCK_ROWS)
struct SortLds { u32 keys[SORT_BLOCK_MOST]; u16 places[SORT_BLOCK_MOST]; u32 counts[16][BINS]; u32 part[16]; };

__global__ __launch_bounds__(1024) void sort_one_block(SortShape q, const int64_t* __restrict__ tokens, u32* __restrict__ keys_out, u32* __restrict__ places_out, u32* __restrict__ n_chains,
                                                       Groups s, Result out) {
    __shared__ SortLds L;
    const u32 tid = threadIdx.x;
    if (blockIdx.x) {
        for (u32 i = (blockIdx.x - 1) * 1024 + tid; i < s.n; i += (gridDim.x - 1) * 1024) fill_group(out, s, i, nullptr);
        return;
    }
    const u32 lane = tid & 63, w = tid >> 6;
    const u32 rows = (q.n + 1023) / 1024;                // of 64 places, of each wave
    if (tid == 0) *n_chains = 0;
    pad_lists(keys_out, places_out, q.n, q.vocab);
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
        u32 sum = 0;
        if (tid < BINS)
            for (u32 i = 0; i < 16; ++i) { const u32 c = L.counts[i][tid]; L.counts[i][tid] = sum; sum += c; }
        const u32 before = scan_block<1024>(sum, L.part);
        if (tid < BINS)
            for (u32 i = 0; i < 16; ++i) L.counts[i][tid] += before;
        __syncthreads();
        const bool last = pass + 1 == q.passes;
#pragma unroll
        for (u32 r = 0; r < SORT_BLOCK_ROWS; ++r)
            if (r < rows && (w * rows + r) * 64 + lane < q.n) {
                const u32 to = L.counts[w][(key[r] >> shift) & mask] + rank[r];
                if (last) { keys_out[to] = key[r]; places_out[to] = place[r]; }
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
// second sets them, the last two fill the rows that have none beside their own work.
#define SORT_TILES 64
#define SORT_STEP 1024                           // items that a block of 256 threads moves at once
struct SortFrom { const int64_t* tokens; const u32 *keys, *places; };            // tokens in the first pass, keys and places later

__device__ __forceinline__ u32 key_at(const SortFrom& f, u64 vocab, u32 i) { return f.tokens ? key_of(f.tokens[i], vocab) : f.keys[i]; }

__global__ __launch_bounds__(256) void sort_count(SortShape q, SortFrom from, u32 shift, u32 tile, u32 tiles, u32* __restrict__ hist, u32* __restrict__ n_chains, u32* __restrict__ clear, u32 clear_words,
                                                  Groups s, Result out, const uint8_t* __restrict__ present) {
    __shared__ u32 counts[BINS];
    const u32 tid = threadIdx.x;
    if (blockIdx.x >= tiles) {
        const u32 at = (blockIdx.x - tiles) * 256 + tid, step = (gridDim.x - tiles) * 256;
        for (u32 i = at; i < clear_words; i += step) clear[i] = 0;
        for (u32 i = at; i < s.n; i += step) fill_group(out, s, i, present);
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
                                                 uint8_t* __restrict__ mark, Groups s, Result out, const uint8_t* __restrict__ present) {
    __shared__ u32 counts[4][BINS];
    __shared__ u32 next[BINS];                   // where the next item of a digit goes
    __shared__ u32 part[4];
    const u32 tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    if (blockIdx.x >= tiles) {
        for (u32 i = (blockIdx.x - tiles) * 256 + tid; i < s.n; i += (gridDim.x - tiles) * 256) fill_group(out, s, i, present);
        return;
    }
    if (blockIdx.x == 0) pad_lists(keys_to, places_to, q.n, q.vocab);
    u32 total[2] = {0, 0}, mine[2] = {0, 0};
#pragma unroll 8
    for (u32 t = 0; t < tiles; ++t) {
        const uint2 c = *(const uint2*)(hist + t * BINS + 2 * tid);
        if (t < blockIdx.x) { mine[0] += c.x; mine[1] += c.y; }
        total[0] += c.x; total[1] += c.y;
    }
    const u32 before = scan_block<256>(total[0] + total[1], part);
    next[2 * tid] = before + mine[0];
    next[2 * tid + 1] = before + total[0] + mine[1];
    const u32 mask = (1u << q.bits) - 1, lo = blockIdx.x * tile, hi = q.n - lo < tile ? q.n : lo + tile;
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
// A thread takes eight columns of a piece of LEN sorted places.  A run (the places of one token) is summed by the piece it begins in, also where it ends in the next one.
// A run that covers the whole next piece is long: its pieces' sums go to `chain` (two rows a piece: [0] of a run that comes from before, [1] of one that goes on)
// and are added up by the next launch.  The pieces know which it is from the keys at their borders; the list of keys has KEY_PAD entries "none" before it and behind it, so
// that nothing asks where it ends.  Eight places at a time: their rows, and the rows of the base, are all in flight before the first is added; the next eight keys with them.
template <class T, bool DROP, int LEN, bool WHOLE>
__global__ __launch_bounds__(256) void grad_pieces(const u32* __restrict__ keys, const u32* __restrict__ places, Groups s, Result out, Mask m, const typename T::elem* __restrict__ dy, u64 dy_stride,
                                                   float* __restrict__ chain, u32* __restrict__ chains, u32* __restrict__ n_chains) {
    const u32 i = blockIdx.x * 256 + threadIdx.x;
    if (i >= s.n) return;
    const u32 groups = s.per_row.d, local = s.per_row.of(i), g = i - local * groups, c = g * 8;
    const u32 piece = (u32)s.row0 + local, none = NO_TOKEN(out.vocab);
    const u32* const key = keys + (u64)piece * LEN;
    const u32* const place = places + (u64)piece * LEN;
    float* const slot = chain + ((u64)piece * 2 * groups + g) * 8;
    u4v own[LEN / 4], after[LEN / 4], at_k[2], at_p[2];
#pragma unroll
    for (int j = 0; j < LEN / 4; ++j) { own[j] = ((const u4v*)key)[j]; after[j] = ((const u4v*)(key + LEN))[j]; }
    at_p[0] = ((const u4v*)place)[0];
    at_p[1] = ((const u4v*)place)[1];
    const u32 before = *(key - 1), far = *(key - LEN - 1), k0 = own[0].x, k1 = own[LEN / 4 - 1].w;
    if (k0 == none) return;
    u32 same0 = 0, same1 = 0;
#pragma unroll
    for (int j = 0; j < LEN; ++j) { same0 += own[j / 4][j % 4] == k0; same1 += after[j / 4][j % 4] == k1; }
    const bool came = before == k0, first_to_chain = came && (far == k0 || k1 == k0);
    const u32 from = came && !first_to_chain ? same0 : 0;
    const bool goes = k1 != none && same1 && !(first_to_chain && k1 == k0), last_to_chain = goes && same1 == LEN;
    const u32 to = goes && !last_to_chain ? LEN + same1 : LEN;
    const u64 draw = DROP ? draw_of(m) : 0;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    at_k[0] = own[0];
    at_k[1] = own[1];
    for (u32 at = 0; at < to; at += 8) {
        u32 k[9], p[8];
        typename T::raw v[8];
        F32::raw base[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool mine = at + j >= from && at + j < to;
            k[j] = mine ? at_k[j / 4][j % 4] : none;
            p[j] = at_p[j / 4][j % 4];
        }
        // (past the last batch these are read too: the lists go on for KEY_PAD entries)
        at_k[0] = *(const u4v*)(key + at + 8);
        at_k[1] = *(const u4v*)(key + at + 12);
        at_p[0] = *(const u4v*)(place + at + 8);
        at_p[1] = *(const u4v*)(place + at + 12);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (k[j] != none) {
                v[j] = load_raw<T, WHOLE>(dy + (u64)p[j] * dy_stride, c, s.cols);
                if (out.base) base[j] = load_raw<F32, WHOLE>(out.base + (u64)k[j] * out.base_stride, c, s.cols);
            }
        k[8] = at + 8 < to ? at_k[0].x : none;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (k[j] == none) continue;
            float x[8];
            T::open(v[j], x);
            if (DROP) gate8(m, draw, (u64)p[j] * groups + g, x);
            for (int e = 0; e < 8; ++e) sum[e] += x[e];
            if (k[j + 1] == k[j]) continue;
            if (first_to_chain && k[j] == k0) {
                F32::put8(slot, sum);
            } else if (last_to_chain && k[j] == k1) {
                F32::put8(slot + (u64)groups * 8, sum);
                if (g == 0) chains[atomicAdd(n_chains, 1u)] = piece;           // in any order: the chains have nothing to do with each other
            } else {
                float y[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                if (out.base) F32::open(base[j], y);
                for (int e = 0; e < 8; ++e) y[e] += out.scale * sum[e];
                store_group<F32>(out.grad + (u64)k[j] * out.grad_stride, c, s.cols, y);
            }
            for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
        }
    }
}

// The long runs: a block takes a chain and 16 groups of columns; 16 threads share the pieces of each.
__global__ __launch_bounds__(256) void grad_chains(const u32* __restrict__ keys, u32 n, u32 len, u32 cols, u32 groups, Result out, const float* __restrict__ chain, const u32* __restrict__ chains,
                                                   const u32* __restrict__ n_chains) {
    __shared__ float sh[16][16][8 + 1];
    const u32 gl = threadIdx.x & 15, strand = threadIdx.x >> 4, g = blockIdx.y * 16 + gl, all = *n_chains;
    for (u32 i = blockIdx.x; i < all; i += gridDim.x) {
        const u32 piece = chains[i];
        const u32 k = keys[(piece + 1) * len];             // the run covers the next piece
        float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (g < groups) {
            if (strand == 0) F32::open(F32::load(chain + (((u64)piece * 2 + 1) * groups + g) * 8), sum);
            for (u64 p = (u64)piece + 1 + strand; p * len < n && keys[p * len] == k; p += 16) {
                float v[8];
                F32::open(F32::load(chain + (p * 2 * groups + g) * 8), v);
                for (int e = 0; e < 8; ++e) sum[e] += v[e];
            }
        }
        for (int e = 0; e < 8; ++e) sh[strand][gl][e] = sum[e];
        for (u32 half = 8; half; half >>= 1) {
            __syncthreads();
            if (strand < half)
                for (int e = 0; e < 8; ++e) sh[strand][gl][e] += sh[strand + half][gl][e];
        }
        if (strand == 0 && g < groups) {
            for (int e = 0; e < 8; ++e) sum[e] = sh[0][gl][e];
            put_row(out.base, out.base_stride, out.grad, out.grad_stride, k, g * 8, cols, out.scale, sum);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------
// logits: a row's maximum and the sum of its exponentials in one pass
// ------------------------------------------------------------------------------------------
#define LOG2E 1.4426950408889634f

// (m, s): largest value met and sum of exp(x - m).  Nothing met: (-inf, 0).
struct Soft { float m, s; };
__device__ __forceinline__ float shift_of(float m) { return m == -INFINITY ? 0.0f : m; }     // exp(-inf - -inf) would be NaN
__device__ __forceinline__ float exp_of(float x, float shift) { return __builtin_amdgcn_exp2f((x - shift) * LOG2E); }
__device__ __forceinline__ Soft soft_join(Soft a, Soft b) {
    const float m = fmaxf(a.m, b.m), at = shift_of(m);
    return {m, a.s * exp_of(a.m, at) + b.s * exp_of(b.m, at)};
}
__device__ __forceinline__ Soft soft_wave(Soft a) {
    for (int d = 1; d < WAVE; d <<= 1) a = soft_join(a, {__shfl_xor(a.m, d), __shfl_xor(a.s, d)});
    return a;
}
// The whole block's, to all of its threads.  `part`: one entry for each wave.
template <int NT>
__device__ __forceinline__ Soft soft_block(Soft a, Soft* part) {
    a = soft_wave(a);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = a;
    __syncthreads();
    a = part[0];
    for (int w = 1; w < NT / WAVE; ++w) a = soft_join(a, part[w]);
    return a;
}
__device__ __forceinline__ void soft_add8(Soft& a, const float (&v)[8]) {
    float m = a.m;
    for (int i = 0; i < 8; ++i) m = fmaxf(m, v[i]);
    const float at = shift_of(m);
    float s = a.s * exp_of(a.m, at);
    for (int i = 0; i < 8; ++i) s += exp_of(v[i], at);
    a = {m, s};
}
template <class T, int NT>
__device__ __forceinline__ Soft soft_row(const typename T::elem* row, u32 n) {
    Soft a = {-INFINITY, 0.0f};
    for (u32 c = threadIdx.x * 8; c < n; c += NT * 8) {
        float v[8];
        if (c + 8 <= n) T::open(T::load(row + c), v);
        else for (u32 i = 0; i < 8; ++i) v[i] = c + i < n ? T::get(row + c + i) : -INFINITY;
        soft_add8(a, v);
    }
    return a;
}

// Logarithms of a row in fp64: a score is a difference of numbers of ten or twenty, and policies' ratios are differences of scores.
// The maximum and the logarithm are not added up first: in a row of the type's lowest value the logarithm would be lost.
__device__ __forceinline__ double logp_of(float x, Soft a) { return ((double)x - (double)a.m) - log((double)a.s); }

template <class T, int NT>
__global__ __launch_bounds__(NT) void logprob_rows(const typename T::elem* __restrict__ logits, u64 stride, u32 vocab, const int64_t* __restrict__ targets,
                                                   float* __restrict__ logp, float* __restrict__ lse) {
    __shared__ Soft part[NT / WAVE];
    const u32 t = blockIdx.x;
    const u64 at = (u64)targets[t];
    if (at >= vocab) {
        if (threadIdx.x == 0) { logp[t] = 0.0f; if (lse) lse[t] = 0.0f; }
        return;
    }
    const typename T::elem* row = logits + (u64)t * stride;
    const Soft a = soft_block<NT>(soft_row<T, NT>(row, vocab), part);
    if (threadIdx.x == 0) {
        if (lse) lse[t] = (float)((double)a.m + log((double)a.s));
        logp[t] = a.m == -INFINITY ? -INFINITY : (float)logp_of(T::get(row + at), a);
    }
}

// ------------------------------------------------------------------------------------------
// policy loss
// ------------------------------------------------------------------------------------------
struct Policy { const int64_t* targets; const float *advantages, *weights, *old_logp, *ref_logp; float low, high, kl, grad_scale; };
struct TokenPart { float policy, kl; u32 counted, clipped; };          // a token's part of the five sums, weighted

// Of a counted token with log probability lp: what it adds to the sums, and d loss / d lp.
__device__ __forceinline__ TokenPart token_part(const Policy& p, u32 t, double lp, double* slope) {
    const double w = p.weights[t], a = p.advantages[t];
    const double r = p.old_logp ? exp(lp - (double)p.old_logp[t]) : 1.0;
    const double lo = 1.0 - (double)p.low, hi = 1.0 + (double)p.high;
    const double free_term = r * a, held = (r < lo ? lo : r > hi ? hi : r) * a;
    const bool clipped = held < free_term;
    double g = clipped ? 0.0 : -free_term, kl = 0.0;
    if (p.ref_logp) {
        const double d = (double)p.ref_logp[t] - lp, e = expm1(d);
        kl = e - d;
        g -= (double)p.kl * e;
    }
    *slope = w * g;
    return {(float)(w * -(clipped ? held : free_term)), (float)(w * kl), 1u, clipped ? 1u : 0u};
}

template <class T>
__device__ __forceinline__ void zero_row(typename T::elem* row, u32 n, u32 tid, u32 nt) {
    const float z[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (u32 c = tid * 8; c < n; c += nt * 8) store_group<T>(row, c, n, z);
}

// A block takes a row: one pass for maximum and sum, a second one for the gradient.
template <class T, int NT>
__global__ __launch_bounds__(NT) void policy_rows(Policy p, const typename T::elem* logits, u64 stride, u32 vocab, typename T::elem* dlogits, u64 dstride,
                                                  float* __restrict__ logp, TokenPart* __restrict__ parts) {
    __shared__ Soft part[NT / WAVE];
    __shared__ float slope_sh;
    const u32 t = blockIdx.x, tid = threadIdx.x;
    const u64 at = (u64)p.targets[t];
    const typename T::elem* row = logits + (u64)t * stride;
    typename T::elem* drow = dlogits ? dlogits + (u64)t * dstride : nullptr;
    Soft a = {-INFINITY, 0.0f};
    const bool read = at < vocab && p.weights[t] != 0.0f;
    if (read) a = soft_block<NT>(soft_row<T, NT>(row, vocab), part);
    if (a.m == -INFINITY) {
        if (tid == 0) { parts[t] = {0.0f, 0.0f, 0u, 0u}; if (logp) logp[t] = read ? -INFINITY : 0.0f; }
        if (drow) zero_row<T>(drow, vocab, tid, NT);
        return;
    }
    if (tid == 0) {
        const double lp = logp_of(T::get(row + at), a);
        double slope;
        parts[t] = token_part(p, t, lp, &slope);
        if (logp) logp[t] = (float)lp;
        slope_sh = (float)(slope * (double)p.grad_scale);
    }
    __syncthreads();
    if (!drow) return;
    const float g = slope_sh, k = -g / a.s;
    for (u32 c = tid * 8; c < vocab; c += NT * 8) {
        float v[8];
        load_group<T>(row, c, vocab, v);
        for (int i = 0; i < 8; ++i) v[i] = k * exp_of(v[i], a.m) + (c + i == at ? g : 0.0f);
        store_group<T>(drow, c, vocab, v);
    }
}

// The five sums over all tokens, in fp64 and a fixed order, by one block.
__global__ __launch_bounds__(1024) void policy_sums(const TokenPart* __restrict__ parts, u32 n, float kl_coef, float* __restrict__ stats) {
    __shared__ double sh[4][16];
    double s[4] = {0, 0, 0, 0};
    for (u32 t = threadIdx.x; t < n; t += 1024) {
        const TokenPart p = parts[t];
        s[0] += (double)p.policy; s[1] += (double)p.kl; s[2] += (double)p.clipped; s[3] += (double)p.counted;
    }
    for (int i = 0; i < 4; ++i) {
        for (int d = 1; d < WAVE; d <<= 1) s[i] += __shfl_xor(s[i], d);
        if ((threadIdx.x & 63) == 0) sh[i][threadIdx.x >> 6] = s[i];
    }
    __syncthreads();
    if (threadIdx.x) return;
    for (int i = 0; i < 4; ++i) { s[i] = 0; for (int w = 0; w < 16; ++w) s[i] += sh[i][w]; }
    stats[0] = (float)(s[0] + (double)kl_coef * s[1]);
    stats[1] = (float)s[0]; stats[2] = (float)s[1]; stats[3] = (float)s[2]; stats[4] = (float)s[3];
}

// ------------------------------------------------------------------------------------------
// C-ABI
// ------------------------------------------------------------------------------------------
static thread_local char worker_err[192] = "";
extern "C" const char* dblp_worker_error(void) { return worker_err; }

static int refuse(const char* call, const char* why) {
    snprintf(worker_err, sizeof worker_err, "%s: %s", call, why);
    return DBLP_EINVAL;
}

// The calling thread's device for the time of a call.
struct OnDevice {
    int before = -1, now;
    hipError_t err;
    explicit OnDevice(int device) : now(device) {
        err = hipGetDevice(&before);
        if (err == hipSuccess && before != device) err = hipSetDevice(device);
    }
    ~OnDevice() { if (before >= 0 && before != now) (void)hipSetDevice(before); }
};

static int launched(const char* call) {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return DBLP_OK;
    snprintf(worker_err, sizeof worker_err, "%s: %s", call, hipGetErrorString(e));
    return DBLP_EHIP;
}
static int no_device(const char* call, hipError_t e) {
    snprintf(worker_err, sizeof worker_err, "%s: hipSetDevice: %s", call, hipGetErrorString(e));
    (void)hipGetLastError();
    return DBLP_EHIP;
}

#define COUNT_LIMIT (1ull << 31)
static u32 type_bytes(int type) { return type == DBLP_F32 ? 4 : 2; }
static bool bad_type(int type) { return type != DBLP_F32 && type != DBLP_BF16 && type != DBLP_F16; }
static bool off(const void* p, u32 bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }
static u64 round_up(u64 n, u64 to) { return (n + to - 1) / to * to; }

#define REFUSE_IF(cond, why) do { if (cond) return refuse(call, why); } while (0)

static int take_drop(const char* call, const dblp_drop* h, Mask* m) {
    *m = Mask{0, 0, nullptr, 0, 1.0f};
    if (!h) return DBLP_OK;
    REFUSE_IF(!(h->p >= 0.0 && h->p <= 1.0), "p must be in 0..1");
    REFUSE_IF(off(h->d_draw, 8), "d_draw must be 8-byte aligned");
    const u32 limit = (u32)rint(65536.0 * h->p);
    *m = Mask{h->seed, h->draw, (const u64*)h->d_draw, limit, limit < 65536 ? (float)(65536.0 / (65536.0 - limit)) : 0.0f};
    return DBLP_OK;
}

// Calls f(Groups) for launches of fewer than 2^31 groups each.
template <class F>
static void each_launch(u64 rows, u32 cols, F f) {
    const u32 per_row = (u32)((cols + 7ull) / 8);
    const u64 most = (COUNT_LIMIT - 1) / per_row;
    for (u64 row0 = 0; row0 < rows; row0 += most) {
        const u64 n = rows - row0 < most ? rows - row0 : most;
        f(Groups{row0, (u32)(n * per_row), cols, Divider::by(per_row)});
    }
}
static dim3 blocks_of(const Groups& s, u32 each = 1) { return dim3((s.n + 256 * each - 1) / (256 * each)); }

template <int N> struct Int { static constexpr int value = N; };

template <class F>
static void by_type(int type, F f) {
    if (type == DBLP_F32) f(F32());
    else if (type == DBLP_BF16) f(BF16());
    else f(F16());
}

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
    by_type(table_type, [&](auto st) {
        by_type(out_type, [&](auto tt) {
            typedef decltype(st) S;
            typedef decltype(tt) T;
            each_launch(n_tokens, dim, [&](Groups s) {
                const bool whole = dim % 8 == 0;
                const auto kernel = m.limit ? (whole ? embed_groups<S, T, true, true> : embed_groups<S, T, true, false>) : (whole ? embed_groups<S, T, false, true> : embed_groups<S, T, false, false>);
                hipLaunchKernelGGL(kernel, blocks_of(s, GROUPS_EACH), dim3(256), 0, (hipStream_t)stream, s, m, d_tokens, (const typename S::elem*)d_table, (u64)table_stride, (u64)vocab, scale,
                                   d_positions, (const typename S::elem*)d_pos_table, (u64)pos_stride, (u64)n_positions, (typename T::elem*)d_out, (u64)out_stride);
            });
        });
    });
    return launched(call);
}

// How the places of a batch are sorted and cut, and where its intermediate results lie in the workspace.
struct GradPlan {
    bool short_batch;            // one launch
    u32 len, pieces, passes, bits, tile, tiles;
    u64 keys[2], places[2], hist, present, chains, n_chains, chain, bytes;
};

static GradPlan grad_plan(u64 n, u64 vocab, u32 dim) {
    GradPlan p = {};
    p.short_batch = n <= GRAD_SHORT;
    p.bytes = 256;
    if (p.short_batch) return p;
    const u64 groups = ((u64)dim + 7) / 8;
    u32 bits = 0;
    while ((vocab >> bits) != 0) ++bits;                 // keys run to vocab itself
    p.passes = (bits + 8) / 9;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.len = n <= SORT_BLOCK_MOST ? 8 : 16;
    p.pieces = (u32)((n + p.len - 1) / p.len);
    p.tile = (u32)round_up((n + SORT_TILES - 1) / SORT_TILES, SORT_STEP);
    p.tiles = (u32)((n + p.tile - 1) / p.tile);
    u64 at = 0;
    const auto take = [&](u64 bytes) { const u64 here = at; at += round_up(bytes, 256); return here; };
    for (int i = 0; i < 2; ++i) { p.keys[i] = take(4 * (n + 2 * KEY_PAD)) + 4 * KEY_PAD; p.places[i] = take(4 * (n + KEY_PAD)); }
    p.hist = take(4ull * SORT_TILES * BINS);
    p.present = take(vocab);
    p.chains = take(4ull * p.pieces);
    p.n_chains = take(4);
    p.chain = take((u64)p.pieces * 2 * groups * 8 * 4);
    p.bytes = at;
    return p;
}

extern "C" uint64_t dblp_embed_grad_workspace(uint64_t n_tokens, uint64_t vocab, uint32_t dim) {
    if (n_tokens >= COUNT_LIMIT || vocab == 0 || vocab >= COUNT_LIMIT || dim == 0 || dim >= COUNT_LIMIT) return 0;
    return grad_plan(n_tokens, vocab, dim).bytes;
}

// The launches that put the places in order and, unless the result is in place, write the rows that have no token.
// Returns which of the two buffers holds the sorted keys and places.
static int sort_places(const GradPlan& p, const int64_t* tokens, u32 n, u32 dim, const Result& out, uint8_t* ws, hipStream_t stream) {
    const bool in_place = out.base == out.grad;
    const SortShape q = {n, p.passes, p.bits, out.vocab};
    u32* const n_chains = (u32*)(ws + p.n_chains);
    const u32 per_row = (u32)((dim + 7ull) / 8);
    const auto rows = [&](u64 row0, u64 count) { return Groups{row0, (u32)(count * per_row), dim, Divider::by(per_row)}; };
    // one launch's share of the rows fits 31 bits of groups, or they are filled apart
    const bool beside = !in_place && out.vocab * per_row < COUNT_LIMIT;
    if (n <= SORT_BLOCK_MOST) {
        const Groups s = rows(0, beside ? out.vocab : 0);
        if (!in_place && !beside)
            each_launch(out.vocab, dim, [&](Groups a) { hipLaunchKernelGGL(fill_rows, blocks_of(a), dim3(256), 0, stream, a, out, (const uint8_t*)nullptr); });
        const u32 fillers = (u32)((s.n + 4095ull) / 4096);
        hipLaunchKernelGGL(sort_one_block, dim3(1 + fillers), dim3(1024), 0, stream, q, tokens, (u32*)(ws + p.keys[0]), (u32*)(ws + p.places[0]), n_chains, s, out);
        return 0;
    }
    uint8_t* const present = ws + p.present;
    u32* const hist = (u32*)(ws + p.hist);
    int to = 0;
    for (u32 pass = 0; pass < p.passes; ++pass) {
        const SortFrom from = {pass ? nullptr : tokens, pass ? (u32*)(ws + p.keys[to ^ 1]) : nullptr, pass ? (u32*)(ws + p.places[to ^ 1]) : nullptr};
        const bool first = pass == 0, last = pass + 1 == p.passes;
        const u64 half = out.vocab / 2;
        const Groups lower = rows(0, beside && last && !first ? half : 0), upper = rows(half, beside && last && !first ? out.vocab - half : 0);
        const u32 clear = first && !in_place ? (u32)(round_up(out.vocab, 256) / 4) : 0;
        const auto fillers = [&](u64 groups, u64 words) { const u64 b = (groups + 1023) / 1024 + (words + 1023) / 1024; return (u32)b; };
        hipLaunchKernelGGL(sort_count, dim3(p.tiles + fillers(lower.n, clear)), dim3(256), 0, stream, q, from, pass * p.bits, p.tile, p.tiles, hist, n_chains, (u32*)present, clear, lower, out, (const uint8_t*)present);
        hipLaunchKernelGGL(sort_move, dim3(p.tiles + fillers(upper.n, 0)), dim3(256), 0, stream, q, from, pass * p.bits, p.tile, p.tiles, (const u32*)hist, (u32*)(ws + p.keys[to]), (u32*)(ws + p.places[to]),
                           first && !in_place ? present : (uint8_t*)nullptr, upper, out, (const uint8_t*)present);
        to ^= 1;
    }
    if (!in_place && (!beside || p.passes == 1))
        each_launch(out.vocab, dim, [&](Groups a) { hipLaunchKernelGGL(fill_rows, blocks_of(a), dim3(256), 0, stream, a, out, (const uint8_t*)present); });
    return to ^ 1;
}

extern "C" int dblp_embed_grad(int device, void* stream, const int64_t* d_tokens, uint64_t n_tokens, uint32_t dim, uint64_t vocab,
                               float scale, const dblp_drop* h_drop, const void* d_dy, uint64_t dy_stride, int dy_type,
                               const float* d_base, uint64_t base_stride, float* d_grad, uint64_t grad_stride,
                               void* d_workspace, uint64_t workspace_bytes) {
    const char* call = "embed_grad";
    REFUSE_IF(bad_type(dy_type), "unknown type");
    REFUSE_IF(dim == 0 || dim >= COUNT_LIMIT || vocab == 0 || vocab >= COUNT_LIMIT || n_tokens >= COUNT_LIMIT, "size out of range");
    REFUSE_IF(!d_grad || (n_tokens && (!d_tokens || !d_dy)), "null pointer");
    REFUSE_IF(off(d_tokens, 8) || off(d_dy, type_bytes(dy_type)) || off(d_base, 4) || off(d_grad, 4), "misaligned pointer");
    REFUSE_IF(vocab > 1 && grad_stride < dim, "the gradient's rows overlap");
    REFUSE_IF(d_base == d_grad && vocab > 1 && base_stride != grad_stride, "in place, the strides must be equal");
    REFUSE_IF(!d_workspace || off(d_workspace, 256) || workspace_bytes < dblp_embed_grad_workspace(n_tokens, vocab, dim), "workspace missing, misaligned or too small");
    Mask m;
    if (const int rc = take_drop(call, h_drop, &m)) return rc;
    OnDevice on(device);
    if (on.err != hipSuccess) return no_device(call, on.err);
    const hipStream_t st = (hipStream_t)stream;
    const Result out = {d_base, base_stride, d_grad, grad_stride, vocab, scale};
    const GradPlan p = grad_plan(n_tokens, vocab, dim);
    const u32 n = (u32)n_tokens, groups = (u32)((dim + 7ull) / 8);
    if (p.short_batch) {
        by_type(dy_type, [&](auto tt) {
            typedef decltype(tt) T;
            const bool whole = dim % 8 == 0;
            const auto kernel = m.limit ? (whole ? grad_short<T, true, true> : grad_short<T, true, false>) : (whole ? grad_short<T, false, true> : grad_short<T, false, false>);
            u32 lead = (u32)((n * ((groups + 63ull) / 64) + 3) / 4);
            const auto go = [&](Groups s) {
                const u32 fill = (u32)((s.n + 256ull * FILL_EACH - 1) / (256 * FILL_EACH));
                if (lead + fill)
                    hipLaunchKernelGGL(kernel, dim3(lead + fill), dim3(256), 0, st, d_tokens, n, dim, groups, lead, s, out, m, (const typename T::elem*)d_dy, (u64)dy_stride);
                lead = 0;
            };
            if (d_base == d_grad) go(Groups{0, 0, dim, Divider::by(groups)});
            else each_launch(vocab, dim, go);
        });
        return launched(call);
    }
    uint8_t* const ws = (uint8_t*)d_workspace;
    const int at = sort_places(p, d_tokens, n, dim, out, ws, st);
    u32 *const keys = (u32*)(ws + p.keys[at]), *const places = (u32*)(ws + p.places[at]), *const chains = (u32*)(ws + p.chains), *const n_chains = (u32*)(ws + p.n_chains);
    float* const chain = (float*)(ws + p.chain);
    by_type(dy_type, [&](auto tt) {
        typedef decltype(tt) T;
        each_launch(p.pieces, dim, [&](Groups s) {
            const auto pick = [&](auto len, auto whole) { return m.limit ? grad_pieces<T, true, decltype(len)::value, decltype(whole)::value> : grad_pieces<T, false, decltype(len)::value, decltype(whole)::value>; };
            const auto kernel = p.len == 8 ? (dim % 8 ? pick(Int<8>(), Int<0>()) : pick(Int<8>(), Int<1>())) : (dim % 8 ? pick(Int<16>(), Int<0>()) : pick(Int<16>(), Int<1>()));
            hipLaunchKernelGGL(kernel, blocks_of(s), dim3(256), 0, st, (const u32*)keys, (const u32*)places, s, out, m, (const typename T::elem*)d_dy, (u64)dy_stride, chain, chains, n_chains);
        });
    });
    hipLaunchKernelGGL(grad_chains, dim3(p.pieces < 256 ? p.pieces : 256, (groups + 15) / 16), dim3(256), 0, st, (const u32*)keys, n, p.len, dim, groups, out, (const float*)chain, (const u32*)chains, (const u32*)n_chains);
    return launched(call);
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
    by_type(type, [&](auto tt) {
        typedef decltype(tt) T;
        typedef const typename T::elem* in;
        each_launch(rows, cols, [&](Groups s) {
            const bool whole = cols % 8 == 0;
            const auto kernel = d_residual ? (whole ? dropout_groups<T, true, true> : dropout_groups<T, true, false>) : (whole ? dropout_groups<T, false, true> : dropout_groups<T, false, false>);
            hipLaunchKernelGGL(kernel, blocks_of(s, GROUPS_EACH), dim3(256), 0, (hipStream_t)stream, s, m, (in)d_x, (u64)x_stride, (in)d_residual, (u64)residual_stride, (typename T::elem*)d_y, (u64)y_stride);
        });
    });
    return launched(call);
}

extern "C" uint64_t dblp_logits_workspace(uint64_t n_tokens, uint32_t vocab) {
    if (n_tokens >= COUNT_LIMIT || vocab == 0 || vocab >= COUNT_LIMIT) return 0;
    return round_up(n_tokens * sizeof(TokenPart), 256) + 256;
}

extern "C" int dblp_token_logprobs(int device, void* stream, uint64_t n_tokens, uint32_t vocab, const void* d_logits,
                                   uint64_t logits_stride, int type, const int64_t* d_targets, float* d_logp, float* d_lse,
                                   void* d_workspace, uint64_t workspace_bytes) {
    const char* call = "token_logprobs";
    REFUSE_IF(bad_type(type), "unknown type");
    REFUSE_IF(vocab == 0 || vocab >= COUNT_LIMIT || n_tokens >= COUNT_LIMIT, "size out of range");
    REFUSE_IF(n_tokens && (!d_logits || !d_targets || !d_logp), "null pointer");
    REFUSE_IF(off(d_logits, type_bytes(type)) || off(d_targets, 8) || off(d_logp, 4) || off(d_lse, 4), "misaligned pointer");
    REFUSE_IF(!d_workspace || off(d_workspace, 256) || workspace_bytes < dblp_logits_workspace(n_tokens, vocab), "workspace missing, misaligned or too small");
    if (n_tokens == 0) return DBLP_OK;
    OnDevice on(device);
    if (on.err != hipSuccess) return no_device(call, on.err);
    by_type(type, [&](auto tt) {
        typedef decltype(tt) T;
        const auto kernel = logprob_rows<T, 512>;
        hipLaunchKernelGGL(kernel, dim3((u32)n_tokens), dim3(512), 0, (hipStream_t)stream, (const typename T::elem*)d_logits, (u64)logits_stride, vocab, d_targets, d_logp, d_lse);
    });
    return launched(call);
}

extern "C" int dblp_policy_loss(int device, void* stream, uint64_t n_tokens, uint32_t vocab, const void* d_logits,
                                uint64_t logits_stride, int type, const int64_t* d_targets, const float* d_advantages,
                                const float* d_weights, const float* d_old_logp, const float* d_ref_logp, float clip_low,
                                float clip_high, float kl_coef, float grad_scale, void* d_dlogits, uint64_t dlogits_stride,
                                float* d_logp, float* d_stats, void* d_workspace, uint64_t workspace_bytes) {
    const char* call = "policy_loss";
    REFUSE_IF(bad_type(type), "unknown type");
    REFUSE_IF(vocab == 0 || vocab >= COUNT_LIMIT || n_tokens >= COUNT_LIMIT, "size out of range");
    REFUSE_IF(!d_stats || (n_tokens && (!d_logits || !d_targets || !d_advantages || !d_weights)), "null pointer");
    REFUSE_IF(off(d_logits, type_bytes(type)) || off(d_dlogits, type_bytes(type)) || off(d_targets, 8) || off(d_advantages, 4) || off(d_weights, 4) || off(d_old_logp, 4) ||
              off(d_ref_logp, 4) || off(d_logp, 4) || off(d_stats, 4), "misaligned pointer");
    REFUSE_IF(!(clip_low >= 0.0f && clip_low <= 1.0f && clip_high >= 0.0f && isfinite(clip_high)), "clip_low must be in 0..1 and clip_high at least 0");
    REFUSE_IF(!isfinite(kl_coef) || !isfinite(grad_scale), "kl_coef and grad_scale must be finite");
    REFUSE_IF(d_dlogits && n_tokens > 1 && dlogits_stride < vocab, "the gradient's rows overlap");
    REFUSE_IF(d_dlogits == d_logits && n_tokens > 1 && dlogits_stride != logits_stride, "in place, the strides must be equal");
    REFUSE_IF(!d_workspace || off(d_workspace, 256) || workspace_bytes < dblp_logits_workspace(n_tokens, vocab), "workspace missing, misaligned or too small");
    OnDevice on(device);
    if (on.err != hipSuccess) return no_device(call, on.err);
    const Policy p = {d_targets, d_advantages, d_weights, d_old_logp, d_ref_logp, clip_low, clip_high, kl_coef, grad_scale};
    TokenPart* parts = (TokenPart*)d_workspace;
    if (n_tokens)
        by_type(type, [&](auto tt) {
            typedef decltype(tt) T;
            const auto kernel = policy_rows<T, 512>;
            hipLaunchKernelGGL(kernel, dim3((u32)n_tokens), dim3(512), 0, (hipStream_t)stream, p, (const typename T::elem*)d_logits, (u64)logits_stride, vocab,
                               (typename T::elem*)d_dlogits, (u64)dlogits_stride, d_logp, parts);
        });
    hipLaunchKernelGGL(policy_sums, dim3(1), dim3(1024), 0, (hipStream_t)stream, (const TokenPart*)parts, (u32)n_tokens, kl_coef, d_stats);
    return launched(call);
}
