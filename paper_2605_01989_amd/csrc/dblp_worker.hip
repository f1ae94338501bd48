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

struct F32 {
    typedef float elem;
    static __device__ __forceinline__ float get(const float* p) { return *p; }
    static __device__ __forceinline__ void put(float* p, float v) { *p = v; }
    static __device__ __forceinline__ void get8(const float* p, float (&v)[8]) {
        const f4v a = *(const f4v_a4*)p, b = *(const f4v_a4*)(p + 4);
        for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
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
    static __device__ __forceinline__ float get(const E* p) { return (float)*p; }
    static __device__ __forceinline__ void put(E* p, float v) { *p = (E)v; }
    static __device__ __forceinline__ void get8(const E* p, float (&v)[8]) {
        const f8v f = __builtin_convertvector(__builtin_bit_cast(V8, (u4v)*(const u4v_a2*)p), f8v);
        for (int i = 0; i < 8; ++i) v[i] = f[i];
    }
    static __device__ __forceinline__ void put8(E* p, const float (&v)[8]) {
        const f8v f = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
        *(u4v_a2*)p = __builtin_bit_cast(u4v, __builtin_convertvector(f, V8));
    }
};
typedef Half<__bf16, bf8v> BF16;
typedef Half<_Float16, h8v> F16;

// Columns [c, c + 8) of a row of `cols`; those past the end read as zero and are not written.
template <class T>
__device__ __forceinline__ void load_group(const typename T::elem* row, u32 c, u32 cols, float (&v)[8]) {
    if (c + 8 <= cols) { T::get8(row + c, v); return; }
    for (u32 i = 0; i < 8; ++i) v[i] = c + i < cols ? T::get(row + c + i) : 0.0f;
}
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

template <class T, bool RES>
__global__ __launch_bounds__(256) void dropout_groups(Groups s, Mask m, const typename T::elem* x, u64 x_stride,
                                                      const typename T::elem* res, u64 res_stride, typename T::elem* y, u64 y_stride) {
    const u32 i = blockIdx.x * 256 + threadIdx.x;
    if (i >= s.n) return;
    const u32 r = s.per_row.of(i), c = (i - r * s.per_row.d) * 8;
    const u64 row = s.row0 + r;
    float v[8], w[8];
    load_group<T>(x + row * x_stride, c, s.cols, v);
    if (RES) load_group<T>(res + row * res_stride, c, s.cols, w);
    gate8(m, draw_of(m), s.row0 * s.per_row.d + i, v);
    if (RES) for (int k = 0; k < 8; ++k) v[k] += w[k];
    store_group<T>(y + row * y_stride, c, s.cols, v);
}

template <class S, class T, bool DROP>
__global__ __launch_bounds__(256) void embed_groups(Groups s, Mask m, const int64_t* __restrict__ tokens, const typename S::elem* __restrict__ table, u64 table_stride, u64 vocab,
                                                    float scale, const int64_t* __restrict__ positions, const typename S::elem* __restrict__ pos_table, u64 pos_stride, u64 n_pos,
                                                    typename T::elem* __restrict__ out, u64 out_stride) {
    const u32 i = blockIdx.x * 256 + threadIdx.x;
    if (i >= s.n) return;
    const u32 r = s.per_row.of(i), c = (i - r * s.per_row.d) * 8;
    const u64 row = s.row0 + r;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    const u64 tok = (u64)tokens[row];
    if (tok < vocab) {
        load_group<S>(table + tok * table_stride, c, s.cols, v);
        for (int k = 0; k < 8; ++k) v[k] *= scale;
    }
    if (positions) {
        const u64 at = (u64)positions[row];
        if (at < n_pos) {
            float w[8];
            load_group<S>(pos_table + at * pos_stride, c, s.cols, w);
            for (int k = 0; k < 8; ++k) v[k] += w[k];
        }
    }
    if (DROP) gate8(m, draw_of(m), s.row0 * s.per_row.d + i, v);
    store_group<T>(out + row * out_stride, c, s.cols, v);
}

// ------------------------------------------------------------------------------------------
// gradient of the embedding
// ------------------------------------------------------------------------------------------
// grad = base, or zeros
__global__ __launch_bounds__(256) void grad_begin(Groups s, const float* base, u64 base_stride, float* grad, u64 grad_stride) {
    const u32 i = blockIdx.x * 256 + threadIdx.x;
    if (i >= s.n) return;
    const u32 r = s.per_row.of(i), c = (i - r * s.per_row.d) * 8;
    const u64 row = s.row0 + r;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (base) load_group<F32>(base + row * base_stride, c, s.cols, v);
    store_group<F32>(grad + row * grad_stride, c, s.cols, v);
}

// A block stands for one token place and some columns.  The block of a token's first place adds up the rows of all its
// places, in order; the others end.
template <class T, bool DROP>
__global__ __launch_bounds__(256) void grad_by_first(const int64_t* __restrict__ tokens, u32 n, u32 cols, u32 groups, u64 vocab, float scale, Mask m,
                                                     const typename T::elem* __restrict__ dy, u64 dy_stride, float* grad, u64 grad_stride) {
    __shared__ u32 places[256];
    __shared__ u32 in_wave[4];
    const u32 t = blockIdx.x, tid = threadIdx.x, nt = blockDim.x;
    const u64 tok = (u64)tokens[t];
    if (tok >= vocab) return;
    int earlier = 0;
    for (u32 j = tid; j < t; j += nt) earlier |= (u64)tokens[j] == tok;
    if (__syncthreads_or(earlier)) return;
    const u32 c = (blockIdx.y * nt + tid) * 8;
    const u64 draw = DROP ? draw_of(m) : 0;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (u32 from = t; from < n; from += nt) {
        const bool hit = from + tid < n && (u64)tokens[from + tid] == tok;
        const u64 hits = __ballot(hit);
        if ((tid & 63) == 0) in_wave[tid >> 6] = (u32)__popcll(hits);
        __syncthreads();
        u32 before = 0, all = 0;
        for (u32 w = 0; w < nt / 64; ++w) { if (w < tid >> 6) before += in_wave[w]; all += in_wave[w]; }
        if (hit) places[before + (u32)__popcll(hits & ((1ull << (tid & 63)) - 1))] = from + tid;
        __syncthreads();
        if (c < cols)
            for (u32 k = 0; k < all; ++k) {
                const u64 row = places[k];
                float v[8];
                load_group<T>(dy + row * dy_stride, c, cols, v);
                if (DROP) gate8(m, draw, row * groups + c / 8, v);
                for (int e = 0; e < 8; ++e) sum[e] += v[e];
            }
        __syncthreads();
    }
    if (c >= cols) return;
    float v[8];
    float* row = grad + tok * grad_stride;
    load_group<F32>(row, c, cols, v);
    for (int e = 0; e < 8; ++e) v[e] += scale * sum[e];
    store_group<F32>(row, c, cols, v);
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
        if (c + 8 <= n) T::get8(row + c, v);
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
static dim3 blocks_of(const Groups& s) { return dim3((s.n + 255) / 256); }

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
                const auto kernel = m.limit ? embed_groups<S, T, true> : embed_groups<S, T, false>;
                hipLaunchKernelGGL(kernel, blocks_of(s), dim3(256), 0, (hipStream_t)stream, s, m, d_tokens, (const typename S::elem*)d_table, (u64)table_stride, (u64)vocab, scale,
                                   d_positions, (const typename S::elem*)d_pos_table, (u64)pos_stride, (u64)n_positions, (typename T::elem*)d_out, (u64)out_stride);
            });
        });
    });
    return launched(call);
}

extern "C" uint64_t dblp_embed_grad_workspace(uint64_t n_tokens, uint64_t vocab, uint32_t dim) {
    if (n_tokens >= COUNT_LIMIT || vocab == 0 || vocab >= COUNT_LIMIT || dim == 0 || dim >= COUNT_LIMIT) return 0;
    return 256;
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
    const u32 groups = (dim + 7) / 8;
    if (d_base != d_grad)
        each_launch(vocab, dim, [&](Groups s) {
            hipLaunchKernelGGL(grad_begin, blocks_of(s), dim3(256), 0, (hipStream_t)stream, s, d_base, (u64)base_stride, d_grad, (u64)grad_stride);
        });
    if (n_tokens)
        by_type(dy_type, [&](auto tt) {
            typedef decltype(tt) T;
            const u32 nt = groups >= 256 ? 256 : (groups + 63) / 64 * 64;
            const auto kernel = m.limit ? grad_by_first<T, true> : grad_by_first<T, false>;
            hipLaunchKernelGGL(kernel, dim3((u32)n_tokens, (groups + nt - 1) / nt), dim3(nt), 0, (hipStream_t)stream, d_tokens, (u32)n_tokens, dim, groups, (u64)vocab, scale, m,
                               (const typename T::elem*)d_dy, (u64)dy_stride, d_grad, (u64)grad_stride);
        });
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
            const auto kernel = d_residual ? dropout_groups<T, true> : dropout_groups<T, false>;
            hipLaunchKernelGGL(kernel, blocks_of(s), dim3(256), 0, (hipStream_t)stream, s, m, (in)d_x, (u64)x_stride, (in)d_residual, (u64)residual_stride, (typename T::elem*)d_y, (u64)y_stride);
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
