// Logits of a worker's training step on gfx950 (MI355X): log probabilities of given tokens, and the clipped policy loss with its gradient.
// Kernels and the C-ABI declared in include/dblp_worker.h.
//
// A row is read once: its largest value and the sum of its exponentials are found together, and where a gradient is wanted the row
// stays in registers between the sum and the gradient (50257 16-bit values: 100 KB of a CU's 512 KB, two rows a CU).
// Memory bounds all of it: log probabilities of 8192 x 50257 16-bit values, 30 % of the rows masked, take 90 us (6.4 TB/s, the rate of a large read), their policy loss
// 276 us (583 MB read, 826 written: 5.1 TB/s, where a large copy reaches 5.2).  A row of 50257 alone is bound by its launch: 5 us of the GPU's time.
#include "worker_common.h"

// ------------------------------------------------------------------------------------------
// a row's largest value m and s = sum of exp(x - m).  Nothing met: (-inf, 0), and nothing else has s = 0: a NaN makes s NaN, whatever m is
// ------------------------------------------------------------------------------------------
#define LOG2E 1.4426950408889634f

struct Soft { float m, s; };
__device__ __forceinline__ float shift_of(float m) { return m == -INFINITY ? 0.0f : m; }     // exp(-inf - -inf) would be NaN
// x - shift is exact where it matters (x near the largest); the product with log2 e is off by |x - shift| 2^-24, the function by one step.
__device__ __forceinline__ float exp_of(float x, float shift) { return __builtin_amdgcn_exp2f((x - shift) * LOG2E); }
__device__ __forceinline__ Soft soft_join(Soft a, Soft b) {
    const float m = fmaxf(a.m, b.m), at = shift_of(m);
    return {m, a.s * exp_of(a.m, at) + b.s * exp_of(b.m, at)};
}
__device__ __forceinline__ Soft soft_wave(Soft a) {
#pragma clang fp contract(off)                             // a lane's product is rounded before it meets another's: all lanes find the same sum
    float m = a.m;
#pragma unroll
    for (int d = 1; d < WAVE; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
    float s = a.s * exp_of(a.m, shift_of(m));              // scaled once
#pragma unroll
    for (int d = 1; d < WAVE; d <<= 1) s += __shfl_xor(s, d);
    return {m, s};
}
// The whole block's, to all of its threads.  `part`: one entry for each wave.
template <int NT>
__device__ __forceinline__ Soft soft_block(Soft a, Soft* part) {
    a = soft_wave(a);
    if (NT == WAVE) return a;
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = a;
    __syncthreads();
    a = part[0];
#pragma unroll
    for (int w = 1; w < NT / WAVE; ++w) a = soft_join(a, part[w]);
    return a;
}
// N vectors of W values at once: one largest value, one change of scale.
template <class V, int W, int N>
__device__ __forceinline__ void soft_add(Soft& a, const typename V::raw (&r)[N]) {
    float v[N][W], m = a.m;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        V::open(r[j], v[j]);
#pragma unroll
        for (int i = 0; i < W; i += 2) m = fmaxf(fmaxf(v[j][i], v[j][i + 1]), m);
    }
    const float at = shift_of(m);
    float s = a.s * exp_of(a.m, at);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < W; ++i) t += exp_of(v[j][i], at);
        s += t;
    }
    a = {m, s};
}

template <class T> struct Wide { static constexpr int W = sizeof(typename T::elem) == 4 ? 4 : 8; };      // 16 bytes

// A row as vectors of W values from the first place whose address is a multiple of four (16-byte accesses at odd multiples of two run at two thirds of the rate: 8192
// rows of 50257 16-bit values take 163 us to read, of 50258 127), and single values: a head of at most one, a tail of fewer than W.
struct Cut { u32 head, vecs, singles; };
template <class T>
__device__ __forceinline__ Cut cut_row(const typename T::elem* row, u32 n) {
    constexpr u32 W = Wide<T>::W;
    const u32 head = ((uintptr_t)row & 2) ? 1 : 0, vecs = (n - head) / W;
    return {head, vecs, n - vecs * W};
}
template <int W>
__device__ __forceinline__ u32 place_of_single(const Cut& c, u32 i) { return i < c.head ? i : i + c.vecs * W; }

template <class V, int W>
__device__ __forceinline__ typename V::raw no_logits() {
    float v[W];
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = -INFINITY;
    return V::pack(v);
}
__device__ __forceinline__ void soft_add_one(Soft& a, float x) { a = soft_join(a, {x, x == -INFINITY ? 0.0f : 1.0f}); }

// A thread's share of vectors [lo, hi) of a row that is only read: STREAM vectors in flight.
#define STREAM 4
template <class T, int NT, bool FAR>
__device__ __forceinline__ void soft_vecs(Soft& a, const typename T::elem* body, u32 lo, u32 hi) {
    constexpr int W = Wide<T>::W;
    typedef Vec<T, W> V;
    const u32 whole = lo + (hi - lo) / (NT * STREAM) * (NT * STREAM);
    typename V::raw r[STREAM];
    for (u32 i = lo; i < whole; i += NT * STREAM) {
#pragma unroll
        for (int j = 0; j < STREAM; ++j) r[j] = FAR ? V::load_far(body + (u64)(i + j * NT + threadIdx.x) * W) : V::load(body + (u64)(i + j * NT + threadIdx.x) * W);
        soft_add<V, W, STREAM>(a, r);
    }
    if (whole < hi) {
#pragma unroll
        for (int j = 0; j < STREAM; ++j) {
            const u32 i = whole + j * NT + threadIdx.x;
            r[j] = no_logits<V, W>();
            if (i < hi) r[j] = FAR ? V::load_far(body + (u64)i * W) : V::load(body + (u64)i * W);
        }
        // as many as hold anything: rows shorter than a step are bound by these instructions (160 MB of rows of 256 16-bit values 107 us, 178 with all four)
        if (hi - whole > 2 * NT) soft_add<V, W, STREAM>(a, r);
        else {
            const typename V::raw first[1] = {r[0]}, second[1] = {r[1]};
            soft_add<V, W, 1>(a, first);
            if (hi - whole > NT) soft_add<V, W, 1>(a, second);
        }
    }
}
template <class T, int NT, bool FAR>
__device__ __forceinline__ Soft soft_row(const typename T::elem* row, u32 n) {
    constexpr int W = Wide<T>::W;
    const Cut c = cut_row<T>(row, n);
    Soft a = {-INFINITY, 0.0f};
    const float single = threadIdx.x < c.singles ? (float)row[place_of_single<W>(c, threadIdx.x)] : -INFINITY;
    soft_vecs<T, NT, FAR>(a, row + c.head, 0, c.vecs);
    soft_add_one(a, single);
    return a;
}

// Log probability of a logit x.  A score is a difference of numbers of ten or twenty, and policies' ratios are differences of scores: the last sums are fp64, and so is
// the logarithm, by the series of 2 artanh f, f = (m - 1) / (m + 1), of a number m in sqrt(1/2) .. sqrt(2) (the first term left out is 2^-39 of the sum).  One thread a row
// takes it.  The largest value and the logarithm are not added up first: in a row of the type's lowest value the logarithm would be lost.
__device__ __forceinline__ double log_of(float s) {
    double m = __builtin_amdgcn_frexp_mantf(s), e = __builtin_amdgcn_frexp_expf(s);
    if (m < 0.7071067811865476) { m *= 2.0; e -= 1.0; }
    const double f = (m - 1.0) / (m + 1.0), q = f * f;
    double t = 1.0 / 13;
    t = fma(t, q, 1.0 / 11); t = fma(t, q, 1.0 / 9); t = fma(t, q, 1.0 / 7); t = fma(t, q, 1.0 / 5); t = fma(t, q, 1.0 / 3); t = fma(t, q, 1.0);
    return fma(e, 0.6931471805599453, 2.0 * f * t);
}
__device__ __forceinline__ double logp_of(float x, Soft a) { return ((double)x - (double)a.m) - log_of(a.s); }

template <class T, int NT, bool FAR>
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
    const float x = threadIdx.x == 0 ? (float)row[at] : 0.0f;
    const Soft a = soft_block<NT>(soft_row<T, NT, FAR>(row, vocab), part);
    if (threadIdx.x == 0) {
        if (lse) lse[t] = (float)((double)a.m + log_of(a.s));
        logp[t] = a.s == 0.0f ? -INFINITY : (float)logp_of(x, a);
    }
}

// Few long rows: blocks share a row.  This launch finds (m, s) of each share and keeps the target's logit (the next launch may write the gradient over it), the next
// one joins them.
#define SHARES_MOST 32
#define SHARE_NT 256
struct Shares { u32 n, vecs; };                  // shares of a row, vectors of each
template <class T>
__device__ __forceinline__ void share_of(const Cut& c, const Shares& q, u32 s, u32* lo, u32* hi) {
    *lo = s * q.vecs < c.vecs ? s * q.vecs : c.vecs;
    *hi = c.vecs - *lo < q.vecs ? c.vecs : *lo + q.vecs;
}
// (`weights`: a row of weight zero is not read; null: all rows with a target are)
template <class T>
__global__ __launch_bounds__(SHARE_NT) void soft_shares(Shares q, const typename T::elem* __restrict__ logits, u64 stride, u32 vocab, const int64_t* __restrict__ targets, const float* __restrict__ weights,
                                                        Soft* __restrict__ softs, float* __restrict__ chosen) {
    constexpr int W = Wide<T>::W;
    __shared__ Soft part[SHARE_NT / WAVE];
    const u32 s = blockIdx.x, t = blockIdx.y;
    if ((u64)targets[t] >= vocab || (weights && weights[t] == 0.0f)) return;
    const typename T::elem* row = logits + (u64)t * stride;
    const Cut c = cut_row<T>(row, vocab);
    u32 lo, hi;
    share_of<T>(c, q, s, &lo, &hi);
    Soft a = {-INFINITY, 0.0f};
    const float single = s == 0 && threadIdx.x < c.singles ? (float)row[place_of_single<W>(c, threadIdx.x)] : -INFINITY;
    soft_vecs<T, SHARE_NT, false>(a, row + c.head, lo, hi);
    soft_add_one(a, single);
    a = soft_block<SHARE_NT>(a, part);
    if (threadIdx.x == 0) {
        softs[t * q.n + s] = a;
        if (s == 0) chosen[t] = (float)row[targets[t]];
    }
}
// A row's (m, s), to every lane of a wave.
__device__ __forceinline__ Soft soft_of_row(const Soft* softs, u32 t, u32 n) {
    const u32 lane = threadIdx.x & 63;
    return soft_wave(lane < n ? softs[t * n + lane] : Soft{-INFINITY, 0.0f});
}
// The same by one thread, with the same bits: the sums of the butterfly above as a tree (entries past n add zero).
__device__ __forceinline__ Soft soft_of_row_alone(const Soft* softs, u32 t, u32 n) {
#pragma clang fp contract(off)
    Soft part[SHARES_MOST];
    float m = -INFINITY, s[SHARES_MOST];
#pragma unroll
    for (u32 i = 0; i < SHARES_MOST; ++i) part[i] = softs[t * n + (i < n ? i : n - 1)];
#pragma unroll
    for (u32 i = 0; i < SHARES_MOST; ++i) m = fmaxf(m, part[i].m);
#pragma unroll
    for (u32 i = 0; i < SHARES_MOST; ++i) s[i] = i < n ? part[i].s * exp_of(part[i].m, shift_of(m)) : 0.0f;
#pragma unroll
    for (u32 d = 1; d < SHARES_MOST; d <<= 1)
#pragma unroll
        for (u32 i = 0; i < SHARES_MOST; i += 2 * d) s[i] += s[i + d];
    return {m, s[0]};
}
__global__ __launch_bounds__(64) void logprob_join(Shares q, u32 vocab, const int64_t* __restrict__ targets, const Soft* __restrict__ softs, const float* __restrict__ chosen,
                                                   float* __restrict__ logp, float* __restrict__ lse) {
    const u32 t = blockIdx.x;
    const u64 at = (u64)targets[t];
    if (at >= vocab) {
        if (threadIdx.x == 0) { logp[t] = 0.0f; if (lse) lse[t] = 0.0f; }
        return;
    }
    const Soft a = soft_of_row(softs, t, q.n);
    if (threadIdx.x) return;
    if (lse) lse[t] = (float)((double)a.m + log_of(a.s));
    logp[t] = a.s == 0.0f ? -INFINITY : (float)logp_of(chosen[t], a);
}

// ------------------------------------------------------------------------------------------
// policy loss
// ------------------------------------------------------------------------------------------
struct Policy { const int64_t* targets; const float *advantages, *weights, *old_logp, *ref_logp; float low, high, kl, grad_scale; };
struct __align__(16) TokenPart { float policy, kl; u32 counted, clipped; };          // a token's part of the five sums, weighted

// exp(x) as 2^n times the series of what is left, below 0.35: the first term left out is 2^-37 of it.
__device__ __forceinline__ double exp_wide(double x) {
    x = x < -800.0 ? -800.0 : x > 800.0 ? 800.0 : x;       // past both ends of fp64; NaN stays
    const double n = rint(x * 1.4426950408889634);
    x = fma(n, -0.6931471805599453, x);
    double t = 1.0 / 362880;
    t = fma(t, x, 1.0 / 40320); t = fma(t, x, 1.0 / 5040); t = fma(t, x, 1.0 / 720); t = fma(t, x, 1.0 / 120); t = fma(t, x, 1.0 / 24);
    t = fma(t, x, 1.0 / 6); t = fma(t, x, 0.5); t = fma(t, x, 1.0); t = fma(t, x, 1.0);
    return ldexp(t, (int)n);
}
// e = exp(d) - 1 and k = e - d, by k's series where the differences would cancel (next term 2^-36 of the sum).  e is not k + d: of a reference far below the
// policy (d = -1e9, -inf) nothing would be left of it, and the gradient is made of it.
struct Past { double e, k; };
__device__ __forceinline__ Past past_of(double d) {
    if (fabs(d) < 0.25) {
        double t = 1.0 / 362880;
        t = fma(t, d, 1.0 / 40320); t = fma(t, d, 1.0 / 5040); t = fma(t, d, 1.0 / 720); t = fma(t, d, 1.0 / 120); t = fma(t, d, 1.0 / 24);
        t = fma(t, d, 1.0 / 6); t = fma(t, d, 0.5);
        const double k = d * d * t;
        return {d + k, k};
    }
    const double e = exp_wide(d) - 1.0;
    return {e, e - d};
}
// Of a counted token with log probability lp: what it adds to the sums, and d loss / d lp.  In fp64, by one thread a row (a block's other waves and the CU's other row
// hide it): a ratio may be past fp32 where its product with a small weight is not, and each part is rounded once.
__device__ __forceinline__ TokenPart token_part(const Policy& p, u32 t, double lp, double* slope) {
    const double w = p.weights[t], a = p.advantages[t];
    double r = p.old_logp ? exp_wide(lp - (double)p.old_logp[t]) : 1.0;
    if (r > DBL_MAX) r = DBL_MAX;                          // a ratio past fp64 times an advantage of zero is zero
    const double lo = 1.0 - (double)p.low, hi = 1.0 + (double)p.high;
    const double free_term = r * a, held = (r < lo ? lo : r > hi ? hi : r) * a;
    const bool clipped = held < free_term;
    double g = clipped ? 0.0 : -free_term, kl = 0.0;
    if (p.ref_logp) {
        const Past past = past_of((double)p.ref_logp[t] - lp);
        kl = past.k;
        if (p.kl != 0.0f) g -= (double)p.kl * past.e;      // (watched only: an infinite term is not multiplied by zero)
    }
    *slope = w * g;
    return {(float)(w * -(clipped ? held : free_term)), (float)(w * kl), 1u, clipped ? 1u : 0u};
}

__device__ __forceinline__ void put_stats(float* stats, const double (&s)[4], float kl_coef) {
    stats[0] = (float)(kl_coef != 0.0f ? s[0] + (double)kl_coef * s[1] : s[0]);
    stats[1] = (float)s[0]; stats[2] = (float)s[1]; stats[3] = (float)s[2]; stats[4] = (float)s[3];
}

// What one thread finds out about a row: its token's part of the sums, and the slope for the row's gradient.  `stats`: of a batch of one token.
__device__ __forceinline__ float close_row(const Policy& p, u32 t, float x, Soft a, float* logp, TokenPart* parts, float* stats) {
    const double lp = logp_of(x, a);
    double slope;
    const TokenPart part = token_part(p, t, lp, &slope);
    parts[t] = part;
    if (logp) logp[t] = (float)lp;
    if (stats) { const double s[4] = {part.policy, part.kl, (double)part.clipped, (double)part.counted}; put_stats(stats, s, p.kl); }
    return (float)(slope * (double)p.grad_scale);
}
// A row that is not counted: `empty`, all its logits are -inf.
template <class T, int NT>
__device__ __forceinline__ void skip_row(typename T::elem* drow, u32 vocab, u32 t, bool empty, float* logp, TokenPart* parts, float* stats) {
    constexpr int W = Wide<T>::W;
    if (threadIdx.x == 0) {
        parts[t] = {0.0f, 0.0f, 0u, 0u};
        if (logp) logp[t] = empty ? -INFINITY : 0.0f;
        if (stats) for (int i = 0; i < 5; ++i) stats[i] = 0.0f;
    }
    if (!drow) return;
    // whole lines: from the first place that is a multiple of 16 bytes
    const u32 ahead = (u32)(-(uintptr_t)drow & 15) / sizeof(typename T::elem), head = ahead < vocab ? ahead : vocab, vecs = (vocab - head) / W, singles = vocab - vecs * W;
    for (u32 i = threadIdx.x; i < vecs; i += NT) *(u4v*)(drow + head + (u64)i * W) = u4v{0, 0, 0, 0};
    if (threadIdx.x < singles) drow[threadIdx.x < head ? threadIdx.x : threadIdx.x + vecs * W] = (typename T::elem)0.0f;
}

// Registers for two rows of 512 threads a CU, or one of 1024: two are faster wherever 512 threads hold the row (3051 rows of 65536 16-bit values 155 us, 196 by 1024).  22 vectors a thread fit without spilling (152 k and 178 k 16-bit values at 92 % of a large copy's rate, which two
// passes reach 68 % of).  Three rows a CU, with a few registers spilled, are slower: 8192 rows of 50257 16-bit values 292 us, 277 with two.
#define HELD_WAVES __attribute__((amdgpu_waves_per_eu(4)))
// A block takes a row and holds it: NV vectors a thread, all on their way at once.  A wave's vectors follow each other.  Where the gradient's row begins at another
// multiple of two than the logits', a vector is stored one place on, with the first value of the next one (of the next lane, or of the wave's next vector's first lane); the
// first value of a wave and the last vector of a wave or of the row are stored value by value.
template <class T, int NT, int NV, bool FAR>
__global__ __launch_bounds__(NT) HELD_WAVES void policy_held(Policy p, const typename T::elem* logits, u64 stride, u32 vocab, typename T::elem* dlogits, u64 dstride,
                                                  float* __restrict__ logp, TokenPart* __restrict__ parts, float* stats) {
    constexpr int W = Wide<T>::W, STEP = NV % 4 == 0 ? 4 : 2;
    typedef Vec<T, W> V;
    typedef typename T::elem E;
    __shared__ Soft part[NT / WAVE];
    __shared__ float slope_sh;
    const u32 t = blockIdx.x, tid = threadIdx.x;
    const u64 at = (u64)p.targets[t];
    const E* row = logits + (u64)t * stride;
    E* drow = dlogits + (u64)t * dstride;
    if (at >= vocab || p.weights[t] == 0.0f) { skip_row<T, NT>(drow, vocab, t, false, logp, parts, stats); return; }
    const Cut cut = cut_row<T>(row, vocab);
    const u32 first = (tid >> 6) * (NV * WAVE), lane = tid & 63;            // of the wave's vectors
    const E* body = row + cut.head + (u64)first * W;
    typename V::raw v[NV / STEP][STEP];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        v[j / STEP][j % STEP] = no_logits<V, W>();
        if (first + j * WAVE + lane < cut.vecs) v[j / STEP][j % STEP] = FAR ? V::load_far(body + (j * WAVE + lane) * W) : V::load(body + (j * WAVE + lane) * W);
    }
    const float single = tid < cut.singles ? (float)row[place_of_single<W>(cut, tid)] : -INFINITY, x = (float)row[at];
    Soft a = {-INFINITY, 0.0f};
#pragma unroll
    for (int j = 0; j < NV / STEP; ++j) {
        soft_add<V, W, STEP>(a, v[j]);
        __builtin_amdgcn_sched_barrier(0);                 // a step's converted values are not kept beside the next one's
    }
    soft_add_one(a, single);
    a = soft_block<NT>(a, part);
    if (a.s == 0.0f) { skip_row<T, NT>(drow, vocab, t, true, logp, parts, stats); return; }
    if (tid == 0) slope_sh = close_row(p, t, x, a, logp, parts, stats);
    __syncthreads();
    const float g = slope_sh, k = -g / a.s;
#pragma unroll
    for (int j = 0; j < NV; ++j) asm("" : "+v"(v[j / STEP][j % STEP]));     // the row as it lies in memory, not its values converted before the sum
    const auto gradient = [&](int j) {
        float y[W];
        V::open(v[j / STEP][j % STEP], y);
#pragma unroll
        for (int i = 0; i < W; ++i) y[i] = k * exp_of(y[i], a.m);
        return V::pack(y);
    };
    E* dbody = drow + cut.head + (u64)first * W;
    bool shifted = false;
    if constexpr (W == 8) shifted = (((uintptr_t)row ^ (uintptr_t)drow) & 2) != 0;
    if (!shifted) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            __builtin_amdgcn_sched_barrier(0);
            if (first + j * WAVE + lane >= cut.vecs) continue;
            const typename V::raw y = gradient(j);
            if (FAR) V::store_far(dbody + (j * WAVE + lane) * W, y);
            else V::store(dbody + (j * WAVE + lane) * W, y);
        }
    }
    if constexpr (W == 8) {
        if (shifted) {
            typename V::raw now = gradient(0), next = now;
            if (lane == 0 && first < cut.vecs) *(u16*)dbody = (u16)now.x;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                __builtin_amdgcn_sched_barrier(0);
                if (j + 1 < NV) next = gradient(j + 1);
                const u32 follow = (u32)__shfl_down((int)now.x, 1), wrap = (u32)__builtin_amdgcn_readfirstlane((int)next.x);
                const u32 i = first + j * WAVE + lane, behind = lane == 63 ? wrap : follow;
                E* to = dbody + (j * WAVE + lane) * W + 1;
                if (i + 1 < cut.vecs && !(j + 1 == NV && lane == 63)) {
                    V::store(to, (typename V::raw){now.x >> 16 | now.y << 16, now.y >> 16 | now.z << 16, now.z >> 16 | now.w << 16, now.w >> 16 | behind << 16});
                } else if (i < cut.vecs) {
                    u16* one = (u16*)to;
                    one[0] = (u16)(now.x >> 16);
                    one[1] = (u16)now.y; one[2] = (u16)(now.y >> 16);
                    one[3] = (u16)now.z; one[4] = (u16)(now.z >> 16);
                    one[5] = (u16)now.w; one[6] = (u16)(now.w >> 16);
                }
                now = next;
            }
        }
    }
    if (tid < cut.singles) drow[place_of_single<W>(cut, tid)] = (E)(k * exp_of(single, a.m));
    // the target's once more, when its first value is written: whichever thread that was, the barrier is behind it
    __syncthreads();
    if (tid == 0) drow[at] = (E)(g + k * exp_of(x, a.m));
}

// Rows that registers do not hold, and calls without a gradient: one pass for the sum, a second one for the gradient, which finds most of the row in the caches.
template <class T, int NT>
__global__ __launch_bounds__(NT) void policy_twice(Policy p, const typename T::elem* logits, u64 stride, u32 vocab, typename T::elem* dlogits, u64 dstride,
                                                   float* __restrict__ logp, TokenPart* __restrict__ parts, float* stats) {
    constexpr int W = Wide<T>::W;
    typedef Vec<T, W> V;
    __shared__ Soft part[NT / WAVE];
    __shared__ float slope_sh;
    const u32 t = blockIdx.x, tid = threadIdx.x;
    const u64 at = (u64)p.targets[t];
    const typename T::elem* row = logits + (u64)t * stride;
    typename T::elem* drow = dlogits ? dlogits + (u64)t * dstride : nullptr;
    if (at >= vocab || p.weights[t] == 0.0f) { skip_row<T, NT>(drow, vocab, t, false, logp, parts, stats); return; }
    const float x = tid == 0 ? (float)row[at] : 0.0f;
    const Soft a = soft_block<NT>(soft_row<T, NT, false>(row, vocab), part);
    if (a.s == 0.0f) { skip_row<T, NT>(drow, vocab, t, true, logp, parts, stats); return; }
    if (tid == 0) slope_sh = close_row(p, t, x, a, logp, parts, stats);
    __syncthreads();
    if (!drow) return;
    const float g = slope_sh, k = -g / a.s;
    const Cut cut = cut_row<T>(row, vocab);
    for (u32 i = tid; i < cut.vecs; i += NT) {
        const u64 c = cut.head + (u64)i * W;
        float y[W];
        V::open(V::load(row + c), y);
#pragma unroll
        for (int e = 0; e < W; ++e) y[e] = k * exp_of(y[e], a.m) + (c + e == at ? g : 0.0f);
        V::store(drow + c, V::pack(y));
    }
    if (tid < cut.singles) {
        const u32 c = place_of_single<W>(cut, tid);
        drow[c] = (typename T::elem)(k * exp_of((float)row[c], a.m) + (c == at ? g : 0.0f));
    }
}

// The sums over all tokens in fp64 and a fixed order: each block those of its share, one block the blocks'.  (8 us for 8192 tokens, a launch and the latency of one block's reads: of the
// 276 us of a large batch little, of the 20 to 30 of a few hundred long rows much.)
#define SUM_SHARE 16384
template <int NT>
__device__ __forceinline__ bool sum_block(double (&s)[4], double (&sh)[4][NT / WAVE]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        for (int d = 1; d < WAVE; d <<= 1) s[i] += __shfl_xor(s[i], d);
        if ((threadIdx.x & 63) == 0) sh[i][threadIdx.x >> 6] = s[i];
    }
    __syncthreads();
    if (threadIdx.x) return false;
#pragma unroll
    for (int i = 0; i < 4; ++i) { s[i] = 0; for (int w = 0; w < NT / WAVE; ++w) s[i] += sh[i][w]; }
    return true;
}
// Few long rows, the second launch: every block of a row joins its shares and finds the slope for itself; one block more does so for all tokens (at most SHARE_NT) and adds
// them up, from the same bits: a token is counted as clipped when its gradient is zero.
template <class T>
__global__ __launch_bounds__(SHARE_NT) void policy_shares(Shares q, Policy p, const typename T::elem* logits, u64 stride, u32 vocab, typename T::elem* dlogits, u64 dstride, u32 n,
                                                          const Soft* __restrict__ softs, const float* __restrict__ chosen, float* __restrict__ logp, float* __restrict__ stats) {
    constexpr int W = Wide<T>::W;
    typedef Vec<T, W> V;
    typedef typename T::elem E;
    const u32 s = blockIdx.x, tid = threadIdx.x;
    if (s == q.n) {                                        // the sums
        __shared__ double sh[4][SHARE_NT / WAVE];
        if (blockIdx.y) return;
        double sum[4] = {0, 0, 0, 0};
        if (tid < n) {
            const u64 at = (u64)p.targets[tid];
            const bool read = at < vocab && p.weights[tid] != 0.0f;
            Soft a = {-INFINITY, 0.0f};
            if (read) a = soft_of_row_alone(softs, tid, q.n);
            double lp = read ? -INFINITY : 0.0;
            if (a.s != 0.0f) {
                double slope;
                lp = logp_of(chosen[tid], a);
                const TokenPart part = token_part(p, tid, lp, &slope);
                sum[0] = part.policy; sum[1] = part.kl; sum[2] = part.clipped; sum[3] = part.counted;
            }
            if (logp) logp[tid] = (float)lp;
        }
        if (sum_block<SHARE_NT>(sum, sh)) put_stats(stats, sum, p.kl);
        return;
    }
    const u32 t = blockIdx.y;
    const u64 at = (u64)p.targets[t];
    const E* row = logits + (u64)t * stride;
    E* drow = dlogits + (u64)t * dstride;
    const Cut c = cut_row<T>(row, vocab);
    u32 lo, hi;
    share_of<T>(c, q, s, &lo, &hi);
    Soft a = {-INFINITY, 0.0f};
    if (at < vocab && p.weights[t] != 0.0f) a = soft_of_row(softs, t, q.n);
    const bool counted = a.s != 0.0f;
    double slope = 0.0;
    if (counted) token_part(p, t, logp_of(chosen[t], a), &slope);
    const float g = (float)(slope * (double)p.grad_scale);
    const float k = counted ? -g / a.s : 0.0f;
    const u32 single = s == 0 && tid < c.singles ? place_of_single<W>(c, tid) : 0;
    for (u32 i = lo + tid; i < hi; i += SHARE_NT * STREAM) {
        typename V::raw r[STREAM] = {};
        if (counted) {
#pragma unroll
            for (int j = 0; j < STREAM; ++j) if (i + j * SHARE_NT < hi) r[j] = V::load(row + c.head + (u64)(i + j * SHARE_NT) * W);
        }
#pragma unroll
        for (int j = 0; j < STREAM; ++j) {
            if (i + j * SHARE_NT >= hi) continue;
            const u64 to = c.head + (u64)(i + j * SHARE_NT) * W;
            float y[W];
            V::open(r[j], y);
#pragma unroll
            for (int e = 0; e < W; ++e) y[e] = counted ? k * exp_of(y[e], a.m) + (to + e == at ? g : 0.0f) : 0.0f;
            V::store(drow + to, V::pack(y));
        }
    }
    if (s == 0 && tid < c.singles) drow[single] = (E)(counted ? k * exp_of((float)row[single], a.m) + (single == at ? g : 0.0f) : 0.0f);
}

__global__ __launch_bounds__(1024) void policy_sums(const TokenPart* __restrict__ parts, u32 n, float kl_coef, double* __restrict__ shares, float* __restrict__ stats) {
    __shared__ double sh[4][16];
    double s[4] = {0, 0, 0, 0};
    const u32 lo = blockIdx.x * SUM_SHARE, hi = n - lo < SUM_SHARE ? n : lo + SUM_SHARE;
#pragma unroll 8
    for (u32 t = lo + threadIdx.x; t < hi; t += 1024) {
        const TokenPart p = parts[t];
        s[0] += (double)p.policy; s[1] += (double)p.kl; s[2] += (double)p.clipped; s[3] += (double)p.counted;
    }
    if (!sum_block<1024>(s, sh)) return;
    if (gridDim.x == 1) put_stats(stats, s, kl_coef);
    else for (int i = 0; i < 4; ++i) shares[4 * blockIdx.x + i] = s[i];
}
__global__ __launch_bounds__(256) void policy_join(const double* __restrict__ shares, u32 n, float kl_coef, float* __restrict__ stats) {
    __shared__ double sh[4][4];
    double s[4] = {0, 0, 0, 0};
    for (u32 b = threadIdx.x; b < n; b += 256)
        for (int i = 0; i < 4; ++i) s[i] += shares[4 * (u64)b + i];
    if (sum_block<256>(s, sh)) put_stats(stats, s, kl_coef);
}

// ------------------------------------------------------------------------------------------
// C-ABI
// ------------------------------------------------------------------------------------------
#define FAR_BYTES (256ull << 20)                 // logits that the memory-side cache does not hold are read and written past it

// Where the workspace holds the shares of sums and of rows; the tokens' parts come first.  (A larger batch's is large enough for a smaller one.)
struct LogitsPlan { u64 sums, softs, chosen, bytes; };
// Fewer rows than FEW_ROWS leave half of the CUs without one: blocks share a row of at least MANY_VECS vectors.  Policy loss, with the sums, of rows of 50257 floats: 64 rows
// 17 us by a block each, 14.5 shared; 100 18, 16; 140 19, 20; 190 21, 25; two rows of 150000 25, 10.
#define FEW_ROWS 128
#define MANY_VECS 2048
static LogitsPlan logits_plan(u64 n) {
    const u64 sums = round_up(n * sizeof(TokenPart), 256), softs = sums + round_up((n + SUM_SHARE - 1) / SUM_SHARE * 32, 256);
    const u64 few = n < FEW_ROWS ? n : FEW_ROWS - 1, chosen = softs + round_up(few * SHARES_MOST * sizeof(Soft), 256);
    return {sums, softs, chosen, chosen + round_up(few * 4, 256) + 256};
}
// About three blocks a CU, of at least two vectors a thread.
static Shares shares_of(u64 n, u32 vecs) {
    u32 k = (u32)(768 / n);
    if (k > vecs / (2 * SHARE_NT)) k = vecs / (2 * SHARE_NT);
    if (k > SHARES_MOST) k = SHARES_MOST;
    return {k, (vecs + k - 1) / k};
}

// Calls f(first row, rows) for launches of a block of NT threads a row: a grid has fewer than 2^32 threads.
template <int NT, class F>
static void each_rows(u64 rows, F f) {
    constexpr u64 most = COUNT_LIMIT / NT;
    for (u64 row0 = 0; row0 < rows; row0 += most) f(row0, (u32)(rows - row0 < most ? rows - row0 : most));
}
static Policy rows_from(Policy p, u64 row0) {
    p.targets += row0; p.advantages += row0; p.weights += row0;
    if (p.old_logp) p.old_logp += row0;
    if (p.ref_logp) p.ref_logp += row0;
    return p;
}

extern "C" uint64_t dblp_logits_workspace(uint64_t n_tokens, uint32_t vocab) {
    if (n_tokens >= COUNT_LIMIT || vocab == 0 || vocab >= COUNT_LIMIT) return 0;
    return logits_plan(n_tokens).bytes;
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
    Launches launch;
    const bool far = n_tokens * vocab * type_bytes(type) > FAR_BYTES;
    by_type(type, [&](auto tt) {
        typedef decltype(tt) T;
        const auto go = [&](auto nt) {
            constexpr int NT = decltype(nt)::value;
            each_rows<NT>(n_tokens, [&](u64 row0, u32 rows) {
                launch(far ? (logprob_rows<T, NT, true>) : (logprob_rows<T, NT, false>), dim3(rows), NT, (hipStream_t)stream, (const typename T::elem*)d_logits + row0 * logits_stride, (u64)logits_stride, vocab,
                                   d_targets + row0, d_logp + row0, d_lse ? d_lse + row0 : nullptr);
            });
        };
        const u32 vecs = vocab / Wide<T>::W;
        // rows that one CU reads for longer than a launch more takes, on the host too: one row of 200000 floats 12 us by a block, 5 shared; of 50257 16-bit values 6, 5
        if (n_tokens < FEW_ROWS / 2 && vecs >= 16 * MANY_VECS) {
            const Shares q = shares_of(n_tokens, vecs);
            Soft* const softs = (Soft*)((uint8_t*)d_workspace + logits_plan(n_tokens).softs);
            float* const chosen = (float*)((uint8_t*)d_workspace + logits_plan(n_tokens).chosen);
            launch(soft_shares<T>, dim3(q.n, (u32)n_tokens), SHARE_NT, (hipStream_t)stream, q, (const typename T::elem*)d_logits, (u64)logits_stride, vocab, d_targets, (const float*)nullptr, softs, chosen);
            launch(logprob_join, dim3((u32)n_tokens), 64, (hipStream_t)stream, q, vocab, d_targets, (const Soft*)softs, (const float*)chosen, d_logp, d_lse);
            return;
        }
        // Threads that end with their row: each has at most six vectors of it, in two steps.  A batch of 160 MB of 2500 16-bit values takes 32 us by 64 threads a row, 38 by 128,
        // 124 by 512; of 7539 33, 31 and 50 (29 by 256); of 12000 32, 32, 33 (30 by 256); of 16000 35, 34, 28 (33 by 256).  Between one and three rows a CU, long rows
        // are read by 256 threads too: 400 of 50257 10 us, 11 by 512; 520 of them 13, 15; 520 of 128256 28, 32; but 130 of 128256 15, 10.
        if (vecs <= 64 * 6) go(Int<64>());
        else if (vecs <= 128 * 6) go(Int<128>());
        else if (vecs <= 256 * 6 || (n_tokens >= 256 && n_tokens < 768)) go(Int<256>());
        else go(Int<512>());
    });
    return launched(call, launch);
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
    Launches launch;
    const Policy p = {d_targets, d_advantages, d_weights, d_old_logp, d_ref_logp, clip_low, clip_high, kl_coef, grad_scale};
    TokenPart* const parts = (TokenPart*)d_workspace;
    double* const shares = (double*)((uint8_t*)d_workspace + logits_plan(n_tokens).sums);
    Soft* const softs = (Soft*)((uint8_t*)d_workspace + logits_plan(n_tokens).softs);
    float* const chosen = (float*)((uint8_t*)d_workspace + logits_plan(n_tokens).chosen);
    bool summed = false;
    const hipStream_t st = (hipStream_t)stream;
    const u32 n = (u32)n_tokens;
    float* const own_stats = n == 1 ? d_stats : nullptr;         // one token's sums are its own
    // (past the cache only where every row begins at a multiple of 16 bytes: other stores with the hint cost parts of lines)
    const bool far = n_tokens * vocab * type_bytes(type) > FAR_BYTES / 2 && !off(d_logits, 16) && !off(d_dlogits, 16) && logits_stride * type_bytes(type) % 16 == 0 && dlogits_stride * type_bytes(type) % 16 == 0;
    if (n)
        by_type(type, [&](auto tt) {
            typedef decltype(tt) T;
            typedef typename T::elem E;
            constexpr u32 W = Wide<T>::W;
            const auto twice = [&](auto nt) {
                constexpr int NT = decltype(nt)::value;
                each_rows<NT>(n, [&](u64 row0, u32 rows) {
                    launch((policy_twice<T, NT>), dim3(rows), NT, st, rows_from(p, row0), (const E*)d_logits + row0 * logits_stride, (u64)logits_stride, vocab,
                                       d_dlogits ? (E*)d_dlogits + row0 * dlogits_stride : nullptr, (u64)dlogits_stride, d_logp ? d_logp + row0 : nullptr, parts + row0, own_stats);
                });
            };
            const auto held = [&](auto nt, auto nv) {
                constexpr int NT = decltype(nt)::value, NV = decltype(nv)::value;
                each_rows<NT>(n, [&](u64 row0, u32 rows) {
                    launch(far ? (policy_held<T, NT, NV, true>) : (policy_held<T, NT, NV, false>), dim3(rows), NT, st, rows_from(p, row0), (const E*)d_logits + row0 * logits_stride, (u64)logits_stride, vocab,
                                       (E*)d_dlogits + row0 * dlogits_stride, (u64)dlogits_stride, d_logp ? d_logp + row0 : nullptr, parts + row0, own_stats);
                });
            };
            const u32 vecs = vocab / W;
            // (one token's row, if registers hold it, needs one launch where sharing needs two)
            if (d_dlogits && n < FEW_ROWS && vecs >= MANY_VECS && !(n == 1 && vocab <= 1024 * 18 * W)) {
                const Shares q = shares_of(n, vecs);
                launch(soft_shares<T>, dim3(q.n, n), SHARE_NT, st, q, (const E*)d_logits, (u64)logits_stride, vocab, d_targets, d_weights, softs, chosen);
                launch(policy_shares<T>, dim3(q.n + 1, n), SHARE_NT, st, q, p, (const E*)d_logits, (u64)logits_stride, vocab, (E*)d_dlogits, (u64)dlogits_stride, n, (const Soft*)softs, (const float*)chosen, d_logp, d_stats);
                summed = true;
            }
            else if (!d_dlogits) vocab <= 64 * W * STREAM ? twice(Int<64>()) : twice(Int<512>());
            else if (vocab <= 64 * 2 * W) held(Int<64>(), Int<2>());
            else if (vocab <= 64 * 8 * W) held(Int<64>(), Int<8>());
            else if (vocab <= 256 * 4 * W) held(Int<256>(), Int<4>());
            else if (vocab <= 256 * 8 * W) held(Int<256>(), Int<8>());
            else if (vocab <= 512 * 8 * W) held(Int<512>(), Int<8>());
            else if (vocab <= 512 * 14 * W) held(Int<512>(), Int<14>());
            else if (vocab <= 512 * 18 * W) held(Int<512>(), Int<18>());
            else if (vocab <= 512 * 22 * W) held(Int<512>(), Int<22>());
            else if (vocab <= 1024 * 14 * W) held(Int<1024>(), Int<14>());
            else if (vocab <= 1024 * 18 * W) held(Int<1024>(), Int<18>());
            else if (vocab <= 1024 * 22 * W) held(Int<1024>(), Int<22>());
            else twice(Int<1024>());
        });
    if (n != 1 && !summed) {
        const u32 blocks = n ? (n + SUM_SHARE - 1) / SUM_SHARE : 1;
        launch(policy_sums, dim3(blocks), 1024, st, (const TokenPart*)parts, n, kl_coef, shares, d_stats);
        if (blocks > 1) launch(policy_join, dim3(1), 256, st, (const double*)shares, blocks, kl_coef, d_stats);
    }
    return launched(call, launch);
}
