// A worker's matrix products and their gradients (include/dblp_layers.h).
#include "layer_tiles.h"

// ------------------------------------------------------------------------------------------
// activations and their slopes
// ------------------------------------------------------------------------------------------
#define LOG2E 1.4426950408889634f
#define ROOT_TWO_OVER_PI 0.79788456080286536f
#define CUBE 0.044715f

__device__ __forceinline__ float one_over(float x) { return __builtin_amdgcn_rcpf(x); }
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// The normal distribution's density over its value at 0, exp(-z z / 2), and its integral from -|z|, Phi(-|z|) = exp(-z z / 2) t R(t), t = 1 / (1 + 0.35 |z|): R is a
// polynomial of degree 8, fitted to the least largest relative error over |z| <= 15, 3.2e-8 (2.9e-7 as it is computed, five roundings), where exp(-z z / 2) has long been zero.
struct Normal { float bell, tail; };
__device__ __forceinline__ Normal normal_of(float z) {
    const float t = one_over(1.0f + 0.35f * fabsf(z)), bell = exp2_of(-0.5f * LOG2E * z * z);
    float r = -0.02916385f;
    r = r * t + 0.14406044f;
    r = r * t - 0.25590114f;
    r = r * t + 0.15939213f;
    r = r * t - 0.02326333f;
    r = r * t + 0.10557461f;
    r = r * t + 0.11981554f;
    r = r * t + 0.13986433f;
    r = r * t + 0.13962126f;
    return {bell, bell * (t * r)};
}
// tanh's argument of GELU_TANH, twice, negated and for a power of two.
__device__ __forceinline__ float tanh_power(float z) { return z * (-2.0f * LOG2E * ROOT_TWO_OVER_PI - 2.0f * LOG2E * ROOT_TWO_OVER_PI * CUBE * z * z); }

// An exponential is a power of two, whose argument's rounding is worth w U of a result with exp(w) in it: as much as the fp32 argument itself.  The kind of activation is chosen
// once for several values, which the matrix instructions' units need not wait for each other's exponentials.
template <int N>
__device__ __forceinline__ void activate(int act, float (&v)[N]) {
    switch (act) {
        case DBLP_ACT_RELU:
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = v[i] <= 0.0f ? 0.0f : v[i];
            break;
        case DBLP_ACT_GELU:
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float tail = normal_of(v[i]).tail;
                v[i] *= v[i] < 0.0f ? tail : 1.0f - tail;
            }
            break;
        case DBLP_ACT_GELU_TANH:
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] *= one_over(1.0f + exp2_of(tanh_power(v[i])));
            break;
        case DBLP_ACT_SILU:
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] *= one_over(1.0f + exp2_of(-LOG2E * v[i]));
            break;
    }
}
// dy = dy act'(z).  A slope's 1 - p has lost U where p is near one; its factor there, z and its square, is below 40 until p is one and the product zero.
template <int N>
__device__ __forceinline__ void gate(int act, const float (&z)[N], float (&dy)[N]) {
    switch (act) {
        case DBLP_ACT_RELU:
#pragma unroll
            for (int i = 0; i < N; ++i) dy[i] = z[i] > 0.0f ? dy[i] : 0.0f;
            break;
        case DBLP_ACT_GELU:
#pragma unroll
            for (int i = 0; i < N; ++i) {
                // of -|z|, and of |z| one less that
                const Normal n = normal_of(z[i]);
                const float below = n.tail - fabsf(z[i]) * (n.bell * (0.5f * ROOT_TWO_OVER_PI));
                dy[i] *= z[i] < 0.0f ? below : 1.0f - below;
            }
            break;
        case DBLP_ACT_GELU_TANH:
#pragma unroll
            for (int i = 0; i < N; ++i) {
                // (past 30 the exponential has long been zero or infinity: a larger z' square would be infinite where zero times it is wanted)
                const float t = fminf(fmaxf(z[i], -30.0f), 30.0f), p = one_over(1.0f + exp2_of(tanh_power(t)));
                dy[i] *= p + z[i] * (p * (1.0f - p) * (2.0f * ROOT_TWO_OVER_PI + 6.0f * ROOT_TWO_OVER_PI * CUBE * t * t));
            }
            break;
        case DBLP_ACT_SILU:
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float p = one_over(1.0f + exp2_of(-LOG2E * z[i]));
                dy[i] *= p + z[i] * (p * (1.0f - p));
            }
            break;
    }
}

// ------------------------------------------------------------------------------------------
// what becomes of a product's sums
// ------------------------------------------------------------------------------------------
struct Matrix { void* p; u64 stride; };          // of a type that is known when the kernel runs

template <class T, int N>
__device__ __forceinline__ void store_rows_as(const Matrix& to, u32 m, u32 apart, u32 n, u32 cols, u32 on, const float (&v)[N]) {
#pragma unroll
    for (int e = 0; e < N / 4; ++e) {
        const float r[4] = {v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]};
        if (on >> e & 1) store_cols<Vec<T, 4>, 4>((typename T::elem*)to.p + (u64)(m + e * apart) * to.stride, n, cols, r);
    }
}
template <int N>
__device__ __forceinline__ void store_rows(int type, const Matrix& to, u32 m, u32 apart, u32 n, u32 cols, u32 on, const float (&v)[N]) {
    if (type == DBLP_F32) store_rows_as<F32>(to, m, apart, n, cols, on, v);
    else if (type == DBLP_BF16) store_rows_as<BF16>(to, m, apart, n, cols, on, v);
    else store_rows_as<F16>(to, m, apart, n, cols, on, v);
}

struct LayerOut {
    int type, act, bias_type;
    const void* bias;
    Matrix residual, y, z;
    struct Met { u4v bias, residual; };
    __device__ __forceinline__ Met get(u32, u32 m, u32 n, u32 cols) const {
        Met r = {};
        if (bias) r.bias = raw4(bias_type, bias, n, cols - n);
        if (residual.p) r.residual = raw4(type, residual.p, m * residual.stride + n, cols - n);
        return r;
    }
    // N rows, `apart` from each other, those that `on` names
    template <int N>
    __device__ __forceinline__ void put_rows(u32, u32, u32 m, u32 apart, u32 n, u32 cols, u32 on, const f4 (&acc)[N], const Met (&met)[N]) const {
        float v[4 * N];
        for (int i = 0; i < 4 * N; ++i) v[i] = acc[i / 4][i % 4];
        if (bias) {
            float b[4];
            open4(bias_type, met[0].bias, b);
            for (int i = 0; i < 4 * N; ++i) v[i] += b[i % 4];
        }
        if (z.p) store_rows(type, z, m, apart, n, cols, on, v);
        activate(act, v);
        if (residual.p)
            for (int e = 0; e < N; ++e) {
                float r[4];
                open4(type, met[e].residual, r);
                for (int i = 0; i < 4; ++i) v[4 * e + i] += r[i];
            }
        store_rows(type, y, m, apart, n, cols, on, v);
    }
    __device__ __forceinline__ void put(u32 matrix, u32 part, u32 m, u32 n, u32 cols, f4 acc, const Met& met) const {
        const f4 a[1] = {acc};
        const Met b[1] = {met};
        put_rows<1>(matrix, part, m, 0, n, cols, 1, a, b);
    }
    __device__ __forceinline__ void sums(u32, u32, u32, float) const {}
};

struct GateOut {
    int type, act;
    Matrix z, base, dx;
    struct Met { u4v z, base; };
    __device__ __forceinline__ Met get(u32, u32 m, u32 n, u32 cols) const {
        Met r = {};
        if (z.p) r.z = raw4(type, z.p, m * z.stride + n, cols - n);
        if (base.p) r.base = raw4(type, base.p, m * base.stride + n, cols - n);
        return r;
    }
    template <int N>
    __device__ __forceinline__ void put_rows(u32, u32, u32 m, u32 apart, u32 n, u32 cols, u32 on, const f4 (&acc)[N], const Met (&met)[N]) const {
        float v[4 * N], b[4 * N];
        for (int i = 0; i < 4 * N; ++i) v[i] = acc[i / 4][i % 4];
        const auto open = [&](auto which) {
            for (int e = 0; e < N; ++e) {
                float r[4];
                open4(type, which(met[e]), r);
                for (int i = 0; i < 4; ++i) b[4 * e + i] = r[i];
            }
        };
        if (z.p) {
            open([](const Met& t) { return t.z; });
            gate(act, b, v);
        }
        if (base.p) {
            open([](const Met& t) { return t.base; });
            for (int i = 0; i < 4 * N; ++i) v[i] += b[i];
        }
        store_rows(type, dx, m, apart, n, cols, on, v);
    }
    __device__ __forceinline__ void put(u32 matrix, u32 part, u32 m, u32 n, u32 cols, f4 acc, const Met& met) const {
        const f4 a[1] = {acc};
        const Met b[1] = {met};
        put_rows<1>(matrix, part, m, 0, n, cols, 1, a, b);
    }
    __device__ __forceinline__ void sums(u32, u32, u32, float) const {}
};

struct WeightOut {
    const float* base;
    u64 base_stride;
    float* dw;
    u64 dw_stride;
    const float* bias_base;
    float* dbias;
    __device__ __forceinline__ u4v get(u32, u32 m, u32 n, u32 cols) const { return base ? raw4(DBLP_F32, base, m * base_stride + n, cols - n) : (u4v)(0u); }
    __device__ __forceinline__ void put(u32, u32, u32 m, u32 n, u32 cols, f4 acc, u4v met) const {
        const f4 b = __builtin_bit_cast(f4, met);
        const float v[4] = {acc[0] + b[0], acc[1] + b[1], acc[2] + b[2], acc[3] + b[3]};
        store4(DBLP_F32, dw, m * dw_stride + n, cols - n, v);
    }
    __device__ __forceinline__ void sums(u32, u32, u32 m, float s) const { if (dbias) dbias[m] = bias_base ? bias_base[m] + s : s; }
};

// ------------------------------------------------------------------------------------------
// the bias' gradient where large tiles make the weight's: sums of columns, eight rows of threads a block, blockIdx.y one of gridDim.y slices of the rows.  Bound by memory: 268 MB in
// 59 us (4.5 TB/s); in the large tiles' own loop the sums' registers spill.
// ------------------------------------------------------------------------------------------
template <class T>
__global__ __launch_bounds__(256) void column_sums(const typename T::elem* p, u64 stride, u32 rows, u32 cols, u32 slice, PartOut out, WeightOut last) {
    constexpr int E = 16 / sizeof(typename T::elem);
    typedef Vec<T, E> V;
    __shared__ float sh[8][32 * E + 4];
    const u32 x = threadIdx.x & 31, y = threadIdx.x >> 5, c = (blockIdx.x * 32 + x) * E;
    const u32 first = blockIdx.y * slice, end = rows - first < slice ? rows : first + slice;
    float sum[E] = {};
    if (c < cols)
        for (u32 r = first + y; r < end; r += 32) {
            typename V::raw v[4];
#pragma unroll
            for (u32 i = 0; i < 4; ++i) if (r + 8 * i < end) v[i] = c + E <= cols ? V::load(p + (r + 8 * i) * stride + c) : V::some(p + (r + 8 * i) * stride + c, cols - c);
#pragma unroll
            for (u32 i = 0; i < 4; ++i)
                if (r + 8 * i < end) {
                    float f[E];
                    V::open(v[i], f);
                    for (int e = 0; e < E; ++e) sum[e] += f[e];
                }
        }
    for (int e = 0; e < E; ++e) sh[y][x * E + e] = sum[e];
    __syncthreads();
    for (u32 i = threadIdx.x; i < 32 * E; i += 256) {
        float all = 0.0f;
        for (u32 j = 0; j < 8; ++j) all += sh[j][i];
        const u32 m = blockIdx.x * 32 * E + i;
        if (m >= cols) continue;
        if (gridDim.y == 1) last.sums(0, 0, m, all);
        else out.sums(0, blockIdx.y, m, all);
    }
}
__global__ __launch_bounds__(64) void join_sums(PartOut in, u32 cols, u32 parts, WeightOut last) {
    const u32 m = blockIdx.x * 64 + threadIdx.x;
    if (m >= cols) return;
    float sum = 0.0f;
    for (u32 i = 0; i < parts; i += 16) {
        float v[16];
#pragma unroll
        for (u32 j = 0; j < 16; ++j) v[j] = i + j < parts ? in.row_sums[(u64)(i + j) * in.rows + m] : 0.0f;
#pragma unroll
        for (u32 j = 0; j < 16; ++j) sum += v[j];
    }
    last.sums(0, 0, m, sum);
}

// ------------------------------------------------------------------------------------------
// activation_grad: a thread takes 16 bytes.  Bound by memory: 805 MB in 135 us (6.0 TB/s) whatever the activation; 180 to 200 where each value chose its activation by itself.
// ------------------------------------------------------------------------------------------
template <class T, int W, bool WHOLE>
__global__ __launch_bounds__(256) void activation_units(Units s, int act, const typename T::elem* dy, u64 dy_stride, const typename T::elem* z, u64 z_stride, typename T::elem* dz, u64 dz_stride) {
    typedef Vec<T, W> V;
    const u32 u = blockIdx.x * 256 + threadIdx.x;
    if (u >= s.n) return;
    const u32 row = s.per_row.of(u), c = (u - row * s.per_row.d) * W;
    if (c >= s.cols) return;
    const u64 r = s.row0 + row;
    const typename V::raw a = load_cols<V, W, WHOLE>(dy + r * dy_stride, c, s.cols), b = load_cols<V, W, WHOLE>(z + r * z_stride, c, s.cols);
    float x[W], y[W];
    V::open(settle_cols<V, W, WHOLE>(a, c, s.cols), x);
    V::open(settle_cols<V, W, WHOLE>(b, c, s.cols), y);
    gate<W>(act, y, x);
    store_cols<V, W>(dz + r * dz_stride, c, s.cols, x);
}

// ------------------------------------------------------------------------------------------
// C-ABI
// ------------------------------------------------------------------------------------------
static bool bad_act(int act) { return act < DBLP_ACT_NONE || act > DBLP_ACT_SILU; }
static bool bad_sizes(u64 tokens, u64 in, u64 out) { return tokens >= COUNT_LIMIT || in >= COUNT_LIMIT || out >= COUNT_LIMIT; }

// A workspace: parts of a product and of a bias' gradient, then room for two operands with rows at multiples of 16 bytes, up to so many bytes.
#define ALIGNED_BYTES (1ull << 30)
static u64 aligned_stride(u64 cols) { return round_up(cols, 8); }
static u64 aligned_bytes(u64 lines, u64 cols) {
    const u64 stride = aligned_stride(cols);                                         // (lines stride 2 <= 2^63)
    return lines * stride * 2 < ALIGNED_BYTES ? round_up(lines * stride * 2, 256) : ALIGNED_BYTES;
}
static u64 aligned_at(u64 n_tokens, u64 in, u64 out) {
    u64 most = parts_bytes(n_tokens, out);
    for (const u64 other : {parts_bytes(n_tokens, in), parts_bytes(out, in)}) if (other > most) most = other;
    return 256 + round_up(most, 256) + round_up((u64)PARTS_MOST * out * 4, 256);
}
extern "C" uint64_t dblp_linear_workspace(uint64_t n_tokens, uint32_t in, uint32_t out) {
    if (bad_sizes(n_tokens, in, out)) return 0;
    const u64 w = aligned_bytes(out, in), dy = aligned_bytes(n_tokens, out), two = aligned_bytes(n_tokens, in) + (w > dy ? w : dy);
    return aligned_at(n_tokens, in, out) + (two < ALIGNED_BYTES ? two : ALIGNED_BYTES);
}

// A way to make a product: tiles of one kind, the sum over k in `parts` parts.
enum Kind { TILES_64, TILES_128, TILES_256, KINDS };
struct Way { Kind kind; u32 parts, part; double us, stages_us; };     // (stages_us: of it, without what each round and the parts' sum take)

// Chosen by an estimate of the time, in microseconds: rounds of tiles over the 256 CUs, each a fixed time and one for each stage of 128 bytes of k, which is longer with more blocks on a CU
// (of the largest tiles, with more CUs at work); parts are written, read and added up at 5 TB/s.  As measured with each kind alone over 27 sizes; the choice is within 15 % of the best
// kind and number of parts on them (8192 x 1024 x 4096 in tiles of 64, 128, 256: 118, 79, 68 us; 2048 x 768 x 2304: 18, 18, 26; the weight's gradient of 8192 x 768 x 2304 in 1 and 4 parts of tiles of 128 85 and 44, in 8 of 256 46).
static Way way_of(u64 rows, u64 cols, u64 depth, u32 elem) {
    static const struct { u32 tile, blocks; double fixed, stage[2][3]; } K[KINDS] = {
        {64, 3, 3.5, {{0.28, 0.40, 0.50}, {0.65, 0.90, 1.10}}}, {128, 2, 5.0, {{0.64, 0.98, 0}, {1.85, 2.65, 0}}}, {256, 1, 10.0, {{1.15, 0, 0}, {0, 0, 0}}}};
    Way best = {TILES_64, 1, 0, 0, 0};
    double& least = best.us = 1e30;
    const u64 ks = 128 / elem, stages = (depth + ks - 1) / ks, bytes = rows * round_up(cols, 4) * 4;
    for (int i = 0; i < KINDS; ++i) {
        if (i == TILES_256 && elem == 4) continue;
        const u64 tiles = ((rows + K[i].tile - 1) / K[i].tile) * ((cols + K[i].tile - 1) / K[i].tile);
        for (u64 p = 1; p <= PARTS_MOST && (p == 1 || (p * bytes <= PARTS_BYTES && stages / p >= 2)); ++p) {
            const u64 each = (stages + p - 1) / p;
            if (p > 1 && (stages + each - 1) / each != p) continue;
            const double blocks = (double)tiles * p, rounds = ceil(blocks / (256.0 * K[i].blocks));
            const int held = blocks > 256.0 * K[i].blocks ? (int)K[i].blocks : blocks > 256.0 ? (int)ceil(blocks / 256.0) : 1;
            const double stage = K[i].stage[elem == 4][held - 1] + (i == TILES_256 ? 0.4 * fmin(1.0, blocks / 256.0) : 0.0);
            const double t = rounds * (K[i].fixed + each * stage) + (p > 1 ? 3.0 + p * bytes * 2 / 5e6 : 0.0);
            if (t < least) {
                best = {(Kind)i, (u32)p, (u32)(each * ks), t, rounds * each * stage};
            }
        }
    }
    if (best.parts == 1) best.part = 0;
    return best;
}

// Whether the rows of P are taken as even and odd ones (the sum of half of them then has one k more).
template <class T, bool P_BY_K, bool Q_BY_K>
static bool in_pairs(const Product& a) { return sizeof(typename T::elem) == 2 && !P_BY_K && Q_BY_K && !copied<T>(a.P) && copied<T>(a.Q); }

template <class T, bool P_BY_K, bool Q_BY_K, bool SUMS, class Out>
static void tiles(Launches& launch, hipStream_t stream, Product a, Kind kind, Out out) {
    const auto go = [&](auto waves, auto p_staged, auto q_staged) {
        typedef decltype(waves) W;
        each_tiles<W::BM, W::BN>(a, 1, [&](const Product& p, dim3 grid, u64) {
            launch(ring_products<T, P_BY_K, Q_BY_K, decltype(p_staged)::value, decltype(q_staged)::value, W, SUMS && W::ALL == 4, Out>, grid, 64 * W::ALL, stream, p, out);
        });
    };
    const auto by_place = [&](auto waves) {
        const bool p = copied<T>(a.P), q = copied<T>(a.Q);
        if (p && q) return go(waves, Int<0>(), Int<0>());
        if constexpr (sizeof(typename T::elem) == 2) {
            if constexpr (!P_BY_K && Q_BY_K) {
                if (in_pairs<T, P_BY_K, Q_BY_K>(a)) {
                    typedef decltype(waves) W;
                    Product b = a;
                    b.rows = (a.rows + 1) / 2;
                    b.odd_rows = a.rows / 2;
                    return each_tiles<W::BM, W::BN>(b, 2, [&](const Product& p, dim3 grid, u64) {
                        launch(ring_products<T, false, true, false, false, W, false, Out, false, false, true>, grid, 64 * W::ALL, stream, p, out);
                    });
                }
            }
            if constexpr (P_BY_K || !Q_BY_K) if (q) return go(waves, Int<1>(), Int<0>());
            go(waves, Int<1>(), Int<1>());
        }
    };
    if (!in_reach<T>(a.P) || !in_reach<T>(a.Q))
        each_tiles<64, 64>(a, 1, [&](const Product& p, dim3 grid, u64) { launch(tile_products<T, P_BY_K, Q_BY_K, 64, 64, SUMS, Out>, grid, TILE_THREADS, stream, p, out); });
    else if (kind == TILES_64) by_place(Waves<2, 2, 2, 2, 3>());
    else if (kind == TILES_128) by_place(Waves<2, 2, 4, 4, 2>());
    else if constexpr (sizeof(typename T::elem) == 2) by_place(Waves<2, 4, 8, 4, 2>());
}

// Few rows, where a block reads little more of P than of Q, or there are few blocks: with 16 rows of 4096 16-bit values and 16384 columns P's reading takes over (40 us, by tiles 30; with
// 4 rows 30 and 30; of floats 84 and 84, with 8 rows 72 and 83).  In parts that make 512 blocks, of at least two turns of a block's waves each.
static bool few_rows(u64 rows, u64 cols, u32 elem) { return rows <= 4 || (rows <= 16 && (cols <= 8192 || elem == 4)); }
template <class T, class Out>
static void few(Launches& launch, hipStream_t stream, Product a, Out out, PartOut parts) {
    constexpr u32 TURN = FEW_WAVES * 128 / sizeof(typename T::elem);
    const u64 blocks = (a.cols + 15ull) / 16, bytes = a.rows * parts.stride * 4;
    u64 p = 512 / blocks;
    if (p > a.depth / (2 * TURN)) p = a.depth / (2 * TURN);
    if (p > PARTS_MOST) p = PARTS_MOST;
    if (p * bytes > PARTS_BYTES) p = PARTS_BYTES / bytes;
    a.part = a.depth;
    a.parts = 1;
    if (p > 1) {
        a.part = (u32)round_up((a.depth + p - 1) / p, TURN);
        a.parts = (a.depth + a.part - 1) / a.part;
        parts.parts = a.parts;
    }
    for (a.tile0 = 0; a.tile0 < blocks; a.tile0 += 1u << 20) {
        const dim3 grid((u32)(blocks - a.tile0 < (1u << 20) ? blocks - a.tile0 : 1u << 20), 1, a.parts);
        if (a.parts == 1) launch(few_products<T, Out>, grid, 64 * FEW_WAVES, stream, a, out);
        else launch(few_products<T, PartOut>, grid, 64 * FEW_WAVES, stream, a, parts);
    }
    if (a.parts > 1) each_launch<4>(a.rows, a.cols, [&](Units s) { launch(join_parts<Out>, dim3(blocks_of(s.n, 256)), 256, stream, parts, s, out); });
}

// Rows of 16-bit values at multiples of 16 bytes: a thread writes eight, those past a row's end anything.  Bound by memory.
__global__ __launch_bounds__(256) void align_units(Units s, const __bf16* from, u64 from_stride, __bf16* to, u64 to_stride) {
    typedef Vec<BF16, 8> V;                                                          // (either type's: bits)
    const u32 u = blockIdx.x * 256 + threadIdx.x;
    if (u >= s.n) return;
    const u32 row = s.per_row.of(u), c = (u - row * s.per_row.d) * 8;
    const u64 r = s.row0 + row;
    if (c < s.cols) V::store(to + r * to_stride + c, settle_cols<V, 8, false>(load_cols<V, 8, false>(from + r * from_stride, c, s.cols), c, s.cols));
}

// Operands that cannot be copied to LDS as they lie go there through registers, or are laid out anew in the workspace where that takes less time: the way through registers adds 0.5
// to 1.4 times the stages' time where both lie by rows, 1.8 to 4 times where one and 1.2 to 5 times where both lie by k (and are odd), and laying out is a launch and reads and writes them.
// P by rows with Q by k stays: its even and odd rows are two matrices.  Through registers and laid out, in us: 8192 x 4097 x 4097 751 and 353, its input's gradient 878 and 326, its
// weight's 802 and 394; the gradients of 1695 x 3893 x 1167 85 and 40, 160 and 47; of 20000 x 129 x 129 the weight's 19 and 24, by the rule 19.
template <class T, bool P_BY_K, bool Q_BY_K>
static void align(Launches& launch, hipStream_t stream, Product& a, void* aligned) {
    struct { Operand* of; u64 lines, cols; } odd[2];
    u32 n = 0;
    if (!copied<T>(a.P) && (P_BY_K || !Q_BY_K)) odd[n++] = {&a.P, P_BY_K ? a.depth : a.rows, P_BY_K ? a.rows : a.depth};
    if (!copied<T>(a.Q)) odd[n++] = {&a.Q, Q_BY_K ? a.depth : a.cols, Q_BY_K ? a.cols : a.depth};
    if (n == 0 || a.rows == 0 || a.cols == 0 || a.depth == 0) return;
    const double added = P_BY_K ? (n == 2 ? 3.0 : 1.0) : Q_BY_K ? 1.9 : 0.7;
    u64 bytes = 0;
    for (u32 i = 0; i < n; ++i) bytes += aligned_bytes(odd[i].lines, odd[i].cols);
    if (bytes >= ALIGNED_BYTES || way_of(a.rows, a.cols, a.depth, sizeof(typename T::elem)).stages_us * added < 2.7 * n + bytes * 2 / 5e6) return;
    uint8_t* to = (uint8_t*)aligned;
    for (u32 i = 0; i < n; ++i) {
        const u64 stride = aligned_stride(odd[i].cols), from_stride = odd[i].of->stride;
        const __bf16* const from = (const __bf16*)odd[i].of->p;
        each_launch<8>(odd[i].lines, (u32)odd[i].cols, [&](Units s) { launch(align_units, dim3(blocks_of(s.n, 256)), 256, stream, s, from, from_stride, (__bf16*)to, stride); });
        odd[i].of->p = to;
        odd[i].of->stride = stride;
        to += aligned_bytes(odd[i].lines, odd[i].cols);
    }
}

template <class T, bool P_BY_K, bool Q_BY_K, bool SUMS, class Out>
static void products(Launches& launch, hipStream_t stream, Product a, Out out, void* workspace, void* aligned) {
    if constexpr (!P_BY_K && !Q_BY_K) {
        if (few_rows(a.rows, a.cols, sizeof(typename T::elem))) {
            const u64 stride = round_up(a.cols, 4);
            return few<T>(launch, stream, a, out, PartOut{(float*)workspace, stride, a.rows * stride, nullptr, a.rows, 1});
        }
    }
    if constexpr (sizeof(typename T::elem) == 2) align<T, P_BY_K, Q_BY_K>(launch, stream, a, aligned);
    const u32 depth = a.depth + (in_pairs<T, P_BY_K, Q_BY_K>(a) ? 1 : 0);             // (of the longer of two sums: what a part or all parts have to cover)
    Way w = way_of(a.rows, a.cols, depth, sizeof(typename T::elem));
    if (!in_reach<T>(a.P) || !in_reach<T>(a.Q)) w = {TILES_64, 1, 0, 0, 0};
    a.parts = w.parts;
    a.part = w.parts > 1 ? w.part : (u32)round_up(depth ? depth : 1, 64);
    PartOut parts = {(float*)workspace, round_up(a.cols, 4), 0, nullptr, a.rows, a.parts};
    parts.step = a.rows * parts.stride;
    bool row_sums = false;
    if constexpr (SUMS) {
        parts.row_sums = (float*)((uint8_t*)workspace + round_up(parts_bytes(a.rows, a.cols), 256));
        row_sums = out.dbias != nullptr;
        if (row_sums && (w.kind == TILES_256 || a.cols == 0)) {
            // in slices of 64 rows and more, as many as make a thousand blocks
            typedef const typename T::elem* in;
            constexpr u32 WIDTH = 512 / sizeof(typename T::elem);
            const u32 across = (a.rows + WIDTH - 1) / WIDTH;
            u32 slices = 1024 / across < PARTS_MOST ? 1024 / across : PARTS_MOST;
            if (slices > a.depth / 64) slices = a.depth / 64;
            if (slices < 1) slices = 1;
            const u32 slice = (u32)round_up((a.depth + slices - 1) / slices, 8);
            slices = a.depth ? (a.depth + slice - 1) / slice : 1;
            launch(column_sums<T>, dim3(across, slices), 256, stream, (in)a.P.p, a.P.stride, a.depth, a.rows, slice, parts, out);
            if (slices > 1) launch(join_sums, dim3((a.rows + 63) / 64), 64, stream, parts, a.rows, slices, out);
            row_sums = false;
            out.dbias = nullptr;
        }
    }
    if (a.cols == 0) return;
    if (!row_sums) parts.row_sums = nullptr;
    if (w.parts == 1) return tiles<T, P_BY_K, Q_BY_K, SUMS>(launch, stream, a, w.kind, out);
    tiles<T, P_BY_K, Q_BY_K, SUMS>(launch, stream, a, w.kind, parts);
    each_launch<4>(a.rows, a.cols, [&](Units s) { launch(join_parts<Out>, dim3(blocks_of(s.n, 256)), 256, stream, parts, s, out); });
}

extern "C" int dblp_linear(int device, void* stream, uint64_t n_tokens, uint32_t in, uint32_t out, const void* d_x, uint64_t x_stride,
                           const void* d_w, uint64_t w_stride, int type, const void* d_bias, int bias_type, int activation,
                           const void* d_residual, uint64_t residual_stride, void* d_y, uint64_t y_stride, void* d_z, uint64_t z_stride,
                           int out_type, void* d_workspace, uint64_t workspace_bytes) {
    const char* call = "linear";
    REFUSE_IF(bad_type(type) || (out_type != type && out_type != DBLP_F32) || (d_bias && bad_type(bias_type)), "unknown type, or a result that is neither of the operands' type nor fp32");
    REFUSE_IF(bad_act(activation), "unknown activation");
    REFUSE_IF(bad_sizes(n_tokens, in, out), "size out of range");
    const bool some = n_tokens && out, sum = some && in;
    REFUSE_IF((some && !d_y) || (sum && (!d_x || !d_w)), "null pointer");
    const u32 tb = type_bytes(type), ob = type_bytes(out_type);
    REFUSE_IF(off(d_x, tb) || off(d_w, tb) || (d_bias && off(d_bias, type_bytes(bias_type))) || off(d_residual, ob) || off(d_y, ob) || off(d_z, ob), "misaligned pointer");
    REFUSE_IF(n_tokens > 1 && (y_stride < out || (d_z && z_stride < out)), "the output's rows overlap");
    REFUSE_IF(some && d_z == d_y, "z and y are one");
    REFUSE_IF(some && n_tokens > 1 && d_residual == d_y && residual_stride != y_stride, "in place, the strides must be equal");
    REFUSE_IF(!d_workspace || off(d_workspace, 256) || workspace_bytes < dblp_linear_workspace(n_tokens, in, out), "workspace missing, misaligned or too small");
    if (!some) return DBLP_OK;
    OnDevice on(device);
    if (on.err != hipSuccess) return no_device(call, on.err);
    Launches launch;
    const LayerOut o = {out_type, activation, bias_type, d_bias, {(void*)d_residual, residual_stride}, {d_y, y_stride}, {d_z, z_stride}};
    by_type(type, [&](auto tt) {
        products<decltype(tt), false, false, false>(launch, (hipStream_t)stream, Product{{d_x, x_stride, 0}, {d_w, w_stride, 0}, (u32)n_tokens, out, in}, o, d_workspace, (uint8_t*)d_workspace + aligned_at(n_tokens, in, out));
    });
    return launched(call, launch);
}

extern "C" int dblp_linear_grad_input(int device, void* stream, uint64_t n_tokens, uint32_t in, uint32_t out, const void* d_dy,
                                      uint64_t dy_stride, const void* d_w, uint64_t w_stride, int type, const void* d_z, uint64_t z_stride,
                                      int activation, const void* d_base, uint64_t base_stride, void* d_dx, uint64_t dx_stride, int out_type,
                                      void* d_workspace, uint64_t workspace_bytes) {
    const char* call = "linear_grad_input";
    REFUSE_IF(bad_type(type) || (out_type != type && out_type != DBLP_F32), "unknown type, or a result that is neither of the operands' type nor fp32");
    REFUSE_IF(bad_act(activation), "unknown activation");
    REFUSE_IF(bad_sizes(n_tokens, in, out), "size out of range");
    const bool some = n_tokens && in, sum = some && out;
    REFUSE_IF(some && !d_z && activation != DBLP_ACT_NONE, "an activation's slope needs its z");
    REFUSE_IF((some && !d_dx) || (sum && (!d_dy || !d_w)), "null pointer");
    const u32 tb = type_bytes(type), ob = type_bytes(out_type);
    REFUSE_IF(off(d_dy, tb) || off(d_w, tb) || off(d_z, ob) || off(d_base, ob) || off(d_dx, ob), "misaligned pointer");
    REFUSE_IF(n_tokens > 1 && dx_stride < in, "the output's rows overlap");
    REFUSE_IF(some && n_tokens > 1 && ((d_z == d_dx && z_stride != dx_stride) || (d_base == d_dx && base_stride != dx_stride)), "in place, the strides must be equal");
    REFUSE_IF(!d_workspace || off(d_workspace, 256) || workspace_bytes < dblp_linear_workspace(n_tokens, in, out), "workspace missing, misaligned or too small");
    if (!some) return DBLP_OK;
    OnDevice on(device);
    if (on.err != hipSuccess) return no_device(call, on.err);
    Launches launch;
    const GateOut o = {out_type, activation, {(void*)d_z, z_stride}, {(void*)d_base, base_stride}, {d_dx, dx_stride}};
    by_type(type, [&](auto tt) {
        products<decltype(tt), false, true, false>(launch, (hipStream_t)stream, Product{{d_dy, dy_stride, 0}, {d_w, w_stride, 0}, (u32)n_tokens, in, out}, o, d_workspace, (uint8_t*)d_workspace + aligned_at(n_tokens, in, out));
    });
    return launched(call, launch);
}

extern "C" int dblp_linear_grad_weight(int device, void* stream, uint64_t n_tokens, uint32_t in, uint32_t out, const void* d_dy,
                                       uint64_t dy_stride, const void* d_x, uint64_t x_stride, int type, const float* d_base,
                                       uint64_t base_stride, float* d_dw, uint64_t dw_stride, const float* d_bias_base, float* d_dbias,
                                       void* d_workspace, uint64_t workspace_bytes) {
    const char* call = "linear_grad_weight";
    REFUSE_IF(bad_type(type), "unknown type");
    REFUSE_IF(bad_sizes(n_tokens, in, out), "size out of range");
    REFUSE_IF(d_bias_base && !d_dbias, "a bias' base without its gradient");
    const bool some = in && out, any = some || (out && d_dbias);
    REFUSE_IF((some && !d_dw) || (any && n_tokens && (!d_dy || (in && !d_x))), "null pointer");
    const u32 tb = type_bytes(type);
    REFUSE_IF(off(d_dy, tb) || off(d_x, tb) || off(d_base, 4) || off(d_dw, 4) || off(d_bias_base, 4) || off(d_dbias, 4), "misaligned pointer");
    REFUSE_IF(out > 1 && dw_stride < in, "the output's rows overlap");
    REFUSE_IF(some && out > 1 && d_base == d_dw && base_stride != dw_stride, "in place, the strides must be equal");
    REFUSE_IF(!d_workspace || off(d_workspace, 256) || workspace_bytes < dblp_linear_workspace(n_tokens, in, out), "workspace missing, misaligned or too small");
    if (!any) return DBLP_OK;
    OnDevice on(device);
    if (on.err != hipSuccess) return no_device(call, on.err);
    Launches launch;
    const WeightOut o = {d_base, base_stride, d_dw, dw_stride, d_bias_base, d_dbias};
    by_type(type, [&](auto tt) {
        products<decltype(tt), true, true, true>(launch, (hipStream_t)stream, Product{{d_dy, dy_stride, 0}, {d_x, x_stride, 0}, out, in, (u32)n_tokens}, o, d_workspace, (uint8_t*)d_workspace + aligned_at(n_tokens, in, out));
    });
    return launched(call, launch);
}

extern "C" int dblp_activation_grad(int device, void* stream, uint64_t rows, uint32_t cols, const void* d_dy, uint64_t dy_stride,
                                    const void* d_z, uint64_t z_stride, int activation, void* d_dz, uint64_t dz_stride, int type) {
    const char* call = "activation_grad";
    REFUSE_IF(bad_type(type), "unknown type");
    REFUSE_IF(bad_act(activation), "unknown activation");
    REFUSE_IF(cols >= COUNT_LIMIT || rows >= COUNT_LIMIT, "size out of range");
    REFUSE_IF(rows && cols && (!d_dy || !d_z || !d_dz), "null pointer");
    const u32 tb = type_bytes(type);
    REFUSE_IF(off(d_dy, tb) || off(d_z, tb) || off(d_dz, tb), "misaligned pointer");
    REFUSE_IF(rows > 1 && dz_stride < cols, "the output's rows overlap");
    REFUSE_IF(rows > 1 && cols && ((d_dz == d_dy && dz_stride != dy_stride) || (d_dz == d_z && dz_stride != z_stride)), "in place, the strides must be equal");
    if (rows == 0 || cols == 0) return DBLP_OK;
    OnDevice on(device);
    if (on.err != hipSuccess) return no_device(call, on.err);
    Launches launch;
    by_type(type, [&](auto tt) {
        typedef decltype(tt) T;
        typedef const typename T::elem* in;
        constexpr int W = 16 / sizeof(typename T::elem);
        each_launch<W>(rows, cols, [&](Units s) {
            launch(cols % W ? activation_units<T, W, false> : activation_units<T, W, true>, dim3(blocks_of(s.n, 256)), 256, (hipStream_t)stream, s, activation, (in)d_dy, dy_stride, (in)d_z, z_stride,
                   (typename T::elem*)d_dz, dz_stride);
        });
    });
    return launched(call, launch);
}
