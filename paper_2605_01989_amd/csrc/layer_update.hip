// The orthogonalised update of a matrix (include/dblp_layers.h).
#include "layer_tiles.h"

#define STEPS_MOST 16
#define BOUND_MOST 32.0                          // of a singular value
static const double USUAL[3] = {3.4445, -4.7750, 2.0315};

// G as X: r x n with r <= n, turned where G has more rows than columns.
struct Shape { u32 rows, cols; bool tall; };

struct Matrices { const void* p; u64 stride, step; };

// ------------------------------------------------------------------------------------------
// X = G / |G|
// ------------------------------------------------------------------------------------------
#define NORM_EACH 16384                          // values of a block
#define NORM_MOST 256                            // blocks of a matrix
static u32 norm_blocks(u64 values) {
    const u64 n = (values + NORM_EACH - 1) / NORM_EACH;
    return (u32)(n < 1 ? 1 : n < NORM_MOST ? n : NORM_MOST);
}

__device__ __forceinline__ double block_sum(double v) {
    __shared__ double sh[4];
    for (int d = 32; d; d >>= 1) v += __shfl_down(v, d);
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    return sh[0] + sh[1] + sh[2] + sh[3];
}

// Sums of squares of rows blockIdx.x, + gridDim.x, ...: in fp64, where neither a square nor a sum of them leaves the range.
template <class T>
__global__ __launch_bounds__(256) void norm_parts(const typename T::elem* g, u64 stride, u64 step, u32 rows, u32 cols, u64 matrix0, double* parts) {
    const u64 matrix = matrix0 + blockIdx.z;
    const u64 n = (u64)rows * cols;
    double sum = 0;
    for (u64 i = (u64)blockIdx.x * 256 + threadIdx.x; i < n; i += (u64)gridDim.x * 256) {
        const double v = (double)(float)g[matrix * step + i / cols * stride + i % cols];
        sum += v * v;
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) parts[matrix * gridDim.x + blockIdx.x] = sum;
}

// One over the norm; 0 of a matrix of zeros, NaN where a value is not finite.
__device__ __forceinline__ double one_over_norm(const double* parts, u32 n) {
    const double sum = block_sum(threadIdx.x < n ? parts[threadIdx.x] : 0.0);
    return sum == 0.0 ? 0.0 : sum <= DBL_MAX ? 1.0 / sqrt(sum) : NAN;
}

template <class T>
__global__ __launch_bounds__(256) void scale_in(const typename T::elem* g, u64 stride, u64 step, Shape s, u64 matrix0, const double* parts, u32 n_parts, float* x) {
    const u64 matrix = matrix0 + blockIdx.z;
    const double q = one_over_norm(parts + matrix * n_parts, n_parts);
    const u64 n = (u64)s.rows * s.cols;
    for (u64 i = (u64)blockIdx.x * 256 + threadIdx.x; i < n; i += (u64)gridDim.x * 256) {
        const u64 row = i / s.cols, col = i % s.cols;
        x[matrix * n + i] = (float)((double)(float)(s.tall ? g[matrix * step + col * stride + row] : g[matrix * step + row * stride + col]) * q);
    }
}

// ------------------------------------------------------------------------------------------
// what becomes of the products' sums
// ------------------------------------------------------------------------------------------
struct GramOut {
    float* a;
    u64 stride, step, matrix0;
    __device__ __forceinline__ None get(u32, u32, u32, u32) const { return None(); }
    __device__ __forceinline__ void put(u32 matrix, u32, u32 m, u32 n, u32 cols, f4 acc, None) const {
        const float v[4] = {acc[0], acc[1], acc[2], acc[3]};
        store_cols<Vec<F32, 4>, 4>(a + (matrix0 + matrix) * step + m * stride, n, cols, v);
    }
    __device__ __forceinline__ void sums(u32, u32, u32, float) const {}
};
// a I + b A + c A A
struct PolyOut {
    const float* gram;
    float* poly;
    u64 stride, step, matrix0;
    float a, b, c;
    __device__ __forceinline__ None get(u32, u32, u32, u32) const { return None(); }
    __device__ __forceinline__ void put(u32 matrix, u32, u32 m, u32 n, u32 cols, f4 acc, None) const {
        const u64 at = (matrix0 + matrix) * step + m * stride;
        float v[4];
        get4<F32>(gram + at, n, cols, v);
        for (int i = 0; i < 4; ++i) v[i] = b * v[i] + c * acc[i] + (n + i == m ? a : 0.0f);
        store_cols<Vec<F32, 4>, 4>(poly + at, n, cols, v);
    }
    __device__ __forceinline__ void sums(u32, u32, u32, float) const {}
};
template <class T> struct UpdateOut {
    typedef typename T::elem elem;
    float scale, base_scale;
    const elem* base;
    u64 base_stride, base_step;
    elem* out;
    u64 out_stride, out_step, matrix0;
    __device__ __forceinline__ None get(u32, u32, u32, u32) const { return None(); }
    __device__ __forceinline__ void put(u32 matrix, u32, u32 m, u32 n, u32 cols, f4 acc, None) const {
        float v[4], b[4];
        for (int i = 0; i < 4; ++i) v[i] = scale * acc[i];
        if (base) {
            get4<T>(base + (matrix0 + matrix) * base_step + m * base_stride, n, cols, b);
            for (int i = 0; i < 4; ++i) v[i] += base_scale * b[i];
        }
        store_cols<Vec<T, 4>, 4>(out + (matrix0 + matrix) * out_step + m * out_stride, n, cols, v);
    }
    __device__ __forceinline__ void sums(u32, u32, u32, float) const {}
};

// No step: X itself.
template <class T>
__global__ __launch_bounds__(256) void update_plain(const float* x, Shape s, UpdateOut<T> out) {
    const u32 rows = s.tall ? s.cols : s.rows, cols = s.tall ? s.rows : s.cols;
    const u64 units = (cols + 3ull) / 4, n = rows * units;
    x += (out.matrix0 + blockIdx.z) * (u64)s.rows * s.cols;
    for (u64 i = (u64)blockIdx.x * 256 + threadIdx.x; i < n; i += (u64)gridDim.x * 256) {
        const u32 m = (u32)(i / units), c = (u32)(i % units) * 4;
        f4 v = {};
        for (u32 e = 0; e < 4; ++e) if (c + e < cols) v[e] = s.tall ? x[(u64)(c + e) * s.cols + m] : x[(u64)m * s.cols + c + e];
        out.put(blockIdx.z, 0, m, c, cols, v, None());
    }
}

// ------------------------------------------------------------------------------------------
// C-ABI
// ------------------------------------------------------------------------------------------
struct Space { u64 parts, x[2], gram, poly, bytes; };

static Space space_of(u64 count, u64 rows, u64 cols) {
    Space s = {};
    u64 at = 0;
    const u64 r = rows < cols ? rows : cols;
    const auto take = [&](u64 bytes) { const u64 here = at; at += round_up(bytes, 256); return here; };
    s.parts = take(count * norm_blocks(rows * cols) * 8);
    for (int i = 0; i < 2; ++i) s.x[i] = take(count * rows * cols * 4);
    s.gram = take(count * r * r * 4);
    s.poly = take(count * r * r * 4);
    s.bytes = at + 256;
    return s;
}

// Workspaces are held below 2^62 bytes: larger ones do not exist.
static bool out_of_range(u64 count, u64 rows, u64 cols) {
    return count >= COUNT_LIMIT || rows >= COUNT_LIMIT || cols >= COUNT_LIMIT || (double)count * rows * cols > 1e16;
}

extern "C" uint64_t dblp_orthogonalize_workspace(uint64_t count, uint32_t rows, uint32_t cols) {
    return out_of_range(count, rows, cols) ? 0 : space_of(count, rows, cols).bytes;
}

// The largest |a s + b s^3 + c s^5| for s in 0..most: at the end or where the slope a + 3 b q + 5 c q^2, q = s^2, is zero.
static double bound_after(const double* k, double most) {
    const auto value = [&](double q) { return fabs(sqrt(q) * (k[0] + q * (k[1] + q * k[2]))); };
    const double end = most * most;
    double best = value(end);
    const auto at = [&](double q) { if (q > 0 && q < end && value(q) > best) best = value(q); };
    if (k[2] == 0.0) {
        if (k[1] != 0.0) at(-k[0] / (3 * k[1]));
        return best;
    }
    const double d = 9 * k[1] * k[1] - 20 * k[0] * k[2];
    if (d < 0) return best;
    at((-3 * k[1] + sqrt(d)) / (10 * k[2]));
    at((-3 * k[1] - sqrt(d)) / (10 * k[2]));
    return best;
}

extern "C" int dblp_orthogonalize(int device, void* stream, uint64_t count, uint32_t rows, uint32_t cols, const void* d_g, uint64_t g_stride,
                                  uint64_t g_step, int g_type, const double* h_coefficients, uint32_t steps, float scale, const void* d_base,
                                  uint64_t base_stride, uint64_t base_step, float base_scale, void* d_out, uint64_t out_stride,
                                  uint64_t out_step, int out_type, void* d_workspace, uint64_t workspace_bytes) {
    const char* call = "orthogonalize";
    REFUSE_IF(bad_type(g_type) || bad_type(out_type), "unknown type");
    REFUSE_IF(out_of_range(count, rows, cols), "size out of range");
    REFUSE_IF(steps > STEPS_MOST, "more than 16 steps");
    REFUSE_IF(!(fabsf(scale) <= FLT_MAX) || !(fabsf(base_scale) <= FLT_MAX), "a scale is not finite");
    double bounds[STEPS_MOST + 1] = {1.0};
    for (u32 i = 0; i < steps; ++i) {
        const double* k = h_coefficients ? h_coefficients + 3 * i : USUAL;
        bounds[i + 1] = bound_after(k, bounds[i] * (1 + 1e-6));
        REFUSE_IF(!(fabs(k[0]) <= FLT_MAX && fabs(k[1]) <= FLT_MAX && fabs(k[2]) <= FLT_MAX && bounds[i + 1] <= BOUND_MOST), "coefficients under which a singular value could pass 32");
    }
    const bool some = count && rows && cols;
    REFUSE_IF(some && (!d_g || !d_out), "null pointer");
    REFUSE_IF(off(d_g, type_bytes(g_type)) || off(d_base, type_bytes(out_type)) || off(d_out, type_bytes(out_type)), "misaligned pointer");
    REFUSE_IF(rows > 1 && out_stride < cols, "the output's rows overlap");
    REFUSE_IF(some && count > 1 && out_step < (u64)(rows - 1) * out_stride + cols && !(out_step >= cols && out_stride >= (count - 1) * out_step + cols), "the output's matrices overlap");
    REFUSE_IF(some && d_base == d_out && ((rows > 1 && base_stride != out_stride) || (count > 1 && base_step != out_step)), "in place, strides and steps must be equal");
    REFUSE_IF(some && d_g == d_out && (g_type != out_type || (rows > 1 && g_stride != out_stride) || (count > 1 && g_step != out_step)), "in place, types, strides and steps must be equal");
    REFUSE_IF(!d_workspace || off(d_workspace, 256) || workspace_bytes < space_of(count, rows, cols).bytes, "workspace missing, misaligned or too small");
    if (!some) return DBLP_OK;
    OnDevice on(device);
    if (on.err != hipSuccess) return no_device(call, on.err);
    Launches launch;
    const hipStream_t st = (hipStream_t)stream;
    const Space at = space_of(count, rows, cols);
    uint8_t* const ws = (uint8_t*)d_workspace;
    double* const parts = (double*)(ws + at.parts);
    float *x = (float*)(ws + at.x[0]), *next = (float*)(ws + at.x[1]);
    float *const gram = (float*)(ws + at.gram), *const poly = (float*)(ws + at.poly);
    const bool tall = rows > cols;
    const Shape s = {tall ? cols : rows, tall ? rows : cols, tall};
    const u64 values = (u64)rows * cols, square = (u64)s.rows * s.rows;
    const u32 n_parts = norm_blocks(values);
    const auto each_matrix = [&](auto f) { for (u64 m = 0; m < count; m += 32768) f(m, (u32)(count - m < 32768 ? count - m : 32768)); };
    each_matrix([&](u64 m, u32 n) {
        by_type(g_type, [&](auto tt) {
            typedef decltype(tt) T;
            typedef const typename T::elem* in;
            launch(norm_parts<T>, dim3(n_parts, 1, n), 256, st, (in)d_g, (u64)g_stride, (u64)g_step, rows, cols, m, parts);
            launch(scale_in<T>, dim3(n_parts, 1, n), 256, st, (in)d_g, (u64)g_stride, (u64)g_step, s, m, (const double*)parts, n_parts, x);
        });
    });
    const auto product = [&](auto p_by_k, auto q_by_k, Operand P, Operand Q, u32 m_rows, u32 m_cols, u32 depth, auto out) {
        constexpr bool PK = decltype(p_by_k)::value, QK = decltype(q_by_k)::value;
        typedef decltype(out) Out;
        const Product a = {P, Q, m_rows, m_cols, depth, 0, (u32)round_up(depth, 64), 1};
        each_tiles<64, 64>(a, count, [&](Product p, dim3 grid, u64 m) {
            out.matrix0 = m;
            p.P.p = (const float*)P.p + m * P.step;
            p.Q.p = (const float*)Q.p + m * Q.step;
            launch(tile_products<F32, PK, QK, 64, 64, false, Out>, grid, TILE_THREADS, st, p, out);
        });
    };
    by_type(out_type, [&](auto tt) {
        typedef decltype(tt) T;
        typedef typename T::elem elem;
        const UpdateOut<T> update = {scale, base_scale, (const elem*)d_base, base_stride, base_step, (elem*)d_out, out_stride, out_step, 0};
        if (steps == 0) {
            each_matrix([&](u64 m, u32 n) {
                UpdateOut<T> u = update;
                u.matrix0 = m;
                launch(update_plain<T>, dim3(n_parts, 1, n), 256, st, (const float*)x, s, u);
            });
            return;
        }
        for (u32 i = 0; i < steps; ++i) {
            const double* k = h_coefficients ? h_coefficients + 3 * i : USUAL;
            const Operand X = {x, s.cols, values}, A = {gram, s.rows, square}, P = {poly, s.rows, square};
            product(Int<0>(), Int<0>(), X, X, s.rows, s.rows, s.cols, GramOut{gram, s.rows, square, 0});
            product(Int<0>(), Int<0>(), A, A, s.rows, s.rows, s.rows, PolyOut{gram, poly, s.rows, square, 0, (float)k[0], (float)k[1], (float)k[2]});
            if (i + 1 < steps) product(Int<0>(), Int<1>(), P, X, s.rows, s.cols, s.rows, GramOut{next, s.cols, values, 0});
            else if (tall) product(Int<1>(), Int<0>(), X, P, s.cols, s.rows, s.rows, update);
            else product(Int<0>(), Int<1>(), P, X, s.rows, s.cols, s.rows, update);
            float* const t = x;
            x = next;
            next = t;
        }
    });
    return launched(call, launch);
}
