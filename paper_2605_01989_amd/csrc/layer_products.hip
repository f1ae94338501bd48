// A worker's matrix products and their gradients (include/dblp_layers.h).
#include "layer_tiles.h"

// ------------------------------------------------------------------------------------------
// activations and their slopes
// ------------------------------------------------------------------------------------------
#define ROOT_HALF 0.70710678118654752f
#define ROOT_TWO_OVER_PI 0.79788456080286536f
#define CUBE 0.044715f

__device__ __forceinline__ float one_over(float x) { return __builtin_amdgcn_rcpf(x); }
// tanh's argument of GELU_TANH, twice and negated.  Past 30 the exponential has long been zero or infinity: the cube of a
// larger z would pass fp32 where zero times it is wanted.
__device__ __forceinline__ float tanh_power(float z) {
    const float t = fminf(fmaxf(z, -30.0f), 30.0f);
    return -2.0f * ROOT_TWO_OVER_PI * t * (1.0f + CUBE * t * t);
}
__device__ __forceinline__ float act_of(int act, float z) {
    switch (act) {
        case DBLP_ACT_RELU: return z <= 0.0f ? 0.0f : z;
        case DBLP_ACT_GELU: return 0.5f * z * erfcf(-z * ROOT_HALF);
        case DBLP_ACT_GELU_TANH: return z * one_over(1.0f + expf(tanh_power(z)));
        case DBLP_ACT_SILU: return z * one_over(1.0f + expf(-z));
        default: return z;
    }
}
// dy act'(z)
__device__ __forceinline__ float gated(int act, float z, float dy) {
    switch (act) {
        case DBLP_ACT_RELU: return z > 0.0f ? dy : 0.0f;
        case DBLP_ACT_GELU: return dy * (0.5f * erfcf(-z * ROOT_HALF) + z * (expf(-0.5f * z * z) * (0.5f * ROOT_TWO_OVER_PI)));
        case DBLP_ACT_GELU_TANH: {
            const float e = expf(tanh_power(z)), p = one_over(1.0f + e), t = fminf(fmaxf(z, -30.0f), 30.0f);
            const float rest = e < 1e30f ? e * p : 1.0f;                        // 1 - p
            return dy * (p + z * (p * rest * (2.0f * ROOT_TWO_OVER_PI * (1.0f + 3.0f * CUBE * t * t))));
        }
        case DBLP_ACT_SILU: {
            const float e = expf(-z), p = one_over(1.0f + e), rest = e < 1e30f ? e * p : 1.0f;
            return dy * (p + z * (p * rest));
        }
        default: return dy;
    }
}

// ------------------------------------------------------------------------------------------
// what becomes of a product's sums
// ------------------------------------------------------------------------------------------
// A matrix of a type that is known when the kernel runs: four columns of a row.
struct Matrix { void* p; u64 stride; };

__device__ __forceinline__ void load4(int type, const void* p, u64 at, u32 left, float (&v)[4]) {
    if (type == DBLP_F32) get4<F32>((const float*)p + at, 0, left, v);
    else if (type == DBLP_BF16) get4<BF16>((const __bf16*)p + at, 0, left, v);
    else get4<F16>((const _Float16*)p + at, 0, left, v);
}
__device__ __forceinline__ void store4(int type, void* p, u64 at, u32 left, const float (&v)[4]) {
    if (type == DBLP_F32) store_cols<Vec<F32, 4>, 4>((float*)p + at, 0, left, v);
    else if (type == DBLP_BF16) store_cols<Vec<BF16, 4>, 4>((__bf16*)p + at, 0, left, v);
    else store_cols<Vec<F16, 4>, 4>((_Float16*)p + at, 0, left, v);
}

struct LayerOut {
    int type, act, bias_type;
    const void* bias;
    Matrix residual, y, z;
    __device__ __forceinline__ void put(u32, u32, u32 m, u32 n, u32 cols, f4 acc) const {
        float v[4] = {acc[0], acc[1], acc[2], acc[3]}, b[4];
        if (bias) {
            load4(bias_type, bias, n, cols - n, b);
            for (int i = 0; i < 4; ++i) v[i] += b[i];
        }
        if (z.p) store4(type, z.p, m * z.stride + n, cols - n, v);
        for (int i = 0; i < 4; ++i) v[i] = act_of(act, v[i]);
        if (residual.p) {
            load4(type, residual.p, m * residual.stride + n, cols - n, b);
            for (int i = 0; i < 4; ++i) v[i] += b[i];
        }
        store4(type, y.p, m * y.stride + n, cols - n, v);
    }
    __device__ __forceinline__ void sums(u32, u32, u32, float) const {}
};

struct GateOut {
    int type, act;
    Matrix z, base, dx;
    __device__ __forceinline__ void put(u32, u32, u32 m, u32 n, u32 cols, f4 acc) const {
        float v[4] = {acc[0], acc[1], acc[2], acc[3]}, b[4];
        if (z.p) {
            load4(type, z.p, m * z.stride + n, cols - n, b);
            for (int i = 0; i < 4; ++i) v[i] = gated(act, b[i], v[i]);
        }
        if (base.p) {
            load4(type, base.p, m * base.stride + n, cols - n, b);
            for (int i = 0; i < 4; ++i) v[i] += b[i];
        }
        store4(type, dx.p, m * dx.stride + n, cols - n, v);
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
    __device__ __forceinline__ void put(u32, u32, u32 m, u32 n, u32 cols, f4 acc) const {
        float v[4] = {acc[0], acc[1], acc[2], acc[3]}, b[4];
        if (base) {
            get4<F32>(base + m * base_stride, n, cols, b);
            for (int i = 0; i < 4; ++i) v[i] += b[i];
        }
        store_cols<Vec<F32, 4>, 4>(dw + m * dw_stride, n, cols, v);
    }
    __device__ __forceinline__ void sums(u32, u32, u32 m, float s) const { if (dbias) dbias[m] = bias_base ? bias_base[m] + s : s; }
};

// ------------------------------------------------------------------------------------------
// activation_grad: a thread takes 16 bytes
// ------------------------------------------------------------------------------------------
template <class T, int W>
__global__ __launch_bounds__(256) void activation_units(Units s, int act, const typename T::elem* dy, u64 dy_stride, const typename T::elem* z, u64 z_stride, typename T::elem* dz, u64 dz_stride) {
    typedef Vec<T, W> V;
    const u32 u = blockIdx.x * 256 + threadIdx.x;
    if (u >= s.n) return;
    const u32 row = s.per_row.of(u), c = (u - row * s.per_row.d) * W;
    if (c >= s.cols) return;
    const u64 r = s.row0 + row;
    float a[W], b[W];
    V::open(settle_cols<V, W, false>(load_cols<V, W, false>(dy + r * dy_stride, c, s.cols), c, s.cols), a);
    V::open(settle_cols<V, W, false>(load_cols<V, W, false>(z + r * z_stride, c, s.cols), c, s.cols), b);
    for (int i = 0; i < W; ++i) a[i] = gated(act, b[i], a[i]);
    store_cols<V, W>(dz + r * dz_stride, c, s.cols, a);
}

// ------------------------------------------------------------------------------------------
// C-ABI
// ------------------------------------------------------------------------------------------
static bool bad_act(int act) { return act < DBLP_ACT_NONE || act > DBLP_ACT_SILU; }
static bool bad_sizes(u64 tokens, u64 in, u64 out) { return tokens >= COUNT_LIMIT || in >= COUNT_LIMIT || out >= COUNT_LIMIT; }

extern "C" uint64_t dblp_linear_workspace(uint64_t n_tokens, uint32_t in, uint32_t out) {
    return bad_sizes(n_tokens, in, out) ? 0 : 256;
}

template <class T, bool P_BY_K, bool Q_BY_K, bool SUMS, class Out>
static void products(Launches& launch, hipStream_t stream, Product a, Out out) {
    a.part = (u32)round_up(a.depth ? a.depth : 1, 64);
    a.parts = 1;
    const u64 area = (u64)a.rows * a.cols;
    if (!in_reach<T>(a.P) || !in_reach<T>(a.Q)) {
        each_tiles<64, 64>(a, 1, [&](const Product& p, dim3 grid, u64) { launch(tile_products<T, P_BY_K, Q_BY_K, 64, 64, SUMS, Out>, grid, TILE_THREADS, stream, p, out); });
        return;
    }
    const auto go = [&](auto waves, auto p_staged, auto q_staged) {
        typedef decltype(waves) W;
        each_tiles<W::BM, W::BN>(a, 1, [&](const Product& p, dim3 grid, u64) {
            launch(ring_products<T, P_BY_K, Q_BY_K, decltype(p_staged)::value, decltype(q_staged)::value, W, SUMS && (W::ALL == 4), Out>, grid, 64 * W::ALL, stream, p, out);
        });
    };
    const auto by_rows = [&](auto waves) {
        const bool p = in_chunks<T>(a.P), q = in_chunks<T>(a.Q);
        if (p && q) go(waves, Int<0>(), Int<0>());
        else if (q) go(waves, Int<1>(), Int<0>());
        else go(waves, Int<1>(), Int<1>());
    };
    if (area < (u64)256 * 128 * 128) by_rows(Waves<2, 2, 2, 2, 3>());
    else if (sizeof(typename T::elem) == 4 || area < (u64)200 * 256 * 256) by_rows(Waves<2, 2, 4, 4, 2>());
    else if constexpr (sizeof(typename T::elem) == 2) by_rows(Waves<2, 4, 8, 4, 2>());
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
        products<decltype(tt), false, false, false>(launch, (hipStream_t)stream, Product{{d_x, x_stride, 0}, {d_w, w_stride, 0}, (u32)n_tokens, out, in}, o);
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
        products<decltype(tt), false, true, false>(launch, (hipStream_t)stream, Product{{d_dy, dy_stride, 0}, {d_w, w_stride, 0}, (u32)n_tokens, in, out}, o);
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
        products<decltype(tt), true, true, true>(launch, (hipStream_t)stream, Product{{d_dy, dy_stride, 0}, {d_x, x_stride, 0}, out, in, (u32)n_tokens}, o);
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
            launch(activation_units<T, W>, dim3(blocks_of(s.n, 256)), 256, (hipStream_t)stream, s, activation, (in)d_dy, dy_stride, (in)d_z, z_stride, (typename T::elem*)d_dz, dz_stride);
        });
    });
    return launched(call, launch);
}
