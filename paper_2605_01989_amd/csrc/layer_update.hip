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
#define NORM_EACH 4096                           // values of a block
#define NORM_MOST 256                            // blocks of a matrix
static u32 norm_blocks(u64 values) {
    const u64 n = (values + NORM_EACH - 1) / NORM_EACH;
    return (u32)(n < 1 ? 1 : n < NORM_MOST ? n : NORM_MOST);
}

template <int WAVES>
__device__ __forceinline__ double block_sum(double v) {
    __shared__ double sh[WAVES];
    for (int d = 32; d; d >>= 1) v += __shfl_down(v, d);
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
    for (int i = 0; i < WAVES; ++i) v += sh[i];
    return v;
}

// Sums of squares, in fp64, where neither a square nor a sum of them leaves the range.  `across` threads, a power of two, take a row, four values each at a time; a
// thread has four rows' on their way.  Bound by memory, and by the fp64 sums: 134 MB in 46 us (2.9 TB/s).
template <class T>
__global__ __launch_bounds__(256) void norm_parts(const typename T::elem* g, u64 stride, u64 step, u32 rows, u32 cols, u32 across, u64 matrix0, double* parts) {
    typedef Vec<T, 4> V;
    const u64 matrix = matrix0 + blockIdx.z;
    const u32 down = 256 / across, x = threadIdx.x % across, y = threadIdx.x / across, turn = gridDim.x * down;
    g += matrix * step;
    double sum = 0;
    for (u64 row = blockIdx.x * down + y; row < rows; row += 4ull * turn)
        for (u32 c = x * 4; c < cols; c += across * 4) {
            typename V::raw r[4];
#pragma unroll
            for (u32 i = 0; i < 4; ++i) {
                r[i] = (typename V::raw)(0);
                const u64 at = row + (u64)i * turn;
                if (at < rows) r[i] = c + 4 <= cols ? V::load(g + at * stride + c) : V::some(g + at * stride + c, cols - c);
            }
#pragma unroll
            for (u32 i = 0; i < 4; ++i) {
                float v[4];
                V::open(r[i], v);
                for (int e = 0; e < 4; ++e) sum += (double)v[e] * (double)v[e];
            }
        }
    sum = block_sum<4>(sum);
    if (threadIdx.x == 0) parts[matrix * gridDim.x + blockIdx.x] = sum;
}

// One over the norm; 0 of a matrix of zeros, NaN where a value is not finite.  (n is 256 at most.)
template <int WAVES>
__device__ __forceinline__ double one_over_norm(const double* parts, u32 n) {
    const double sum = block_sum<WAVES>(threadIdx.x < n ? parts[threadIdx.x] : 0.0);
    return sum == 0.0 ? 0.0 : sum <= DBL_MAX ? 1.0 / sqrt(sum) : NAN;
}

// A value in halves: the nearest fp16 value, and the nearest one to 2^11 times what that leaves, which is no larger than the value.  Both are of the value times a power of two that takes the
// largest one possible to 2^14 and more, below 2^15, so that a value keeps 22 bits, or 2^-50 of that largest one (without the factor 2^-39: a row 2^-24 as large as the rest was off by 2^-7 to 2^-10).
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
struct Halves { half4 high, low; };
__device__ __forceinline__ Halves halves_of(const float (&v)[4]) {
    Halves h;
    for (int i = 0; i < 4; ++i) {
        h.high[i] = (_Float16)v[i];
        h.low[i] = (_Float16)fmaf((float)h.high[i], -LOW_UP, v[i] * LOW_UP);
    }
    return h;
}
__device__ __forceinline__ float value_of(_Float16 high, _Float16 low) { return (float)high + (float)low * LOW_DOWN; }
struct HalvesAt {
    _Float16* p;
    u64 stride, step, low;       // of rows, of matrices, from the high halves to the low ones
    __device__ __forceinline__ void put(u64 matrix, u32 m, u32 n, const float (&v)[4]) const {
        const Halves h = halves_of(v);
        _Float16* const at = p + matrix * step + m * stride + n;
        *(half4*)at = h.high;
        *(half4*)(at + low) = h.low;
    }
    __device__ __forceinline__ Halves get(u64 matrix, u32 m, u32 n) const {
        const _Float16* const at = p + matrix * step + m * stride + n;
        return {*(const half4*)at, *(const half4*)(at + low)};
    }
};

// X in halves, zeros behind its rows and columns: a block takes 64 x 64 of them, through LDS where G is turned.  Bound by memory: 134 MB to 134 in 42 us (6.4 TB/s).
template <class T>
__global__ __launch_bounds__(256) void scale_in(const typename T::elem* g, u64 stride, u64 step, Shape s, u64 matrix0, const double* parts, u32 n_parts, float up, HalvesAt x) {
    typedef Vec<T, 4> V;
    __shared__ float turned[64][65];
    const u64 matrix = matrix0 + blockIdx.z;
    const u32 row0 = blockIdx.y * 64, col0 = blockIdx.x * 64, down = threadIdx.x / 16, across = threadIdx.x % 16 * 4;
    const u32 g_rows = s.tall ? s.cols : s.rows, g_cols = s.tall ? s.rows : s.cols, g_row = (s.tall ? col0 : row0) + down, g_col = (s.tall ? row0 : col0) + across;
    g += matrix * step;
    typename V::raw r[4];
#pragma unroll
    for (u32 i = 0; i < 4; ++i) {
        r[i] = (typename V::raw)(0);
        const typename T::elem* const at = g + (u64)(g_row + 16 * i) * stride + g_col;
        if (g_row + 16 * i < g_rows && g_col < g_cols) r[i] = g_col + 4 <= g_cols ? V::load(at) : V::some(at, g_cols - g_col);
    }
    const double q = one_over_norm<4>(parts + matrix * n_parts, n_parts) * up;
#pragma unroll
    for (u32 i = 0; i < 4; ++i) {
        float v[4];
        V::open(r[i], v);
        // (zeros behind the matrix stay zeros where the norm is NaN)
        for (int e = 0; e < 4; ++e) v[e] = g_row + 16 * i < g_rows && g_col + e < g_cols ? (float)((double)v[e] * q) : 0.0f;
        if (s.tall)
            for (int e = 0; e < 4; ++e) turned[across + e][down + 16 * i] = v[e];
        else
            x.put(matrix, row0 + down + 16 * i, col0 + across, v);
    }
    if (!s.tall) return;
    __syncthreads();
#pragma unroll
    for (u32 i = 0; i < 4; ++i) {
        float v[4];
        for (int e = 0; e < 4; ++e) v[e] = turned[down + 16 * i][across + e];
        x.put(matrix, row0 + down + 16 * i, col0 + across, v);
    }
}

// ------------------------------------------------------------------------------------------
// what becomes of the products' sums: everything of X, A and b A + c A A is in halves, of padded rows and columns, whose sums are zeros.  Three products of halves take the place of one of
// floats on units of sixteen times the rate: X X^T of 4096 x 8192 on and above the diagonal 387 us (1.10 PFLOP/s of fp16), A A 222, P X 646 (1.28 PFLOP/s).
// ------------------------------------------------------------------------------------------
struct GramOut {
    HalvesAt a;
    float by;                    // from the operands' powers of two to the result's
    u64 matrix0;
    __device__ __forceinline__ None get(u32, u32, u32, u32) const { return None(); }
    __device__ __forceinline__ void put(u32 matrix, u32, u32 m, u32 n, u32, f4 acc, None) const {
        const float v[4] = {acc[0] * by, acc[1] * by, acc[2] * by, acc[3] * by};
        a.put(matrix0 + matrix, m, n, v);
    }
    __device__ __forceinline__ void sums(u32, u32, u32, float) const {}
};
// a I + b A + c A A
struct PolyOut {
    HalvesAt gram, poly;
    float a, b, c;               // (with the powers of two)
    u32 rows;                    // without the padding
    u64 matrix0;
    __device__ __forceinline__ Halves get(u32 matrix, u32 m, u32 n, u32) const { return gram.get(matrix0 + matrix, m, n); }
    __device__ __forceinline__ void put(u32 matrix, u32, u32 m, u32 n, u32, f4 acc, const Halves& g) const {
        float v[4];
        for (int i = 0; i < 4; ++i) v[i] = b * value_of(g.high[i], g.low[i]) + c * acc[i] + (n + i == m && m < rows ? a : 0.0f);
        poly.put(matrix0 + matrix, m, n, v);
    }
    __device__ __forceinline__ void sums(u32, u32, u32, float) const {}
};
struct UpdateOut {
    int type;
    float scale, base_scale;
    const void* base;
    u64 base_stride, base_step;
    void* out;
    u64 out_stride, out_step, matrix0;
    __device__ __forceinline__ u4v get(u32 matrix, u32 m, u32 n, u32 cols) const { return base ? raw4(type, base, (matrix0 + matrix) * base_step + m * base_stride + n, cols - n) : (u4v)(0u); }
    __device__ __forceinline__ void put(u32 matrix, u32, u32 m, u32 n, u32 cols, f4 acc, u4v met) const {
        float v[4], b[4];
        for (int i = 0; i < 4; ++i) v[i] = scale * acc[i];
        if (base) {
            open4(type, met, b);
            for (int i = 0; i < 4; ++i) v[i] += base_scale * b[i];
        }
        store4(type, out, (matrix0 + matrix) * out_step + m * out_stride + n, cols - n, v);
    }
    __device__ __forceinline__ void sums(u32, u32, u32, float) const {}
};

// ------------------------------------------------------------------------------------------
// Small matrices, X of at most 64 R x 64 N: a block takes one through all of its steps, X and then A, then a + b A + c A A, in halves in LDS.  Eight waves, four by two, each 16 R x
// 32 R columns of A and 16 R x 32 N of X.  What bounds it is the way from one product to the next: reading, multiplying, a barrier, writing.  128 x 128 in five steps 51 us (four and
// sixteen waves are slower), 91 as products of tiles through memory.
// A row in LDS is 128 bytes for each 64 values, chunk c of 16 bytes of row r at c ^ (r & 7).
// ------------------------------------------------------------------------------------------
template <int WIDTH> __device__ __forceinline__ u32 small_at(u32 row, u32 col) { return row * (WIDTH * 2) + (((col >> 3) ^ (row & 7)) << 4) + (col & 7) * 2; }

// 16 rows' (or, by k, columns') 32 k of a matrix in LDS.
template <int WIDTH>
__device__ __forceinline__ u4v small_rows(const uint8_t* m, u32 row0, u32 k0) {
    const u32 lane = threadIdx.x & 63;
    return *(const u4v*)(m + small_at<WIDTH>(row0 + (lane & 15), k0 + (lane >> 4) * 8));
}
template <int WIDTH>
__device__ __forceinline__ u4v small_columns(const uint8_t* m, u32 col0, u32 k0) {
    typedef short s4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s4* lds;
    const u32 lane = threadIdx.x & 63, k = k0 + (lane >> 4) * 8 + ((lane & 15) >> 2), col = col0 + (lane & 3) * 4;
    const u2v a = __builtin_bit_cast(u2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(m + small_at<WIDTH>(k, col)))), b = __builtin_bit_cast(u2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(m + small_at<WIDTH>(k + 4, col))));
    return (u4v){a.x, a.y, b.x, b.y};
}
template <int WIDTH>
__device__ __forceinline__ void small_put(uint8_t* m, u32 low, u32 row, u32 col, const float (&v)[4]) {
    const Halves h = halves_of(v);
    *(half4*)(m + small_at<WIDTH>(row, col)) = h.high;
    *(half4*)(m + low + small_at<WIDTH>(row, col)) = h.low;
}

// low by high and high by low to sums of their own, high by high: each a round over the results, whose sums wait for each other.  TURNED: a result's rows and columns change places.
template <int R, int C, bool TURNED = false>
__device__ __forceinline__ void add_halves(f4 (&acc)[R][C], f4 (&low)[R][C], const u4v (&bh)[R], const u4v (&bl)[R], const u4v (&ch)[C], const u4v (&cl)[C]) {
    const auto round = [&](f4 (&to)[R][C], const u4v (&b)[R], const u4v (&c)[C]) {
#pragma unroll
        for (int j = 0; j < C; ++j)
#pragma unroll
            for (int e = 0; e < R; ++e) to[e][j] = TURNED ? mfma<F16>(b[e], c[j], to[e][j]) : mfma<F16>(c[j], b[e], to[e][j]);
    };
    round(low, bl, ch);
    round(low, bh, cl);
    round(acc, bh, ch);
}
template <int R, int C>
__device__ __forceinline__ void join_halves(f4 (&acc)[R][C], const f4 (&low)[R][C]) {
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
        for (int e = 0; e < R; ++e) acc[e][j] += low[e][j] * LOW_DOWN;
}

struct SmallSteps { float gram[STEPS_MOST], a[STEPS_MOST], b[STEPS_MOST], c[STEPS_MOST], next[STEPS_MOST]; u32 n; };

template <int R, int N>
struct Small {
    static constexpr u32 ROWS = 64 * R, COLS = 64 * N, X_LOW = ROWS * COLS * 2, A_LOW = ROWS * ROWS * 2, EACH = ROWS * COLS / 2048;       // EACH: fours of X of a thread
    u32 group, in_group, m0, an0, xn0;
    __device__ __forceinline__ Small() {
        const u32 lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        group = lane >> 4;
        in_group = lane & 15;
        m0 = wave / 2 * 16 * R;
        an0 = wave % 2 * 32 * R;
        xn0 = wave % 2 * 32 * N;
    }
    // Values of G on their way to X's columns col0 and up.
    template <class T> struct Values {
        typedef Vec<T, 4> V;
        typename V::raw r[EACH];
        u32 rows, cols, across, row0, col0;
        bool tall;
        __device__ __forceinline__ Values(const typename T::elem* g, u64 stride, const Shape& s, u32 first) : tall(s.tall) {
            rows = tall ? s.cols : s.rows;
            cols = tall ? s.rows : s.cols;
            across = (tall ? ROWS : COLS) / 4;
            row0 = tall ? first : 0;
            col0 = tall ? 0 : first;
#pragma unroll
            for (u32 i = 0; i < EACH; ++i) {
                r[i] = (typename V::raw)(0);
                const u32 row = row0 + at(i) / across, col = col0 + at(i) % across * 4;
                if (row < rows && col < cols) r[i] = col + 4 <= cols ? V::load(g + row * stride + col) : V::some(g + row * stride + col, cols - col);
            }
        }
        static __device__ __forceinline__ u32 at(u32 i) { return threadIdx.x + i * 512; }
        __device__ __forceinline__ double squares() const {
            double sum = 0;
#pragma unroll
            for (u32 i = 0; i < EACH; ++i) {
                float v[4];
                V::open(r[i], v);
                for (int e = 0; e < 4; ++e) sum += (double)v[e] * (double)v[e];
            }
            return sum;
        }
        // (zeros behind the matrix stay zeros where the norm is NaN)
        __device__ __forceinline__ void put(uint8_t* x, double q) const {
#pragma unroll
            for (u32 i = 0; i < EACH; ++i) {
                const u32 row = at(i) / across, col = at(i) % across * 4;
                float v[4];
                V::open(r[i], v);
                for (int e = 0; e < 4; ++e) v[e] = row0 + row < rows && col0 + col + e < cols ? (float)((double)v[e] * q) : 0.0f;
                if (!tall) small_put<COLS>(x, X_LOW, row, col, v);
                else
                    for (int e = 0; e < 4; ++e) {
                        const _Float16 high = (_Float16)v[e];
                        *(_Float16*)(x + small_at<COLS>(col + e, row)) = high;
                        *(_Float16*)(x + X_LOW + small_at<COLS>(col + e, row)) = (_Float16)fmaf((float)high, -LOW_UP, v[e] * LOW_UP);
                    }
            }
        }
    };
    // acc += M M^T of a matrix of WIDTH columns
    template <int WIDTH>
    __device__ __forceinline__ void square(f4 (&acc)[R][2 * R], const uint8_t* of, u32 low) const {
        f4 small[R][2 * R] = {};
#pragma unroll
        for (u32 k0 = 0; k0 < WIDTH; k0 += 32) {
            u4v bh[R], bl[R], ch[2 * R], cl[2 * R];
#pragma unroll
            for (int e = 0; e < R; ++e) { bh[e] = small_rows<WIDTH>(of, m0 + 16 * e, k0); bl[e] = small_rows<WIDTH>(of + low, m0 + 16 * e, k0); }
#pragma unroll
            for (int j = 0; j < 2 * R; ++j) { ch[j] = small_rows<WIDTH>(of, an0 + 16 * j, k0); cl[j] = small_rows<WIDTH>(of + low, an0 + 16 * j, k0); }
            add_halves<R, 2 * R>(acc, small, bh, bl, ch, cl);
        }
        join_halves<R, 2 * R>(acc, small);
    }
    // From A's sums a + b A + c A A to m, A by the way there too; a wave's part of A A is at the same places as its part of A.
    __device__ __forceinline__ void poly(f4 (&acc)[R][2 * R], uint8_t* m, u32 rows, float gram, float a, float b, float c) const {
        Halves own[R][2 * R];
#pragma unroll
        for (int e = 0; e < R; ++e)
#pragma unroll
            for (int j = 0; j < 2 * R; ++j) {
                float v[4];
                for (int t = 0; t < 4; ++t) v[t] = acc[e][j][t] * gram;
                own[e][j] = halves_of(v);
                const u32 row = m0 + 16 * e + in_group, col = an0 + 16 * j + group * 4;
                *(half4*)(m + small_at<ROWS>(row, col)) = own[e][j].high;
                *(half4*)(m + A_LOW + small_at<ROWS>(row, col)) = own[e][j].low;
                acc[e][j] = (f4)(0.0f);
            }
        __syncthreads();
        square<ROWS>(acc, m, A_LOW);
        __syncthreads();
#pragma unroll
        for (int e = 0; e < R; ++e)
#pragma unroll
            for (int j = 0; j < 2 * R; ++j) {
                const u32 row = m0 + 16 * e + in_group, col = an0 + 16 * j + group * 4;
                float v[4];
                for (int t = 0; t < 4; ++t) v[t] = b * value_of(own[e][j].high[t], own[e][j].low[t]) + c * acc[e][j][t] + (col + t == row && row < rows ? a : 0.0f);
                small_put<ROWS>(m, A_LOW, row, col, v);
            }
        __syncthreads();
    }
    // next = m x; TURNED: a result's rows and columns change places
    template <bool TURNED>
    __device__ __forceinline__ void apply_as(f4 (&next)[R][2 * N], const uint8_t* m, const uint8_t* x) const {
        f4 small[R][2 * N] = {};
#pragma unroll
        for (u32 k0 = 0; k0 < ROWS; k0 += 32) {
            u4v bh[R], bl[R], ch[2 * N], cl[2 * N];
#pragma unroll
            for (int e = 0; e < R; ++e) { bh[e] = small_rows<ROWS>(m, m0 + 16 * e, k0); bl[e] = small_rows<ROWS>(m + A_LOW, m0 + 16 * e, k0); }
#pragma unroll
            for (int j = 0; j < 2 * N; ++j) { ch[j] = small_columns<COLS>(x, xn0 + 16 * j, k0); cl[j] = small_columns<COLS>(x + X_LOW, xn0 + 16 * j, k0); }
            add_halves<R, 2 * N, TURNED>(next, small, bh, bl, ch, cl);
        }
        join_halves<R, 2 * N>(next, small);
    }
    __device__ __forceinline__ void apply(f4 (&next)[R][2 * N], const uint8_t* m, const uint8_t* x, bool turned) const {
        if (turned) apply_as<true>(next, m, x);
        else apply_as<false>(next, m, x);
    }
    __device__ __forceinline__ void keep(const f4 (&next)[R][2 * N], float by, uint8_t* x) const {
#pragma unroll
        for (int e = 0; e < R; ++e)
#pragma unroll
            for (int j = 0; j < 2 * N; ++j) {
                float v[4];
                for (int t = 0; t < 4; ++t) v[t] = next[e][j][t] * by;
                small_put<COLS>(x, X_LOW, m0 + 16 * e + in_group, xn0 + 16 * j + group * 4, v);
            }
    }
    __device__ __forceinline__ void leave(const f4 (&next)[R][2 * N], const UpdateOut& out, u32 matrix, const Shape& s, u32 first) const {
        const u32 rows = s.tall ? s.cols : s.rows, cols = s.tall ? s.rows : s.cols;
#pragma unroll
        for (int e = 0; e < R; ++e)
#pragma unroll
            for (int j = 0; j < 2 * N; ++j) {
                const u32 row = s.tall ? first + xn0 + 16 * j + in_group : m0 + 16 * e + in_group, col = s.tall ? m0 + 16 * e + group * 4 : first + xn0 + 16 * j + group * 4;
                if (row < rows && col < cols) out.put(matrix, 0, row, col, cols, next[e][j], out.get(matrix, row, col, cols));
            }
    }
};

template <class T, int R, int N>
__global__ __launch_bounds__(512) void small_steps(const typename T::elem* g, u64 stride, u64 step, Shape s, float up, SmallSteps k, UpdateOut out) {
    typedef Small<R, N> S;
    __shared__ __attribute__((aligned(16))) uint8_t x[2 * S::X_LOW];
    __shared__ __attribute__((aligned(16))) uint8_t m[2 * S::A_LOW];
    const S small;
    const typename S::template Values<T> values(g + (out.matrix0 + blockIdx.x) * step, stride, s, 0);
    const double sum = block_sum<8>(values.squares());
    values.put(x, (sum == 0.0 ? 0.0 : sum <= DBL_MAX ? 1.0 / sqrt(sum) : NAN) * up);
    for (u32 i = 0; i < k.n; ++i) {
        __syncthreads();
        f4 acc[R][2 * R] = {};
        small.template square<S::COLS>(acc, x, S::X_LOW);
        small.poly(acc, m, s.rows, k.gram[i], k.a[i], k.b[i], k.c[i]);
        const bool last = i + 1 == k.n;
        f4 next[R][2 * N] = {};
        small.apply(next, m, x, last && s.tall);
        if (last) {
            small.leave(next, out, blockIdx.x, s, 0);
        } else {
            __syncthreads();
            small.keep(next, k.next[i], x);
        }
    }
}

// ------------------------------------------------------------------------------------------
// Long ones of at most 128 rows: the same by many blocks, each with some pieces of 128 columns of X.  A step is two launches: blocks multiply their pieces and add up their part of the
// next A from them, as they lie in LDS, and one block a matrix joins the parts and makes a + b A + c A A.  What bounds it is the launches, 5 to 7 us each with a block's few products
// in a row: 40 x 64 x 1536 in 112 us, 153 as products of tiles that go through memory; X's reads and writes where the matrices are many (300 x 64 x 3000 1193 us, 2.3 TB/s).
// ------------------------------------------------------------------------------------------
// 16 bytes a thread between LDS and a piece of a matrix in halves.
template <int ROWS, int WIDTH, bool OUT>
__device__ __forceinline__ void piece(const HalvesAt& of, u64 matrix, u32 col0, uint8_t* lds) {
    constexpr u32 LOW = ROWS * WIDTH * 2;
#pragma unroll
    for (u32 i = 0; i < ROWS * WIDTH / 8 / 512; ++i) {
        const u32 u = threadIdx.x + i * 512, row = u / (WIDTH / 8), col = u % (WIDTH / 8) * 8;
        u4v* const high = (u4v*)(of.p + matrix * of.step + row * of.stride + col0 + col);
        u4v* const low = (u4v*)((_Float16*)high + of.low);
        u4v* const a = (u4v*)(lds + small_at<WIDTH>(row, col));
        u4v* const b = (u4v*)(lds + LOW + small_at<WIDTH>(row, col));
        if (OUT) { *high = *a; *low = *b; }
        else { *a = *high; *b = *low; }
    }
}

// (a thread's values of A's part lie where the same thread of the block that joins them reads 16 bytes beside its neighbours')
template <int R>
__device__ __forceinline__ void thin_part(const f4 (&acc)[R][2 * R], float* part) {
#pragma unroll
    for (int e = 0; e < R; ++e)
#pragma unroll
        for (int j = 0; j < 2 * R; ++j) ((f4*)part)[(e * 2 * R + j) * 512 + threadIdx.x] = acc[e][j];
}

template <class T, int R>
__global__ __launch_bounds__(512) void thin_first(const typename T::elem* g, u64 stride, u64 step, Shape s, u64 matrix0, const double* norms, u32 n_norms, float up, HalvesAt to, float* parts) {
    typedef Small<R, 2> S;
    __shared__ __attribute__((aligned(16))) uint8_t x[2 * S::X_LOW];
    const S small;
    const u64 matrix = matrix0 + blockIdx.z;
    const double q = one_over_norm<8>(norms + matrix * n_norms, n_norms) * up;
    f4 acc[R][2 * R] = {};
    for (u32 col0 = blockIdx.x * 128; col0 < to.stride; col0 += gridDim.x * 128) {
        const typename S::template Values<T> values(g + matrix * step, stride, s, col0);
        __syncthreads();
        values.put(x, q);
        __syncthreads();
        piece<S::ROWS, S::COLS, true>(to, matrix, col0, x);
        small.template square<S::COLS>(acc, x, S::X_LOW);
    }
    thin_part<R>(acc, parts + (matrix * gridDim.x + blockIdx.x) * (S::ROWS * S::ROWS));
}

template <int R>
__global__ __launch_bounds__(512) void thin_poly(const float* parts, u32 n_parts, u32 rows, float gram, float a, float b, float c, u64 matrix0, HalvesAt poly) {
    typedef Small<R, 2> S;
    __shared__ __attribute__((aligned(16))) uint8_t m[2 * S::A_LOW];
    const S small;
    const u64 matrix = matrix0 + blockIdx.x;
    parts += matrix * n_parts * (S::ROWS * S::ROWS);
    f4 acc[R][2 * R] = {};
    for (u32 i = 0; i < n_parts; i += 4)
#pragma unroll
        for (int e = 0; e < R; ++e)
#pragma unroll
            for (int j = 0; j < 2 * R; ++j) {
                const f4* const at = (const f4*)(parts + (u64)i * (S::ROWS * S::ROWS)) + (e * 2 * R + j) * 512 + threadIdx.x;
                f4 v[4];
#pragma unroll
                for (u32 t = 0; t < 4; ++t) v[t] = i + t < n_parts ? at[t * (S::ROWS * S::ROWS / 4)] : (f4)(0.0f);
#pragma unroll
                for (u32 t = 0; t < 4; ++t) acc[e][j] += v[t];
            }
    small.poly(acc, m, rows, gram, a, b, c);
    piece<S::ROWS, S::ROWS, true>(poly, matrix, 0, m);
}

template <int R>
__global__ __launch_bounds__(512) void thin_apply(HalvesAt poly, HalvesAt xs, Shape s, float by, bool last, UpdateOut out, float* parts) {
    typedef Small<R, 2> S;
    __shared__ __attribute__((aligned(16))) uint8_t x[2 * S::X_LOW];
    __shared__ __attribute__((aligned(16))) uint8_t m[2 * S::A_LOW];
    const S small;
    const u64 matrix = out.matrix0 + blockIdx.z;
    piece<S::ROWS, S::ROWS, false>(poly, matrix, 0, m);
    f4 acc[R][2 * R] = {};
    for (u32 col0 = blockIdx.x * 128; col0 < xs.stride; col0 += gridDim.x * 128) {
        __syncthreads();
        piece<S::ROWS, S::COLS, false>(xs, matrix, col0, x);
        __syncthreads();
        f4 next[R][4] = {};
        small.apply(next, m, x, last && s.tall);
        if (last) {
            small.leave(next, out, blockIdx.z, s, col0);
            continue;
        }
        __syncthreads();
        small.keep(next, by, x);
        __syncthreads();
        piece<S::ROWS, S::COLS, true>(xs, matrix, col0, x);
        small.template square<S::COLS>(acc, x, S::X_LOW);
    }
    if (!last) thin_part<R>(acc, parts + (matrix * gridDim.x + blockIdx.x) * (S::ROWS * S::ROWS));
}

// No step: X itself.
__global__ __launch_bounds__(256) void update_plain(HalvesAt x, Shape s, UpdateOut out) {
    const u32 rows = s.tall ? s.cols : s.rows, cols = s.tall ? s.rows : s.cols;
    const u64 units = (cols + 3ull) / 4, n = rows * units, matrix = out.matrix0 + blockIdx.z;
    for (u64 i = (u64)blockIdx.x * 256 + threadIdx.x; i < n; i += (u64)gridDim.x * 256) {
        const u32 m = (u32)(i / units), c = (u32)(i % units) * 4;
        f4 v = {};
        for (u32 e = 0; e < 4; ++e)
            if (c + e < cols) {
                const _Float16* const at = x.p + matrix * x.step + (s.tall ? (c + e) * x.stride + m : m * x.stride + c + e);
                v[e] = value_of(at[0], at[x.low]);
            }
        out.put(blockIdx.z, 0, m, c, cols, v, out.get(blockIdx.z, m, c, cols));
    }
}

// ------------------------------------------------------------------------------------------
// C-ABI
// ------------------------------------------------------------------------------------------
// Where the matrices lie in the workspace, each as high and low halves of padded rows and columns, and the partial norms.
static constexpr bool is_parts(const PartOut&) { return true; }
template <class Out> static constexpr bool is_parts(const Out&) { return false; }

struct Space { u64 rows, cols, norms, x[2], gram, poly, parts, bytes; };

static Space space_of(u64 count, u64 rows, u64 cols) {
    Space s = {};
    u64 at = 0;
    const auto take = [&](u64 bytes) { const u64 here = at; at += round_up(bytes, 256); return here; };
    s.rows = round_up(rows < cols ? rows : cols, 64);
    s.cols = round_up(rows < cols ? cols : rows, s.rows <= 128 ? 128 : 64);        // (long ones of few rows go by pieces of 128)
    s.norms = take(count * norm_blocks(rows * cols) * 8);
    for (int i = 0; i < 2; ++i) s.x[i] = take(count * s.rows * s.cols * 4);
    s.gram = take(count * s.rows * s.rows * 4);
    s.poly = take(count * s.rows * s.rows * 4);
    s.parts = take(parts_bytes(count * s.rows, s.rows));
    s.bytes = at + 256;
    return s;
}

// 64 rows' offsets fit 31 bits; workspaces are held below 2^60 bytes: larger ones do not exist.
#define SIDE_LIMIT (1ull << 24)
static bool out_of_range(u64 count, u64 rows, u64 cols) {
    return count >= COUNT_LIMIT || rows >= SIDE_LIMIT || cols >= SIDE_LIMIT || (double)count * (rows + 64.0) * (cols + 64.0) > 1e16;
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

// ... and |a + b q + c q^2|.
static double poly_bound(const double* k, double most) {
    const auto value = [&](double q) { return fabs(k[0] + q * (k[1] + q * k[2])); };
    const double end = most * most, turn = k[2] != 0.0 ? -k[1] / (2 * k[2]) : 0.0;
    double best = fmax(value(0.0), value(end));
    if (turn > 0 && turn < end) best = fmax(best, value(turn));
    return best;
}
// Bounds are held to this and more (coefficients may be any small ones): powers of two of them, and products of those, stay in fp64's range.
#define BOUND_LEAST 0x1p-300
// The power of two that takes values up to `most` to 2^15 and less: fp16 reaches past it.
static double power_for(double most) { return exp2(floor(15 - log2(fmax(most, BOUND_LEAST) * (1 + 1e-5)))); }

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
        if (bounds[i + 1] < BOUND_LEAST) bounds[i + 1] = BOUND_LEAST;
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
    double* const norms = (double*)(ws + at.norms);
    const u64 values = at.rows * at.cols, square = at.rows * at.rows;
    const auto halves = [&](u64 place, u64 cols) { return HalvesAt{(_Float16*)(ws + place), cols, 2 * at.rows * cols, at.rows * cols}; };
    HalvesAt x = halves(at.x[0], at.cols), next = halves(at.x[1], at.cols);
    const HalvesAt gram = halves(at.gram, at.rows), poly = halves(at.poly, at.rows);
    const bool tall = rows > cols;
    const Shape s = {tall ? cols : rows, tall ? rows : cols, tall};
    const u32 n_parts = norm_blocks((u64)rows * cols);
    const auto each_matrix = [&](auto f) { for (u64 m = 0; m < count; m += 32768) f(m, (u32)(count - m < 32768 ? count - m : 32768)); };
    UpdateOut update = {out_type, scale, base_scale, d_base, base_stride, base_step, d_out, out_stride, out_step, 0};
    // what step i multiplies its products' sums by: from the operands' powers of two to the result's
    SmallSteps by = {};
    by.n = steps;
    for (u32 i = 0; i < steps; ++i) {
        const double* k = h_coefficients ? h_coefficients + 3 * i : USUAL;
        const double x_up = power_for(bounds[i]), gram_up = power_for(bounds[i] * bounds[i]), poly_up = power_for(poly_bound(k, bounds[i])), next_up = power_for(bounds[i + 1]);
        by.gram[i] = (float)(gram_up / (x_up * x_up));
        by.a[i] = (float)(poly_up * k[0]);
        by.b[i] = (float)(poly_up / gram_up * k[1]);
        by.c[i] = (float)(poly_up / (gram_up * gram_up) * k[2]);
        by.next[i] = (float)(next_up / (poly_up * x_up));
        update.scale = (float)(scale / (poly_up * x_up));
    }
    const float up = (float)power_for(bounds[0]);
    if (steps == 0) update.scale = (float)(scale / up);
    if (steps && at.cols <= 128) {
        by_type(g_type, [&](auto tt) {
            typedef decltype(tt) T;
            const auto go = [&](auto kernel) {
                for (u64 m = 0; m < count; m += 1u << 20) {
                    update.matrix0 = m;
                    launch(kernel, dim3((u32)(count - m < (1u << 20) ? count - m : 1u << 20)), 512, st, (const typename T::elem*)d_g, (u64)g_stride, (u64)g_step, s, up, by, update);
                }
            };
            if (at.cols == 64) go(small_steps<T, 1, 1>);
            else if (at.rows == 64) go(small_steps<T, 1, 2>);
            else go(small_steps<T, 2, 2>);
        });
        return launched(call, launch);
    }
    // Long ones of at most 128 rows by thin_first and what follows it, where they are many or not too long (the first of two times, in us): one block a matrix joins A's parts, and few
    // blocks hold a single long one up.  Of 64 rows as many blocks as two fit a CU, 12 x 64 x 1671 78 and 124, 1 x 64 x 5297 87 and 121, 1 x 64 x 1000000 3321 and 2837; of 128 one a CU
    // and 16 parts, 128 x 128 x 2048 565 and 762, 16 x 128 x 4096 244 and 237, 1 x 128 x 512 97 and 110, 1 x 128 x 5297 218 and 150.  A's parts lie where the others' do, a single one where A would.
    const bool few_rows = at.rows == 64;
    const u32 pieces = (u32)(at.cols / 128);
    u32 blocks = (u32)((few_rows ? 512 : 256) / count);
    if (blocks > (few_rows ? PARTS_MOST : 16)) blocks = few_rows ? PARTS_MOST : 16;
    if (blocks > pieces) blocks = pieces;
    if (blocks < 1) blocks = 1;
    const bool thin = steps && at.rows <= 128 && (blocks * count >= 256 || pieces <= (few_rows ? 256 : 4));
    u32 across = 1;
    while (across < 256 && across * 4 < cols) across *= 2;
    each_matrix([&](u64 m, u32 n) {
        by_type(g_type, [&](auto tt) {
            typedef decltype(tt) T;
            typedef const typename T::elem* in;
            launch(norm_parts<T>, dim3(n_parts, 1, n), 256, st, (in)d_g, (u64)g_stride, (u64)g_step, rows, cols, across, m, norms);
            if (thin) return;
            // (a grid has at most 2^16 blocks that way: 64 rows each are more than there are of the shorter side)
            launch(scale_in<T>, dim3((u32)(at.cols / 64), (u32)(at.rows / 64), n), 256, st, (in)d_g, (u64)g_stride, (u64)g_step, s, m, (const double*)norms, n_parts, up, x);
        });
    });
    if (thin) {
        float* const a_parts = (float*)(ws + (blocks == 1 ? at.gram : at.parts));
        const auto go = [&](auto r) {
            constexpr int R = decltype(r)::value;
            each_matrix([&](u64 m, u32 n) {
                by_type(g_type, [&](auto tt) {
                    typedef decltype(tt) T;
                    launch(thin_first<T, R>, dim3(blocks, 1, n), 512, st, (const typename T::elem*)d_g, (u64)g_stride, (u64)g_step, s, m, (const double*)norms, n_parts, up, x, a_parts);
                });
                UpdateOut out = update;
                out.matrix0 = m;
                for (u32 i = 0; i < steps; ++i) {
                    launch(thin_poly<R>, dim3(n), 512, st, (const float*)a_parts, blocks, s.rows, by.gram[i], by.a[i], by.b[i], by.c[i], m, poly);
                    launch(thin_apply<R>, dim3(blocks, 1, n), 512, st, poly, x, s, by.next[i], i + 1 == steps, out, a_parts);
                }
            });
        };
        if (few_rows) go(Int<1>());
        else go(Int<2>());
        return launched(call, launch);
    }
    // R = P Q^T for all matrices, summed over all k of the halves; of a symmetric one the tiles on and above the diagonal, in parts where that is a few of them.
    // The kind of tiles and the number of parts by an estimate of the time: rounds over the 256 CUs, of a fixed time and one for each stage of 64 k, in microseconds as measured; parts
    // are written, read and added up at 5 TB/s.
    const auto product = [&](auto p_by_k, auto q_by_k, auto symmetric, const HalvesAt& P, const HalvesAt& Q, u64 m_rows, u64 m_cols, u64 depth, auto out) {
        constexpr bool PK = decltype(p_by_k)::value, QK = decltype(q_by_k)::value, SYM = decltype(symmetric)::value;
        static const struct { u32 tile, blocks; double fixed, first, more; } K[4] = {{64, 3, 4.0, 0.30, 0.11}, {128, 2, 8.0, 0.76, 0.35}, {192, 1, 14.0, 1.08, 0}, {256, 1, 14.0, 1.60, 0}};
        Product a = {{P.p, P.stride, P.step, P.low}, {Q.p, Q.stride, Q.step, Q.low}, (u32)m_rows, (u32)m_cols, (u32)(3 * depth), 0, (u32)(3 * depth), 1};
        const bool far = !in_reach<F16>(a.P) || !in_reach<F16>(a.Q);                      // (a tile of more rows would be out of reach)
        const u64 stages = a.depth / 64, bytes = count * m_rows * m_cols * 4;
        int best = 0;
        double least = 1e30;
        for (int i = 0; i < (far ? 1 : 4); ++i) {
            if (K[i].tile == 192 && !SYM) continue;
            const double down = ceil(m_rows / (double)K[i].tile), across = ceil(m_cols / (double)K[i].tile), tiles = count * (SYM ? down * (down + 1) / 2 : down * across);
            for (u64 p = 1; p <= (SYM ? PARTS_MOST : 1) && (p == 1 || (p * bytes <= PARTS_BYTES && stages / p >= 4)); ++p) {
                const u64 each = (stages + p - 1) / p;
                if ((stages + each - 1) / each != p) continue;
                const double blocks = tiles * p, rounds = ceil(blocks / (256.0 * K[i].blocks)), held = rounds > 1 ? K[i].blocks : ceil(blocks / 256.0);
                const double t = rounds * (K[i].fixed + each * (K[i].first + (held - 1) * K[i].more)) + (p > 1 ? 4.0 + p * bytes * 2 / 5e6 : 0.0);
                if (t < least) {
                    least = t;
                    best = i;
                    a.parts = (u32)p;
                    a.part = (u32)(each * 64);
                }
            }
        }
        const PartOut parts = {(float*)(ws + at.parts), m_cols, m_rows * m_cols, nullptr, (u32)m_rows, a.parts};
        const auto tiles_of = [&](auto waves, auto to) {
            typedef decltype(waves) W;
            each_tiles<W::BM, W::BN>(a, count, [&](Product p, dim3 grid, u64 m) {
                if constexpr (is_parts(to)) to.p = parts.p + m * a.parts * parts.step;
                else to.matrix0 = m;
                p.P.p = P.p + m * P.step;
                p.Q.p = Q.p + m * Q.step;
                launch(ring_products<F16, PK, QK, false, false, W, false, decltype(to), true, SYM>, grid, 64 * W::ALL, st, p, to);
            }, SYM);
        };
        const auto go = [&](auto waves) {
            if constexpr (SYM) if (a.parts > 1) return tiles_of(waves, parts);
            tiles_of(waves, out);
        };
        if (best == 0) go(Waves<2, 2, 2, 2, 3>());
        else if (best == 1) go(Waves<2, 2, 4, 4, 2>());
        else if (best == 3) go(Waves<2, 4, 8, 4, 2>());
        else if constexpr (SYM) go(Waves<2, 4, 6, 3, 3>());
        if constexpr (SYM)
            if (a.parts > 1)
                each_matrix([&](u64 m, u32 n) {
                    PartOut in = parts;
                    in.p += m * a.parts * parts.step;
                    out.matrix0 = m;
                    each_launch<4>(m_rows, (u32)m_cols, [&](Units s) { launch(join_parts<decltype(out)>, dim3(blocks_of(s.n, 256), 1, n), 256, st, in, s, out); });
                });
    };
    if (steps == 0)
        each_matrix([&](u64 m, u32 n) {
            update.matrix0 = m;
            launch(update_plain, dim3(norm_blocks(values), 1, n), 256, st, x, s, update);
        });
    for (u32 i = 0; i < steps; ++i) {
        product(Int<0>(), Int<0>(), Int<1>(), x, x, at.rows, at.rows, at.cols, GramOut{gram, by.gram[i], 0});
        product(Int<0>(), Int<0>(), Int<1>(), gram, gram, at.rows, at.rows, at.rows, PolyOut{gram, poly, by.a[i], by.b[i], by.c[i], s.rows, 0});
        if (i + 1 < steps) product(Int<0>(), Int<1>(), Int<0>(), poly, x, at.rows, at.cols, at.rows, GramOut{next, by.next[i], 0});
        else if (tall) product(Int<1>(), Int<0>(), Int<0>(), x, poly, s.cols, s.rows, at.rows, update);
        else product(Int<0>(), Int<1>(), Int<0>(), poly, x, s.rows, s.cols, at.rows, update);
        const HalvesAt t = x;
        x = next;
        next = t;
    }
    return launched(call, launch);
}
