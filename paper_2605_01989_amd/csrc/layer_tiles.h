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

// Floats as sums of three bf16 values: the upper half of the bits, rounded, that of what is left, cut off, and the rest, which has eight bits at most.  A product of two such sums is taken as
// the six of its nine products that are above 2^-24 of it, each exact, on units of sixteen times the rate.  With |x| in 1..2 what is left of it is at most 2^-8 and the rest below 2^-16:
// middle by rest, twice, and rest by rest are below 2^-23 of the product, one step of fp32.  Of values that are not finite, or whose upper half is rounded to infinity, it is NaN.  Below
// 2^-110 the rest may have bits below 2^-133, where bf16 ends: `cut` gets them, in its lower half.  (The bits' arithmetic runs at the full rate, conversions do not.)
struct Thirds { u4v high, middle, low; };
__device__ __forceinline__ u32 upper_halves(u32 a, u32 b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }       // of b, of a
__device__ __forceinline__ Thirds thirds_of(u4v a, u4v b, u32& cut) {
    const u32 x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    u32 h[8], m[8], l[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        h[i] = (x[i] + 0x8000u) & 0xFFFF0000u;
        const float r = __builtin_bit_cast(float, x[i]) - __builtin_bit_cast(float, h[i]);
        m[i] = __builtin_bit_cast(u32, r) & 0xFFFF0000u;
        l[i] = __builtin_bit_cast(u32, r - __builtin_bit_cast(float, m[i]));
    }
    const auto pack = [](const u32 (&v)[8]) { return (u4v){upper_halves(v[0], v[1]), upper_halves(v[2], v[3]), upper_halves(v[4], v[5]), upper_halves(v[6], v[7])}; };
    // (assembly that the values go through: the compiler would keep them in registers until it comes to `cut`)
#pragma unroll
    for (int i = 0; i < 8; i += 2) asm("v_or3_b32 %0, %1, %2, %0" : "+v"(cut), "+v"(l[i]), "+v"(l[i + 1]));
    return {pack(h), pack(m), pack(l)};
}
// For several b, whose sums then need not wait for each other.
template <int N>
__device__ __forceinline__ void mfma_thirds(const Thirds& a, const Thirds (&b)[N], f4* const (&c)[N]) {
    const auto round = [&](u4v x, auto y) {
#pragma unroll
        for (int i = 0; i < N; ++i) *c[i] = mfma<BF16>(x, y(b[i]), *c[i]);
    };
    const auto high = [](const Thirds& t) { return t.high; };
    const auto middle = [](const Thirds& t) { return t.middle; };
    round(a.low, high);
    round(a.high, [](const Thirds& t) { return t.low; });
    round(a.middle, middle);
    round(a.middle, high);
    round(a.high, middle);
    round(a.high, high);
}

// One operand of a batch of products: element (row, k) at row * stride + k, or at k * stride + row where it lies by k.  An operand in halves is two such matrices of
// fp16, `low` elements apart, the second times 2^-11: 22 significant bits, also where a half without that factor would be below fp16's normal numbers.  A product of two of those is three of
// the halves', low by high, high by low and high by high, one behind the other in one sum over 3 k, which is multiplied by 2^-11 before the third (the small ones first: they are rounded as
// what they are); what is left out is below the halves' own rounding.
#define LOW_UP 2048.0f
#define LOW_DOWN (1.0f / LOW_UP)
struct Operand { const void* p; u64 stride, step, low; };

// What a launch computes: rows x cols results of sums over `depth` k, of which block z takes part z % parts of matrix z / parts.
struct Product {
    Operand P, Q;
    u32 rows, cols, depth, tile_cols, part, parts;   // part: k of one part, a multiple of 128 bytes' (a stage's); tile_cols: tiles of a row of tiles
    u32 tile_rows, odd_rows;                         // odd_rows: see PAIRS
    u64 tiles, tile0;                                // of the whole result; first one of this launch
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

// Four waves, two by two, each a quarter of a BM x BN tile: operands of any place and stride.  SUMS: of the first column of tiles, also P's own sums over k.  `out` gets the
// results, four columns of a row at a time, and what its `get` has found in memory for them; `sums` gets a row's sum.  For operands whose rows are so far apart that a tile's
// offsets pass 31 bits.  Bound by the loads' way through registers: 2048 x 2048 x 2048 of bf16, rows 2^21 elements apart, 39 us (444 TFLOP/s), 31 by ring_products on near ones.
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
            if (n < a.cols) out.put(matrix, part, m, n, a.cols, acc[i][j], out.get(matrix, m, n, a.cols));
        }
    }
}

// ------------------------------------------------------------------------------------------
// The same products with operands copied from memory to LDS past the registers.
//
// LDS holds RING stages of 128 bytes of k (64 16-bit values, 32 floats): whole lines of memory.  A stage is multiplied in two halves, and while one half's
// fragments are multiplied the next half's are read from LDS.  Behind the barrier between the halves nothing of the stage is read any more: a later stage
// is copied into its place, and has two halves' time to arrive.
// A copy writes 64 lanes' 16 bytes one after the other, so an order in LDS other than memory's is made by what each lane asks for:
//   by rows  a row is 128 bytes, chunk c of row r at place c ^ (r & 7): eight rows' chunks, which eight lanes read at once, lie in all banks.
//   by k     a row is one k of BT rows, in granules of 16 rows; granule g of k lies at g ^ turn(k), so that the rows of k that one transposing read of four k
//            takes lie in different banks.  16-bit values are transposed on the way out (ds_read_b64_tr_b16: of 16 lanes with
//            four values each, lane i gets value i % 4 of lanes i / 4, i / 4 + 4, ...), floats are read one by one.
// Bound by the matrix instructions and by LDS' reads beside them (the instructions at work 65 % of the time in the largest products), small products by the rounds of tiles.  The largest
// tile, 256 x 256 of eight waves with 128 x 64 results each, reads 96 KiB of LDS for 32 k, four of 128 x 128 128 KiB; four waves' results do not fit the registers.  8192 x 8192 x 8192 of
// bf16: 815 us (1.35 PFLOP/s) by rows and rows, 782 by rows and k, 802 by k and k into floats; 4096 x 4096 x 4096 105, 106, 107; the library's 694, 808, 908 and 109, 116, 130.
// ------------------------------------------------------------------------------------------
#define STAGE_BYTES 128

typedef u32 rsrc_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ u32 uniform(u32 v) { return (u32)__builtin_amdgcn_readfirstlane((int)v); }
#define PAST_ALL 0x80000000u                     // an offset that no buffer here reaches: a copy of it writes zeros

// 64 lanes' 16 bytes at `offset` of a buffer to 1024 bytes of LDS at `to`.  No register is written, so nothing can be overwritten by it, and the compiler waits
// for it nowhere: by a builtin it would before each read of LDS.  m0 is nobody's else in these kernels.  Nor does the compiler look into these lines for the wait states
// that a copy needs behind a write of m0, one, and behind a vector instruction's write of a register of `from`, five, of which the write of m0 is one.
__device__ __forceinline__ void copy_to_lds(rsrc_t from, u32 offset, u32 to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(offset), "s"(from));
}
template <int N> __device__ __forceinline__ void arrived_and_barrier() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

__device__ __forceinline__ u32 lds_address(const void* p) { return (u32)(uintptr_t)(const __attribute__((address_space(3))) uint8_t*)p; }

// An operand's way to LDS: BT rows and 128 bytes of k a stage, shared by WAVES waves.  STAGED: through registers, for rows of 16-bit values that do not begin at multiples of four bytes.
template <class T, int BT, bool BY_K, bool STAGED, int WAVES, int HALVES = 0>
struct Feed {
    typedef typename T::elem elem;
    static constexpr u32 E = 16 / sizeof(elem), KS = STAGE_BYTES / sizeof(elem);  // elements of a chunk, k of a stage
    static constexpr u32 BYTES = BT * STAGE_BYTES, N = BYTES / (1024 * WAVES);    // of a stage; copies of a wave
    static constexpr u32 ROW = BY_K ? BT * sizeof(elem) : STAGE_BYTES, CG = sizeof(elem);  // bytes of a row in LDS; chunks of 16 values
    static constexpr u32 COPIES = STAGED ? 0 : N, KD = BY_K ? 1024 / ROW : 0;
    typedef Vec<T, E> V;

    const elem* base;            // of the block's first row, at the stage that is copied next
    u64 left;                    // bytes from there to the operand's end
    u64 stride;
    u32 k, depth;                // of that stage; end of the sum
    u32 rows;                    // of the operand from the block's first
    u32 offset[N], kk;           // a lane's chunks: from the base; the first one's first k in a stage, KD before the next one's
    u32 r[BY_K && STAGED ? N : 1];                       // their rows
    u32 wave;
    u4v v[STAGED ? N : 1];
    // HALVES 1, 2: as the first, the second operand of a product of halves, all of whose matrices end with whole stages
    const elem* whole;
    u64 low;
    u32 third, k_in, product;    // k of one product of halves, where in it, and which
    __device__ __forceinline__ void of_halves(const elem* p, u64 low_, u32 row0, u32 k0, u32 depth_) {
        whole = p + (BY_K ? row0 : (u64)row0 * stride);
        low = low_;
        third = depth_ / 3;
        product = k0 / third;
        k_in = k0 - product * third;
        left = ~0ull >> 1;
        place();
    }
    __device__ __forceinline__ void place() { base = whole + (product == (HALVES == 1 ? 0 : 1) ? low : 0) + (BY_K ? (u64)k_in * stride : k_in); }

    static __device__ __forceinline__ u32 turn(u32 k) {
        const u32 t = sizeof(elem) == 2 ? (k & 3) | (k >> 3 & 1) << 2 : k >> 2 & 3;
        return t & (BT / 16 - 1);
    }
    __device__ __forceinline__ Feed(const elem* p, u64 stride_, u32 row0, u32 rows_, u32 k0, u32 depth_) : stride(stride_), k(k0), depth(depth_), rows(rows_ - row0) {
        base = p + (BY_K ? (u64)k0 * stride + row0 : (u64)row0 * stride + k0);
        left = (BY_K ? (u64)(depth - 1 - k0) * stride + rows : (u64)(rows - 1) * stride + depth - k0) * sizeof(elem);
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const u32 lane = threadIdx.x & 63;
#pragma unroll
        for (u32 i = 0; i < N; ++i) {
            const u32 at = (wave * N + i) * 1024 + lane * 16, line = at / ROW, place = at % ROW / 16;
            if (BY_K) {
                const u32 chunk = (place / CG ^ turn(line)) * CG + place % CG, row = chunk * E;
                if (i == 0) kk = line;
                if (STAGED) r[i] = row;
                offset[i] = (u32)(line * stride + (row < rows ? row : 0)) * sizeof(elem);      // (a chunk of rows past the end: any)
            } else {
                const u32 chunk = place ^ (line & 7), row = line < rows ? line : rows - 1;
                if (i == 0) kk = chunk * E;
                offset[i] = (u32)(row * stride + chunk * E) * sizeof(elem);
            }
        }
    }
    __device__ __forceinline__ void next() {
        const u64 by = BY_K ? KS * stride : KS;
        if (HALVES) {
            k += KS;
            k_in += KS;
            base += by;
            if (k_in != third) return;
            k_in = 0;
            ++product;
            return place();
        }
        base += by;
        left -= by * sizeof(elem);
        k += KS;
    }
    // The stage's copy number i of this wave, to LDS at `to`; k past the end, and before `begin`, as zeros.
    __device__ __forceinline__ void copy(u32 i, u32 to, u32 begin = 0) const {
        const u64 at = (u64)base;
        const u32 bytes = left < PAST_ALL - 4 ? ((u32)left + 3) & ~3u : PAST_ALL;        // (a chunk that goes past the operand's end brings zeros from there)
        const u32 rest = k < depth ? depth - k : 0;
        // (the same in all lanes: the compiler does not see it through the turns of halves)
        const rsrc_t from = {uniform((u32)at), uniform((u32)(at >> 32)), uniform(bytes), 0x00020000u};
        const u32 k_here = kk + i * KD;
        copy_to_lds(from, k_here < rest && (begin == 0 || k + k_here >= begin) ? offset[i] : PAST_ALL, to + (wave * N + i) * 1024);
    }
    // Through registers: asked for, and put down later.
    __device__ __forceinline__ void ask(u32 i) {
        v[i] = (u4v)(0u);
        if (k >= depth) return;
        const u32 n = depth - k;
        const elem* const at = base + offset[i] / sizeof(elem);
        if (BY_K) {
            if (kk + i * KD < n && r[i] < rows) v[i] = __builtin_bit_cast(u4v, r[i] + E <= rows ? V::load(at) : V::some(at, rows - r[i]));
        } else if (kk < n) {
            v[i] = __builtin_bit_cast(u4v, kk + E <= n ? V::load(at) : V::some(at, n - kk));
        }
    }
    __device__ __forceinline__ void put(u32 i, uint8_t* stage) const { *(u4v*)(stage + (wave * N + i) * 1024 + (threadIdx.x & 63) * 16) = v[i]; }
    // The chunks that hold the end of the sum, n k into a stage, in rows whose k do not end with it: zeros behind.
    static __device__ __forceinline__ void trim(uint8_t* stage, u32 n) {
        if (BY_K || STAGED) return;
        for (u32 row = threadIdx.x; row < BT; row += 64 * WAVES)
            for (u32 e = n % E; e < E; ++e) *(elem*)(stage + row * STAGE_BYTES + ((n / E ^ (row & 7)) << 4) + e * sizeof(elem)) = (elem)0.0f;
    }
};

// A wave's fragments of an operand: 16 rows each, from row w0 of the tile.
template <class T, int BT, bool BY_K>
struct Reader {
    typedef typename T::elem elem;
    typedef Feed<T, BT, BY_K, false, 1> F;
    u32 base;                    // of fragment 0
    __device__ __forceinline__ explicit Reader(u32 w) {
        const u32 lane = threadIdx.x & 63, group = lane >> 4, in = lane & 15;
        if (!BY_K) base = (w + in) * STAGE_BYTES + ((group ^ (in & 7)) << 4);
        else if (sizeof(elem) == 2) base = (8 * group + (in >> 2)) * F::ROW + (in & 3) * 8 + ((w / 16 ^ F::turn(8 * group + (in >> 2))) << 5);
        else base = 4 * group * F::ROW + in * 4 + ((w / 16 ^ F::turn(4 * group)) << 6);
    }
    // Fragment i of half `half` of the stage at `stage`, a multiple of 1024.  By k, a wave's first granule is a multiple of the number of its fragments (a power of
    // two), so that (first + i) ^ turn is first ^ turn ^ i.
    __device__ __forceinline__ u4v get(const uint8_t* ring, u32 stage, u32 half, u32 i) const {
        if (!BY_K) return *(const u4v*)(ring + ((stage + base) ^ (half << 6)) + i * 16 * STAGE_BYTES);
        const uint8_t* const at = ring + ((stage + base) ^ (i << (sizeof(elem) == 2 ? 5 : 6))) + half * (F::KS / 2) * F::ROW;
        if (sizeof(elem) == 2) {
            typedef short s4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s4* lds;
            const u2v a = __builtin_bit_cast(u2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(at))), b = __builtin_bit_cast(u2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(at + 4 * F::ROW)));
            return (u4v){a.x, a.y, b.x, b.y};
        }
        u4v v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = *(const u32*)(at + j * F::ROW);
        return v;
    }
};

// This block's number among the launch's tiles of all z.  Blocks go to the eight dies in turn; each die gets tiles, and matrices or parts of k, that lie together, so that its L2 holds
// what its blocks read at the same time.
__device__ __forceinline__ u32 block_by_die() {
    const u32 n = gridDim.x * gridDim.z, b = blockIdx.z * gridDim.x + blockIdx.x, each = n / 8, more = n % 8, die = b % 8;        // (below 2^31: each_tiles)
    return die * each + (die < more ? die : more) + b / 8;
}
// Tiles go in bands of eight rows of tiles, down and then across.
__device__ __forceinline__ void tile_of(u64 id, u32 tile_rows, u32 tile_cols, u32& m, u32& c) {
    u32 band, in_band;
    if (id >> 32 || tile_cols >> 28) {
        band = (u32)(id / (8ull * tile_cols));
        in_band = (u32)(id % (8ull * tile_cols));
    } else {
        band = (u32)id / (8 * tile_cols);
        in_band = (u32)id % (8 * tile_cols);
    }
    const u32 first = band * 8, high = tile_rows - first < 8 ? tile_rows - first : 8;
    m = first + in_band % high;
    c = in_band / high;
}

// ... and of a symmetric result, n tiles high and wide, those on and above the diagonal, n (n + 1) / 2.
__device__ __forceinline__ void upper_tile_of(u64 id, u32 n, u32& m, u32& c) {
    u32 left = (u32)id, row = 0;
    while (left >= n - row) left -= n - row++;
    m = row;
    c = row + left;
}

// Four rows' results to an Out: together, if it takes them so.
template <class Out, class Met>
__device__ __forceinline__ auto put_all(const Out& out, u32 matrix, u32 part, u32 m, u32 apart, u32 n, u32 cols, u32 on, const f4 (&v)[4], const Met (&met)[4]) -> decltype(out.put_rows(0, 0, 0, 0, 0, 0, 0, v, met)) {
    if (on) out.put_rows(matrix, part, m, apart, n, cols, on, v, met);
}
template <class Out, class... Met>
__device__ __forceinline__ void put_all(const Out& out, u32 matrix, u32 part, u32 m, u32 apart, u32 n, u32 cols, u32 on, const f4 (&v)[4], const Met (&... met)[4]) {
#pragma unroll
    for (u32 e = 0; e < 4; ++e)
        if (on >> e & 1) out.put(matrix, part, m + e * apart, n, cols, v[e], met[e]...);
}

// PAIRS: P has rows of 16-bit values an odd number of elements apart, so that no more than every other one begins at a multiple of four bytes, and Q lies by k.  The
// others do so one element earlier.  Even and odd rows are two matrices, each with rows at multiples of four bytes that can be copied; of the shifted one k is one more
// than the sum's, its first value, an element of another row, is set to zero, and Q's rows are taken one earlier: the parts have to cover that one as well.
// WR x WC waves, each 16 NM x 16 NN of the tile.
template <int WR_, int WC_, int NM_, int NN_, int RING_> struct Waves { static constexpr int WR = WR_, WC = WC_, NM = NM_, NN = NN_, RING = RING_, BM = 16 * NM * WR, BN = 16 * NN * WC, ALL = WR * WC; };

template <class T, bool P_BY_K, bool Q_BY_K, bool P_STAGED, bool Q_STAGED, class W, bool SUMS, class Out, bool HALVES = false, bool SYMMETRIC = false, bool PAIRS = false>
__global__ __launch_bounds__(64 * W::ALL, 2) void ring_products(Product a, Out out) {
    typedef typename T::elem elem;
    constexpr int BM = W::BM, BN = W::BN, NM = W::NM, NN = W::NN, RING = W::RING;
    typedef Feed<T, BM, P_BY_K, P_STAGED, W::ALL, HALVES ? 1 : 0> FP;
    typedef Feed<T, BN, Q_BY_K, Q_STAGED, W::ALL, HALVES ? 2 : 0> FQ;
    constexpr u32 KS = FP::KS, STAGE = FP::BYTES + FQ::BYTES, COPIES = FP::COPIES + FQ::COPIES;
    __shared__ __attribute__((aligned(1024))) uint8_t ring[RING * STAGE];
    u32 tm, tn;
    const u32 id = block_by_die();
    const u32 z = gridDim.z > 1 ? id / gridDim.x : 0, tile = gridDim.z > 1 ? id % gridDim.x : id;
    if (SYMMETRIC) upper_tile_of(a.tile0 + tile, a.tile_rows, tm, tn);
    else tile_of(a.tile0 + tile, a.tile_rows, a.tile_cols, tm, tn);
    const u32 m0 = tm * BM, n0 = tn * BN;
    const u32 matrix = a.parts > 1 ? z / a.parts : z, part = a.parts > 1 ? z % a.parts : 0;
    const u64 parity = PAIRS ? uniform(matrix) : 0;
    const u32 shift = PAIRS ? ((u32)((uintptr_t)a.P.p >> 1) + (u32)(parity * a.P.stride)) & 1 : 0;
    const u32 rows = PAIRS && parity ? a.odd_rows : a.rows, depth = a.depth + shift;
    if (PAIRS && m0 >= rows) return;
    const u32 lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = lane >> 4, in_group = lane & 15;
    const u32 wm = wave / W::WC * (16 * NM), wn = wave % W::WC * (16 * NN);
    const u32 k_first = part * a.part, k_end = depth - k_first > a.part ? k_first + a.part : depth;
    const u32 stages = (k_end - k_first + KS - 1) / KS;
    const bool summing = SUMS && __builtin_amdgcn_readfirstlane(n0 == 0 && wn == 0);
    f4 acc[NM][NN] = {}, sum[SUMS ? NM : 1] = {};
    FP fp((const elem*)a.P.p + (PAIRS ? parity * a.P.stride - shift : matrix * a.P.step), PAIRS ? 2 * a.P.stride : a.P.stride, m0, rows, k_first, k_end);
    FQ fq((const elem*)a.Q.p + (PAIRS ? 0 - shift * a.Q.stride : matrix * a.Q.step), a.Q.stride, n0, a.cols, k_first, k_end);
    if (HALVES) {
        fp.of_halves((const elem*)a.P.p + matrix * a.P.step, a.P.low, m0, k_first, a.depth);
        fq.of_halves((const elem*)a.Q.p + matrix * a.Q.step, a.Q.low, n0, k_first, a.depth);
    }
    const Reader<T, BM, P_BY_K> rp(wm);
    const Reader<T, BN, Q_BY_K> rq(wn);
    const u32 ring_at = __builtin_amdgcn_readfirstlane(lds_address(ring));
    const auto copy = [&](u32 e, u32 slot) {
        if (e < FP::COPIES) fp.copy(e, ring_at + slot * STAGE);
        else fq.copy(e - FP::COPIES, ring_at + slot * STAGE + FP::BYTES, PAIRS ? shift : 0);
    };
    const auto ask = [&] {
        if (P_STAGED)
#pragma unroll
            for (u32 i = 0; i < FP::N; ++i) fp.ask(i);
        if (Q_STAGED)
#pragma unroll
            for (u32 i = 0; i < FQ::N; ++i) fq.ask(i);
        if (P_STAGED) fp.next();
        if (Q_STAGED) fq.next();
    };
    const auto put = [&](u32 slot) {
        if (P_STAGED)
#pragma unroll
            for (u32 i = 0; i < FP::N; ++i) fp.put(i, ring + slot * STAGE);
        if (Q_STAGED)
#pragma unroll
            for (u32 i = 0; i < FQ::N; ++i) fq.put(i, ring + slot * STAGE + FP::BYTES);
    };
    const auto next_copied = [&] { if (!P_STAGED) fp.next(); if (!Q_STAGED) fq.next(); };
    const u32 end = (k_end - k_first) % KS;        // of the last stage, where it is no whole one
    const auto trim = [&](u32 slot) {
        if (end % (16 / sizeof(elem)) == 0 || (P_BY_K && Q_BY_K)) return;
        arrived_and_barrier<0>();
        fp.trim(ring + slot * STAGE, end);
        fq.trim(ring + slot * STAGE + FP::BYTES, end);
    };
    // Floats in thirds: a stage is one step of 32 k, of which a lane holds chunks `group` and 4 + group.  Bound by the making of the thirds, seven instructions a value and wave.  A tile is
    // made again of floats where a result is not finite or an operand of its own results is no sum of three: 4096 x 4096 x 4096: 738 us (186 TFLOP/s), 1.5 % of it for the looking; 1770 where all are
    // made again, of floats alone 1050, by the library 920.
    constexpr bool THIRDS = sizeof(elem) == 4 && NM * NN == 16;
    if constexpr (THIRDS) {
        const auto all = [&](auto plain) {
            constexpr bool PLAIN = decltype(plain)::value;
            FP p = fp;
            FQ q = fq;
            u32 cut_p[NM] = {}, cut_q[NN] = {};
            const auto copy_all = [&](u32 to) {
#pragma unroll
                for (u32 e = 0; e < FP::COPIES; ++e) p.copy(e, ring_at + to * STAGE);
#pragma unroll
                for (u32 e = 0; e < FQ::COPIES; ++e) q.copy(e, ring_at + to * STAGE + FP::BYTES);
                p.next();
                q.next();
            };
            for (u32 i = 0; i < RING; ++i) copy_all(i);
            u32 slot = 0;
            for (u32 s = 0; s < stages; ++s) {
                if (s + 1 == stages) trim(slot);
                arrived_and_barrier<(RING - 1) * COPIES>();
                const u32 at = slot * STAGE;
                u4v b[NM][2];
                Thirds t[NM];
#pragma unroll
                for (int i = 0; i < NM; ++i) {
                    b[i][0] = rp.get(ring, at, 0, i);
                    b[i][1] = rp.get(ring, at, 1, i);
                    if (!PLAIN) t[i] = thirds_of(b[i][0], b[i][1], cut_p[i]);
                }
                u4v c[NN][2];
#pragma unroll
                for (int j = 0; j < NN; ++j) {
                    c[j][0] = rq.get(ring, at + FP::BYTES, 0, j);
                    c[j][1] = rq.get(ring, at + FP::BYTES, 1, j);
                }
                Thirds u = {};
                if (!PLAIN) u = thirds_of(c[0][0], c[0][1], cut_q[0]);
#pragma unroll
                for (int j = 0; j < NN; ++j) {
                    if (PLAIN) {
#pragma unroll
                        for (int i = 0; i < NM; ++i) acc[i][j] = mfma<F32>(c[j][1], b[i][1], mfma<F32>(c[j][0], b[i][0], acc[i][j]));
                    } else {
                        // the next thirds are made while these are multiplied
                        Thirds next = {};
                        if (j + 1 < NN) next = thirds_of(c[j + 1 < NN ? j + 1 : j][0], c[j + 1 < NN ? j + 1 : j][1], cut_q[j + 1 < NN ? j + 1 : j]);
                        f4* const to[4] = {&acc[0][j], &acc[1][j], &acc[2][j], &acc[3][j]};
                        mfma_thirds<4>(u, t, to);
                        u = next;
                    }
                }
                if (SUMS && summing) {
                    asm volatile("");
#pragma unroll
                    for (int i = 0; i < NM; ++i)
#pragma unroll
                        for (int h = 0; h < 2; ++h) sum[i] = mfma<F32>(ones<F32>(), b[i][h], sum[i]);
                }
                arrived_and_barrier<(RING - 1) * COPIES>();
                copy_all(slot);
                slot = slot + 1 == RING ? 0 : slot + 1;
            }
            // (rows and columns past the ends are anything)
            u32 cut = 0;
#pragma unroll
            for (int i = 0; i < NM; ++i) cut |= m0 + wm + 16 * i + in_group < rows ? cut_p[i] : 0;
#pragma unroll
            for (int j = 0; j < NN; ++j) cut |= n0 + wn + 16 * j + in_group < a.cols ? cut_q[j] : 0;
            return (cut & 0xFFFFu) == 0;
        };
        if (stages) {
            bool good = all(Int<0>());
#pragma unroll
            for (int i = 0; i < NM; ++i)
#pragma unroll
                for (int j = 0; j < NN; ++j)
                    for (int e = 0; e < 4; ++e) good &= fabsf(acc[i][j][e]) <= FLT_MAX || m0 + wm + 16 * i + in_group >= rows || n0 + wn + 16 * j + group * 4 + e >= a.cols;
            arrived_and_barrier<0>();
            if (__syncthreads_or(!good)) {
#pragma unroll
                for (int i = 0; i < NM; ++i)
#pragma unroll
                    for (int j = 0; j < NN; ++j) acc[i][j] = (f4)(0.0f);
                for (f4& of : sum) of = (f4)(0.0f);
                all(Int<1>());
            }
        }
    } else {
        u4v b[2][NM], c[NN];
        if (stages) {
            for (u32 i = 0; i < RING; ++i) {
#pragma unroll
                for (u32 e = 0; e < COPIES; ++e) copy(e, i);
                next_copied();
            }
            for (u32 i = 0; i < 2; ++i) {
                ask();
                put(i);
            }
            ask();
            if (stages == 1) trim(0);
            if (PAIRS && shift && k_first == 0) {
                arrived_and_barrier<0>();
                for (u32 row = threadIdx.x; row < BM; row += 64 * W::ALL) *(elem*)(ring + row * STAGE_BYTES + ((row & 7) << 4)) = (elem)0.0f;
            }
            arrived_and_barrier<(RING - 1) * COPIES>();
#pragma unroll
            for (int i = 0; i < NM; ++i) b[0][i] = rp.get(ring, 0, 0, i);
#pragma unroll
            for (int j = 0; j < NN; ++j) c[j] = rq.get(ring, FP::BYTES, 0, j);
        }
        // Multiplies one half's fragments; between rows of matrix instructions, which take longer, the next half's are read and, COPYING, a stage is copied.
        const auto half = [&](auto copying, const u4v (&b)[NM], u4v (&b1)[NM], u32 slot1, u32 half1, u32 to) {
            constexpr int EACH = (COPIES + NN - 1) / NN;
#pragma unroll
            for (int j = 0; j < NN; ++j) {
#pragma unroll
                for (int i = j * NM / NN; i < (j + 1) * NM / NN; ++i) b1[i] = rp.get(ring, slot1 * STAGE, half1, i);
                if (decltype(copying)::value)
#pragma unroll
                    for (u32 e = j * EACH; e < (j + 1) * EACH && e < COPIES; ++e) copy(e, to);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < NM; ++i) acc[i][j] = mfma<T>(c[j], b[i], acc[i][j]);
                __builtin_amdgcn_sched_barrier(0);
                c[j] = rq.get(ring, slot1 * STAGE + FP::BYTES, half1, j);
            }
            // sums over k: products with ones, each fragment's by itself (what one row holds must not meet another's, be it times zero)
            if (SUMS && summing) {
                asm volatile("");                      // (or the compiler computes them everywhere and chooses)
#pragma unroll
                for (int i = 0; i < NM; ++i) sum[i] = mfma<T>(ones<T>(), b[i], sum[i]);
            }
        };
        // (of halves: the stages that hold low ones)
        const u32 two = 2 * (a.depth / 3), low_stages = !HALVES || two <= k_first ? 0 : (two - k_first) / KS < stages ? (two - k_first) / KS : stages;
        const auto lower = [&] {
#pragma unroll
            for (int i = 0; i < NM; ++i)
#pragma unroll
                for (int j = 0; j < NN; ++j) acc[i][j] *= LOW_DOWN;
        };
        u32 slot = 0;
        for (u32 s = 0; s < stages; ++s) {
            if (HALVES && s == low_stages) lower();
            const u32 then = slot + 1 == RING ? 0 : slot + 1;
            half(Int<0>(), b[0], b[1], slot, 1, 0);
            if (s + 2 == stages) trim(then);
            arrived_and_barrier<(RING - 2) * COPIES>();
            put((s + 2) % RING);
            ask();
            half(Int<1>(), b[1], b[0], then, 0, slot);
            next_copied();
            slot = then;
        }
        if (HALVES && low_stages == stages) lower();
    }
    // the result's tile through LDS, some of a wave's rows at a time: rows leave whole, and what is done with them stands here once
    arrived_and_barrier<0>();
    constexpr u32 WIDTH = 16 * NN, LINE = WIDTH * 4 + 16;                            // (16 bytes more: the rows of a lane's group in different banks)
    uint8_t* const mine = ring + wave * (RING * STAGE / W::ALL);
    constexpr int AT_ONCE = NM * 16 * LINE <= RING * STAGE / W::ALL ? NM : NM / 2 * 16 * LINE <= RING * STAGE / W::ALL ? NM / 2 : NM / 4;
#pragma nounroll
    for (int turn = 0; turn < NM / AT_ONCE; ++turn) {
#pragma unroll
        for (int t = 0; t < NM / AT_ONCE; ++t)
            if (t == turn)
#pragma unroll
                for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
                    for (int j = 0; j < NN; ++j) *(f4*)(mine + (i * 16 + in_group) * LINE + (j * 16 + group * 4) * 4) = acc[t * AT_ONCE + i][j];
        const auto to_row = [&](u32 m) { return PAIRS ? 2 * m + (u32)parity : m; };
        // four at a time, so that what they meet in memory is asked for together.  TURNED: a result's columns as rows, of a symmetric one below the diagonal
        const auto leave = [&](auto turned) {
            constexpr bool TURNED = decltype(turned)::value;
            constexpr u32 HIGH = TURNED ? WIDTH : AT_ONCE * 16, QUADS = (TURNED ? AT_ONCE * 16 : WIDTH) / 4, LINES = 64 / QUADS;
            const u32 q = lane % QUADS * 4, rows0 = m0 + wm + turn * AT_ONCE * 16, n = TURNED ? rows0 + q : n0 + wn + q, row0 = TURNED ? n0 + wn : rows0;
            if (lane >= LINES * QUADS) return;
#pragma nounroll
            for (u32 line = lane / QUADS; line < HIGH; line += 4 * LINES) {
                decltype(out.get(0, 0, 0, 0)) met[4];
#pragma unroll
                for (u32 e = 0; e < 4; ++e)
                    if (line + e * LINES < HIGH && row0 + line + e * LINES < rows && n < a.cols) met[e] = out.get(PAIRS ? 0 : matrix, to_row(row0 + line + e * LINES), n, a.cols);
                f4 v[4];
                u32 on = 0;
#pragma unroll
                for (u32 e = 0; e < 4; ++e) {
                    if (line + e * LINES >= HIGH) continue;
                    if (TURNED)
                        for (u32 t = 0; t < 4; ++t) v[e][t] = *(const float*)(mine + (q + t) * LINE + (line + e * LINES) * 4);
                    else v[e] = *(const f4*)(mine + (line + e * LINES) * LINE + q * 4);
                    if (row0 + line + e * LINES < rows && n < a.cols) on |= 1u << e;
                }
                put_all(out, PAIRS ? 0 : matrix, part, to_row(row0 + line), PAIRS ? 2 * LINES : LINES, n, a.cols, on, v, met);
            }
        };
        leave(Int<0>());
        if (SYMMETRIC && tm != tn) leave(Int<1>());
    }
    if (SUMS && summing)
#pragma unroll
        for (int i = 0; i < NM; ++i)
            if (group == 0 && m0 + wm + i * 16 + in_group < a.rows) out.sums(matrix, part, m0 + wm + i * 16 + in_group, sum[i][0]);
}

// ------------------------------------------------------------------------------------------
// At most 16 rows (tokens that are decoded): the weights are read once, from memory straight into the matrix instructions' registers.  A block makes 16 columns of all rows; its
// waves share k, 128 bytes of it at a time, and add their sums up in LDS.  Bound by the reading of Q; P comes from the caches.  Of bf16 weights that are not in the caches 16384 x 4096 for
// one row 27 us (4.9 TB/s), for four 29; 4096 x 1024 for one 4.6, where the launch counts, 7.3 from call to call.
// ------------------------------------------------------------------------------------------
#define FEW_WAVES 16
template <class T, class Out>
__global__ __launch_bounds__(64 * FEW_WAVES) void few_products(Product a, Out out) {
    typedef typename T::elem elem;
    constexpr u32 E = 16 / sizeof(elem), KS = 128 / sizeof(elem);
    typedef Vec<T, E> V;
    __shared__ f4 sums[FEW_WAVES][64];
    const u32 n0 = (u32)(a.tile0 + blockIdx.x) * 16, part = blockIdx.z;
    const u32 lane = threadIdx.x & 63, wave = threadIdx.x >> 6, group = lane >> 4, in_group = lane & 15;
    const u32 k_first = part * a.part, k_end = a.depth - k_first > a.part ? k_first + a.part : a.depth;
    const elem* const p = (const elem*)a.P.p + (in_group < a.rows ? in_group : a.rows - 1) * a.P.stride;
    const elem* const q = (const elem*)a.Q.p + (n0 + in_group < a.cols ? n0 + in_group : a.cols - 1) * a.Q.stride;
    f4 acc = {};
    // A lane's chunks of 128 bytes of k: number `group` of the first and of the second half.
    const auto step = [&](u32 k, auto whole) {
        u4v b[2], c[2];
        const auto get = [&](const elem* row, u32 at) {
            if (decltype(whole)::value || at + E <= k_end) return __builtin_bit_cast(u4v, V::load(row + at));
            return at < k_end ? __builtin_bit_cast(u4v, V::some(row + at, k_end - at)) : (u4v)(0u);
        };
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            c[h] = get(q, k + h * (KS / 2) + group * E);
            b[h] = get(p, k + h * (KS / 2) + group * E);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) acc = mfma<T>(c[h], b[h], acc);
    };
    u32 k = k_first + wave * KS;
#pragma unroll 4
    for (; k + KS <= k_end; k += FEW_WAVES * KS) step(k, Int<1>());
    if (k < k_end) step(k, Int<0>());
    sums[wave][lane] = acc;
    __syncthreads();
    const u32 m = in_group, n = n0 + group * 4;
    if (wave != 0 || m >= a.rows || n >= a.cols) return;
    const auto met = out.get(0, m, n, a.cols);
#pragma unroll
    for (int w = 1; w < FEW_WAVES; ++w) acc += sums[w][lane];
    out.put(0, part, m, n, a.cols, acc, met);
}

// What memory holds for four columns of a row, as it lies there, so that several can be on their way: 16 bytes of floats or 8 of 16-bit values, by a type that is known
// when the kernel runs.
__device__ __forceinline__ u4v raw4(int type, const void* p, u64 at, u32 left) {
    if (type == DBLP_F32) {
        const float* const f = (const float*)p + at;
        return __builtin_bit_cast(u4v, left >= 4 ? Vec<F32, 4>::load(f) : Vec<F32, 4>::some(f, left));
    }
    const __bf16* const h = (const __bf16*)p + at;                                   // (either type's: bits)
    const u2v r = left >= 4 ? Vec<BF16, 4>::load(h) : Vec<BF16, 4>::some(h, left);
    return (u4v){r.x, r.y, 0, 0};
}
__device__ __forceinline__ void open4(int type, u4v r, float (&v)[4]) {
    if (type == DBLP_F32) Vec<F32, 4>::open(__builtin_bit_cast(f4v, r), v);
    else if (type == DBLP_BF16) Vec<BF16, 4>::open((u2v){r.x, r.y}, v);
    else Vec<F16, 4>::open((u2v){r.x, r.y}, v);
}
__device__ __forceinline__ void store4(int type, void* p, u64 at, u32 left, const float (&v)[4]) {
    if (type == DBLP_F32) store_cols<Vec<F32, 4>, 4>((float*)p + at, 0, left, v);
    else if (type == DBLP_BF16) store_cols<Vec<BF16, 4>, 4>((__bf16*)p + at, 0, left, v);
    else store_cols<Vec<F16, 4>, 4>((_Float16*)p + at, 0, left, v);
}
struct None {};

// Parts of a sum over k, each a matrix of floats of its own, to be joined; those of one matrix of a batch behind each other.
struct PartOut {
    float* p;
    u64 stride, step;            // of rows, a multiple of four; of parts
    float* row_sums;
    u32 rows, parts;
    __device__ __forceinline__ None get(u32, u32, u32, u32) const { return None(); }
    __device__ __forceinline__ void put(u32 matrix, u32 part, u32 m, u32 n, u32, f4 acc, None) const { *(f4*)(p + ((u64)matrix * parts + part) * step + m * stride + n) = acc; }
    __device__ __forceinline__ void sums(u32, u32 part, u32 m, float s) const { if (row_sums) row_sums[(u64)part * rows + m] = s; }
};

// Adds the parts up, one after the other, eight of them on their way, and hands the results on: a thread takes four columns.  Bound by memory: 138 MB to 13 in 25 us (6 TB/s).
template <class Out>
__global__ __launch_bounds__(256) void join_parts(PartOut in, Units s, Out out) {
    const u32 parts = in.parts, matrix = blockIdx.z;
    const u32 u = blockIdx.x * 256 + threadIdx.x;
    if (u >= s.n) return;
    const u32 row = s.per_row.of(u), c = (u - row * s.per_row.d) * 4, m = (u32)s.row0 + row;
    if (in.row_sums && c == 0) {
        float sum = 0.0f;
        for (u32 i = 0; i < parts; i += 8) {
            float v[8];
#pragma unroll
            for (u32 j = 0; j < 8; ++j) v[j] = i + j < parts ? in.row_sums[(u64)(i + j) * in.rows + m] : 0.0f;
#pragma unroll
            for (u32 j = 0; j < 8; ++j) sum += v[j];
        }
        out.sums(0, 0, m, sum);
    }
    if (c >= s.cols) return;
    const auto met = out.get(matrix, m, c, s.cols);
    const float* const p = in.p + (u64)matrix * parts * in.step + m * in.stride + c;
    f4 sum = {};
    for (u32 i = 0; i < parts; i += 8) {
        f4 v[8];
#pragma unroll
        for (u32 j = 0; j < 8; ++j) v[j] = i + j < parts ? *(const f4*)(p + (i + j) * in.step) : (f4)(0.0f);
#pragma unroll
        for (u32 j = 0; j < 8; ++j) sum += v[j];
    }
    out.put(matrix, 0, m, c, s.cols, sum, met);
}

// At most this many parts, and as many as fit these bytes.
#define PARTS_MOST 64
#define PARTS_BYTES (128ull << 20)
static u64 parts_bytes(u64 rows, u64 cols) {
    const u64 one = rows * round_up(cols, 4) * 4;                                    // (below 2^64: both are below 2^31)
    return one >= PARTS_BYTES / PARTS_MOST ? PARTS_BYTES : one * PARTS_MOST;
}

// Launches of a product's tiles: at most 2^20 tiles, or 2^16 of 2^15 matrices' parts (a grid's threads along x stay below 2^32, its z below 2^16, its blocks below 2^32).
template <int BM, int BN, class F>
static void each_tiles(Product a, u64 matrices, F f, bool symmetric = false) {
    a.tile_cols = (u32)((a.cols + (u64)BN - 1) / BN);
    a.tile_rows = (u32)((a.rows + (u64)BM - 1) / BM);
    a.tiles = symmetric ? (u64)a.tile_rows * (a.tile_rows + 1) / 2 : (u64)a.tile_rows * a.tile_cols;
    for (u64 m = 0; m < matrices; m += 32768 / a.parts) {
        const u64 here = matrices - m < 32768 / a.parts ? matrices - m : 32768 / a.parts;
        const u32 z = (u32)here * a.parts, most = z > 1 ? 1u << 16 : 1u << 20;
        for (a.tile0 = 0; a.tile0 < a.tiles; a.tile0 += most) f(a, dim3((u32)(a.tiles - a.tile0 < most ? a.tiles - a.tile0 : most), 1, z), m);
    }
}

// Whether an operand can be copied to LDS (its chunks begin at multiples of four bytes, as any float does), and whether a tile's offsets fit 31 bits.
template <class T> static bool copied(const Operand& o) {
    const u64 e = sizeof(typename T::elem);
    return !off(o.p, 4) && o.stride * e % 4 == 0 && o.step * e % 4 == 0;
}
template <class T> static bool in_reach(const Operand& o) { return o.stride < (1ull << 31) / 512 / sizeof(typename T::elem); }        // (of 256 rows twice as far apart)
