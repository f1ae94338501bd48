// What the worker's operators share: element types and their vectors, dropout masks, and the host's checks and launches.
#pragma once
#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include "../../include/dblp_worker.h"

typedef unsigned long long u64;
typedef uint32_t u32;
typedef uint16_t u16;

#define WAVE 64

// ------------------------------------------------------------------------------------------
// element types and vectors of them
// ------------------------------------------------------------------------------------------
typedef float f4v __attribute__((ext_vector_type(4)));
typedef u32 u2v __attribute__((ext_vector_type(2)));
typedef u32 u4v __attribute__((ext_vector_type(4)));
typedef f4v f4v_a4 __attribute__((aligned(4)));         // wide accesses at an element's alignment
typedef u2v u2v_a2 __attribute__((aligned(2)));
typedef u4v u4v_a2 __attribute__((aligned(2)));
typedef u16 u16x2 __attribute__((ext_vector_type(2)));

struct F32 { typedef float elem; };
struct BF16 { typedef __bf16 elem; };
struct F16 { typedef _Float16 elem; };

// W neighbouring elements.  `raw`: as they lie in memory, so that several loads can be in flight before the first is converted.
// Lanes that follow each other should hold 16 bytes each: four floats, where a thread with eight would read and write every other 16 bytes
// (a copy of 154 MB takes 52 us one way and 55 to 64 the other, zeros with the streaming hint 27 and 60).
template <class T, int W> struct Vec;

template <> struct Vec<F32, 4> {
    typedef float elem;
    typedef f4v raw;
    static __device__ __forceinline__ raw load(const float* p) { return *(const f4v_a4*)p; }
    static __device__ __forceinline__ raw load_far(const float* p) { return __builtin_nontemporal_load((const f4v_a4*)p); }
    static __device__ __forceinline__ void store(float* p, raw r) { *(f4v_a4*)p = r; }
    static __device__ __forceinline__ void store_far(float* p, raw r) { __builtin_nontemporal_store((f4v_a4)r, (f4v_a4*)p); }
    static __device__ __forceinline__ raw some(const float* p, u32 n) {                    // the first n < 4, zeros behind
        raw r = {};
        for (u32 i = 0; i < 3; ++i) if (i < n) r[i] = p[i];
        return r;
    }
    static __device__ __forceinline__ raw down(raw r, u32 by) {                            // by 0..3 elements, zeros behind
        if (by & 2) r = (raw){r.z, r.w, 0.0f, 0.0f};
        if (by & 1) r = (raw){r.y, r.z, r.w, 0.0f};
        return r;
    }
    static __device__ __forceinline__ void shut(raw& r, const u32* gate) {                 // zeros where the gate is shut
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int half = (i & 1) ? (int)gate[i >> 1] >> 16 : (int)(gate[i >> 1] << 16) >> 16;
            r[i] = __builtin_bit_cast(float, __builtin_bit_cast(int, (float)r[i]) & half);
        }
    }
    static __device__ __forceinline__ void open(raw r, float (&v)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = r[i];
    }
    static __device__ __forceinline__ raw pack(const float (&v)[4]) { return (raw){v[0], v[1], v[2], v[3]}; }
};

template <class T>
struct Vec<T, 8> {
    typedef typename T::elem elem;
    typedef u4v raw;
    typedef elem half8 __attribute__((ext_vector_type(8)));
    typedef float f8v __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ raw load(const elem* p) { return *(const u4v_a2*)p; }
    static __device__ __forceinline__ raw load_far(const elem* p) { return __builtin_nontemporal_load((const u4v_a2*)p); }
    static __device__ __forceinline__ void store(elem* p, raw r) { *(u4v_a2*)p = r; }
    static __device__ __forceinline__ void store_far(elem* p, raw r) { __builtin_nontemporal_store((u4v_a2)r, (u4v_a2*)p); }
    static __device__ __forceinline__ raw some(const elem* p, u32 n) {
        half8 r = {};
        for (u32 i = 0; i < 7; ++i) if (i < n) r[i] = p[i];
        return __builtin_bit_cast(raw, r);
    }
    static __device__ __forceinline__ raw down(raw r, u32 by) {
        if (by & 4) r = (raw){r.z, r.w, 0u, 0u};
        if (by & 2) r = (raw){r.y, r.z, r.w, 0u};
        if (by & 1) r = (raw){r.x >> 16 | r.y << 16, r.y >> 16 | r.z << 16, r.z >> 16 | r.w << 16, r.w >> 16};
        return r;
    }
    static __device__ __forceinline__ void shut(raw& r, const u32* gate) { r &= (raw){gate[0], gate[1], gate[2], gate[3]}; }
    static __device__ __forceinline__ void open(raw r, float (&v)[8]) {
        const f8v f = __builtin_convertvector(__builtin_bit_cast(half8, r), f8v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = f[i];
    }
    static __device__ __forceinline__ raw pack(const float (&v)[8]) {
        return __builtin_bit_cast(raw, __builtin_convertvector(((f8v){v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]}), half8));
    }
};

template <class T>
struct Vec<T, 4> {
    typedef typename T::elem elem;
    typedef u2v raw;
    typedef elem half4 __attribute__((ext_vector_type(4)));
    static __device__ __forceinline__ raw load(const elem* p) { return *(const u2v_a2*)p; }
    static __device__ __forceinline__ raw load_far(const elem* p) { return __builtin_nontemporal_load((const u2v_a2*)p); }
    static __device__ __forceinline__ void store(elem* p, raw r) { *(u2v_a2*)p = r; }
    static __device__ __forceinline__ void store_far(elem* p, raw r) { __builtin_nontemporal_store((u2v_a2)r, (u2v_a2*)p); }
    static __device__ __forceinline__ raw some(const elem* p, u32 n) {
        half4 r = {};
        for (u32 i = 0; i < 3; ++i) if (i < n) r[i] = p[i];
        return __builtin_bit_cast(raw, r);
    }
    static __device__ __forceinline__ raw down(raw r, u32 by) {
        if (by & 2) r = (raw){r.y, 0u};
        if (by & 1) r = (raw){r.x >> 16 | r.y << 16, r.y >> 16};
        return r;
    }
    static __device__ __forceinline__ void shut(raw& r, const u32* gate) { r &= (raw){gate[0], gate[1]}; }
    static __device__ __forceinline__ void open(raw r, float (&v)[4]) {
        const f4v f = __builtin_convertvector(__builtin_bit_cast(half4, r), f4v);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = f[i];
    }
    static __device__ __forceinline__ raw pack(const float (&v)[4]) { return __builtin_bit_cast(raw, __builtin_convertvector(((f4v){v[0], v[1], v[2], v[3]}), half4)); }
};

// Columns [c, c + W) of a row of `cols`, c < cols; those past the end are zero.  WHOLE: there are none.  Otherwise a row's last
// columns are read from its last W elements and shifted down in registers (rows of fewer than W elements apart): one load for every thread.
// The shift is a call of its own, for when all loads have been asked for: made with the load it would wait for each of them (embed_grad of
// 17000 tokens of 333 columns).  FAR: with the hint that the data are not used again soon.
template <class V, int W, bool WHOLE, bool FAR = false>
__device__ __forceinline__ typename V::raw load_cols(const typename V::elem* row, u32 c, u32 cols) {
    if (WHOLE) return FAR ? V::load_far(row + c) : V::load(row + c);
    if (cols < W) return V::some(row, cols);
    const u32 at = c + W <= cols ? c : cols - W;
    return FAR ? V::load_far(row + at) : V::load(row + at);
}
template <class V, int W, bool WHOLE>
__device__ __forceinline__ typename V::raw settle_cols(typename V::raw r, u32 c, u32 cols) {
    return WHOLE || cols < W ? r : V::down(r, c + W <= cols ? 0 : c + W - cols);
}
// ... and those past the end are not written.
template <class V, int W, bool FAR = false>
__device__ __forceinline__ void store_cols(typename V::elem* row, u32 c, u32 cols, const float (&v)[W]) {
    if (c + W <= cols) {
        if (FAR) V::store_far(row + c, V::pack(v));
        else V::store(row + c, V::pack(v));
        return;
    }
    for (u32 i = 0; i < W; ++i) if (c + i < cols) row[c + i] = (typename V::elem)v[i];
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
// limit: fields below it are dropped (65535 at most); some: zero if everything is dropped; keep: factor of what is kept
struct Mask { u64 seed, draw; const u64* d_draw; u32 some; float keep; u16 limit; bool on; };

__device__ __forceinline__ u64 draw_of(const Mask& m) { return m.draw + (m.d_draw ? *m.d_draw : 0); }

// The gates of eight columns, two a word: all ones in the half of a value that is kept.
// Ten rounds are 20 products of 32 x 32 bits (a quarter of the vector rate) and 20 exclusive ors for eight values, about 400 of a SIMD's
// cycles a wave: nearly as long as it takes to move 64 x 8 16-bit values in and out.  So gates are computed while the values are on their way.
struct Gates { u32 w[4]; };
__device__ __forceinline__ u32 xor3(u32 a, u32 b, u32 c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }
__device__ __forceinline__ Gates gates_of(const Mask& m, u64 draw, u64 g) {
    u32 a = (u32)g, b = (u32)(g >> 32), c = (u32)draw, d = (u32)(draw >> 32), k0 = (u32)m.seed, k1 = (u32)(m.seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const u64 p = (u64)a * 0xD2511F53u, q = (u64)c * 0xCD9E8D57u;
        a = xor3((u32)(q >> 32), b, k0);
        b = (u32)q;
        c = xor3((u32)(p >> 32), d, k1);
        d = (u32)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    const u32 w[4] = {a, b, c, d};
    Gates r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // limit - field, not below zero: more than zero where the value is dropped; one of it is one, less one is all ones or zero
        const u16x2 short_of = __builtin_elementwise_sub_sat((u16x2){m.limit, m.limit}, __builtin_bit_cast(u16x2, w[i]));
        r.w[i] = __builtin_bit_cast(u32, __builtin_elementwise_min(short_of, (u16x2){1, 1}) - (u16x2){1, 1}) & m.some;
    }
    return r;
}
// For threads of four columns: lanes 2i and 2i + 1 share the eight of groups ga and gb (of two rows that both hold).  Each computes one of them
// and they exchange halves.  Both lanes have to be active.
__device__ __forceinline__ u32 from_neighbour(u32 v) { return (u32)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true); }     // quad_perm 1, 0, 3, 2
__device__ __forceinline__ void gates_of_two(const Mask& m, u64 draw, u64 ga, u64 gb, u32 (&wa)[2], u32 (&wb)[2]) {
    const bool odd = threadIdx.x & 1;
    const Gates q = gates_of(m, draw, odd ? gb : ga);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const u32 got = from_neighbour(odd ? q.w[i] : q.w[2 + i]);
        wa[i] = odd ? got : q.w[i];
        wb[i] = odd ? q.w[2 + i] : got;
    }
}

// ------------------------------------------------------------------------------------------
// matrices as one row of units: a unit is the W columns of one thread.  A row has an even number of units of four columns, so that lanes
// 2i and 2i + 1 always share a group of eight (the last unit of a row may have no column)
// ------------------------------------------------------------------------------------------
struct Units { u64 row0; u32 n, cols; Divider per_row; };     // units of this launch (below 2^31), its first row

template <int W> static u32 units_per_row(u32 cols) { return (u32)((cols + 7ull) / 8) * (8 / W); }

#define COUNT_LIMIT (1ull << 31)

// Calls f(Units) for launches of fewer than 2^31 units each.
template <int W, class F>
static void each_launch(u64 rows, u32 cols, F f) {
    const u32 per_row = units_per_row<W>(cols);
    const u64 most = (COUNT_LIMIT - 1) / per_row;
    for (u64 row0 = 0; row0 < rows; row0 += most) {
        const u64 n = rows - row0 < most ? rows - row0 : most;
        f(Units{row0, (u32)(n * per_row), cols, Divider::by(per_row)});
    }
}
static inline u32 blocks_of(u64 units, u32 each) { return (u32)((units + each - 1) / each); }

// ------------------------------------------------------------------------------------------
// host: errors, checks, devices
// ------------------------------------------------------------------------------------------
extern thread_local char worker_err[192];

static inline int refuse(const char* call, const char* why) {
    snprintf(worker_err, sizeof worker_err, "%s: %s", call, why);
    return DBLP_EINVAL;
}
#define REFUSE_IF(cond, why) do { if (cond) return refuse(call, why); } while (0)

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

// Launches of a call.  A launch's own result is asked for: the thread's last error may be one of the caller's, which is neither this call's failure nor
// its to clear.  After a failure nothing more is launched.
struct Launches {
    hipError_t err = hipSuccess;
    template <class... P, class... A>
    void operator()(void (*kernel)(P...), dim3 grid, u32 threads, hipStream_t stream, A... args) {
        if (err == hipSuccess) err = one<P...>((const void*)kernel, grid, threads, stream, args...);
    }
private:
    template <class... P>
    static hipError_t one(const void* kernel, dim3 grid, u32 threads, hipStream_t stream, P... params) {
        void* at[] = {(void*)&params...};
        return hipLaunchKernel(kernel, grid, dim3(threads), at, 0, stream);
    }
};
static inline int launched(const char* call, const Launches& l) {
    if (l.err == hipSuccess) return DBLP_OK;
    snprintf(worker_err, sizeof worker_err, "%s: %s", call, hipGetErrorString(l.err));
    (void)hipGetLastError();
    return DBLP_EHIP;
}
static inline int no_device(const char* call, hipError_t e) {
    snprintf(worker_err, sizeof worker_err, "%s: hipSetDevice: %s", call, hipGetErrorString(e));
    (void)hipGetLastError();
    return DBLP_EHIP;
}

static inline u32 type_bytes(int type) { return type == DBLP_F32 ? 4 : 2; }
static inline bool bad_type(int type) { return type != DBLP_F32 && type != DBLP_BF16 && type != DBLP_F16; }
static inline bool off(const void* p, u32 bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }
static inline u64 round_up(u64 n, u64 to) { return (n + to - 1) / to * to; }

static inline int take_drop(const char* call, const dblp_drop* h, Mask* m) {
    *m = Mask{0, 0, nullptr, 0xFFFFFFFFu, 1.0f, 0, false};
    if (!h) return DBLP_OK;
    REFUSE_IF(!(h->p >= 0.0 && h->p <= 1.0), "p must be in 0..1");
    REFUSE_IF(off(h->d_draw, 8), "d_draw must be 8-byte aligned");
    const u32 limit = (u32)rint(65536.0 * h->p);
    *m = Mask{h->seed, h->draw, (const u64*)h->d_draw, limit < 65536 ? 0xFFFFFFFFu : 0u, limit < 65536 ? (float)(65536.0 / (65536.0 - limit)) : 0.0f, (u16)(limit < 65536 ? limit : 65535), limit != 0};
    return DBLP_OK;
}

template <int N> struct Int { static constexpr int value = N; };

template <class F>
static void by_type(int type, F f) {
    if (type == DBLP_F32) f(F32());
    else if (type == DBLP_BF16) f(BF16());
    else f(F16());
}
