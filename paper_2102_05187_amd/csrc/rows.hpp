// What the kernels over dense rows share: element types, 16-byte vectors of a row that starts anywhere, the running
// maximum and sum of a softmax, and reductions over a workgroup.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

#include "../../include/comet.h"

namespace comet {

constexpr float kNegInf = -__builtin_huge_valf();
constexpr double kNegInfD = -__builtin_huge_val();
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWave = 64;

// A barrier for what the threads tell each other through LDS.  __syncthreads() also waits for every load and store to memory that the thread
// has under way; here a row's loads go on across barriers, and nothing passes from thread to thread through memory.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// ---- element types ------------------------------------------------------------------------------------
typedef float F2 __attribute__((ext_vector_type(2)));
typedef __bf16 B2 __attribute__((ext_vector_type(2)));
typedef _Float16 H2 __attribute__((ext_vector_type(2)));

template <int TYPE> struct Elem;
template <> struct Elem<COMET_F32> {
    using T = uint32_t;
    static constexpr int kPer = 4;                          // elements of a 16-byte vector
    static constexpr uint32_t kNone = 0xff800000u;          // 32 bits of -inf
    static __device__ __forceinline__ float one(uint32_t x) { return __uint_as_float(x); }
    static __device__ __forceinline__ void widen(const uint4 &v, float *f) {
        f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ uint32_t bits(float f) { return __float_as_uint(f); }
    static __device__ __forceinline__ uint4 narrow(const float *f) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
};
template <> struct Elem<COMET_BF16> {
    using T = uint16_t;
    static constexpr int kPer = 8;
    static constexpr uint32_t kNone = 0xff80ff80u;
    static __device__ __forceinline__ float one(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
    static __device__ __forceinline__ void widen(const uint4 &v, float *f) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    // to the nearest, ties to even; a NaN stays one
    static __device__ __forceinline__ uint16_t bits(float f) {
        const __bf16 b = (__bf16)f;
        return __builtin_bit_cast(uint16_t, b);
    }
    static __device__ __forceinline__ uint4 narrow(const float *f) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const F2 two = {f[2 * i], f[2 * i + 1]};
            w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(two, B2));
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <> struct Elem<COMET_F16> {
    using T = uint16_t;
    static constexpr int kPer = 8;
    static constexpr uint32_t kNone = 0xfc00fc00u;
    static __device__ __forceinline__ float one(uint16_t x) { return (float)__builtin_bit_cast(_Float16, x); }
    static __device__ __forceinline__ void widen(const uint4 &v, float *f) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = one((uint16_t)(w[i] & 0xffffu));
            f[2 * i + 1] = one((uint16_t)(w[i] >> 16));
        }
    }
    static __device__ __forceinline__ uint16_t bits(float f) { return __builtin_bit_cast(uint16_t, (_Float16)f); }
    static __device__ __forceinline__ uint4 narrow(const float *f) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const F2 two = {f[2 * i], f[2 * i + 1]};
            w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(two, H2));
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

// ---- a row as 16-byte vectors ---------------------------------------------------------------------------
// Vector i holds the elements i * kPer .. of the row wherever the row starts, so that what is computed from a row does not
// depend on its address.  The device loads and stores 16 bytes at any address: at multiples of 4 as fast as at multiples of
// 16 (6.6 TB/s over rows of 256 KB), at odd multiples of 2 a fifth slower (5.2 TB/s).
// A row of 16-bit elements at such an odd multiple (`odd`: every other row where the rows' distance is odd) can therefore be read from one
// element before it on, which is the row before's; every vector gets its last element from the vector behind it: the next lane's, or,
// for the wavefront's last lane, from edges(), one load for all of a thread's vectors.  Row 0 has none before it, and is read as it lies.  So
// are short rows (forward of 8192 x 8003 58 us shifted, 54 as they lie).  Long ones gain where they come from memory and lose where the last
// cache has them, at any size: top 64 of 1677 x 60013 55 us shifted and 57 as they lie from memory, 48 and 44 from the cache, forward of
// 559 x 60013 23 and 24, 21 and 20, gradient of 512 x 131071 53 and 58, 44 and 45.  From 256 MB on (3494 x 60013: 95 and 108, 89 and 94, 157 and 176) they
// come from memory, below 48 MB mostly from the cache, and in between it is as often one as the other.
inline bool read_shifted(int type, int64_t N, int64_t V) { return type != COMET_F32 && V >= 16384 && N * V * 2 >= (int64_t(48) << 20); }
// Rows of 256 MB and more in all do not stay in the last cache (of that size).  Where nothing is written that is of their size they are read past
// it: top 64 of 2048 x 131072 of 16 bits 101 us through it, 95.6 past it, of 8192 x 32000 107 and 104, forward 102 and 91, 102 and 97.  Smaller ones
// are often there already: forward of 256 x 131072 17 us through it, 21 past it.  The gradient gains nothing that way (4096 x 131072 349 us and 345, 16384 x
// 32000 374 and 378, the step with a quarter of its rows ignored 424 and 431).
inline bool read_once(int type, int64_t N, int64_t V) { return N * V * (type == COMET_F32 ? 4 : 2) >= (int64_t(256) << 20); }

typedef uint32_t V4At4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t V4At2 __attribute__((ext_vector_type(4), aligned(2)));
template <int ALIGN> struct Wide { using type = V4At4; };
template <> struct Wide<2> { using type = V4At2; };

template <int TYPE> struct Row {
    using E = Elem<TYPE>;
    using T = typename E::T;
    using V4 = typename Wide<sizeof(T)>::type;
    const T *p;              // the row's first element
    int64_t n;               // its length
    bool odd;
    __device__ __forceinline__ Row(const void *base, int64_t row, int64_t ld, int64_t len, bool shift = false)
        : p((const T *)base + row * ld), n(len), odd(sizeof(T) == 2 && shift && row > 0 && ((uintptr_t)p & 2)) {}
    __device__ __forceinline__ int64_t first(int64_t i) const { return i * E::kPer; }           // column of the vector's first element
    __device__ __forceinline__ bool whole(int64_t i) const { return first(i) + E::kPer <= n; }
    __device__ __forceinline__ uint4 raw(int64_t i) const {
        const V4 v = *(const V4 *)(p + first(i));
        return make_uint4(v.x, v.y, v.z, v.w);
    }
    // A load that goes past the caches.  Of two branches with a plain load and this one the compiler would make one, with the plain load: it is
    // kept from seeing that the addresses are the same.
    static __device__ __forceinline__ V4 load_once(const V4 *at) {
        auto *g = (const __attribute__((address_space(1))) V4 *)at;
        asm("" : "+v"(g));
        return __builtin_nontemporal_load(g);
    }
    // 16 bytes from vector i's first element on, or from the one before it of an odd row
    template <bool ONCE> __device__ __forceinline__ uint4 stream(int64_t i) const {
        const V4 *at = (const V4 *)(p + first(i) - (odd ? 1 : 0));
        const V4 v = ONCE ? load_once(at) : *at;
        return make_uint4(v.x, v.y, v.z, v.w);
    }
    // What settle() needs of a piece of `own` whole vectors from v0 on: lane j's `each` is the last element of the wavefront's 64 vectors j THREADS + t,
    // `last` that of the piece's last vector.
    struct Edges { uint32_t each, last; };
    template <int THREADS> __device__ __forceinline__ Edges edges(int64_t v0, int own) const {
        Edges e{0, 0};
        if constexpr (sizeof(T) == 2) {
            if (odd && own > 0) {
                const int i = (int)(threadIdx.x & (kWave - 1)) * THREADS + (int)(threadIdx.x | (kWave - 1));
                if (i < own) e.each = p[first(v0 + i) + E::kPer - 1];
                e.last = p[first(v0 + own) - 1];
            }
        }
        return e;
    }
    // Of an odd row, the piece's vector i = j THREADS + t from what stream() gave the wavefront; nothing where it is not of the `own`.  By whole wavefronts.
    __device__ __forceinline__ uint4 settle(uint4 v, const Edges &e, int j, int i, int own) const {
        uint32_t next = __builtin_amdgcn_update_dpp(__builtin_amdgcn_readlane(e.each, j), v.x, 0x130, 0xf, 0xf, false);      // the next lane's
        next = i == own - 1 ? e.last : next;
        const uint4 r = make_uint4(__builtin_amdgcn_alignbit(v.y, v.x, 16), __builtin_amdgcn_alignbit(v.z, v.y, 16),
                                   __builtin_amdgcn_alignbit(v.w, v.z, 16), __builtin_amdgcn_alignbit(next, v.w, 16));
        return i < own ? r : make_uint4(E::kNone, E::kNone, E::kNone, E::kNone);
    }
    // elements of vector i as floats, -inf behind the row's end
    __device__ __forceinline__ void load(int64_t i, float *f) const {
        if (whole(i)) { E::widen(raw(i), f); return; }
        const int64_t c = first(i);
#pragma unroll
        for (int k = 0; k < E::kPer; ++k) f[k] = c + k < n ? E::one(p[c + k]) : kNegInf;
    }
};

// A copy of registers that the compiler knows nothing about: what is computed from it is computed anew, and not kept from the last
// time.  Nothing is moved across, either: the floats of one vector are live at a time.
__device__ __forceinline__ uint4 again(uint4 v) {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w));
    return v;
}

// ---- running maximum and sum ------------------------------------------------------------------------------
// s = sum of exp2(c (z - m)) over what was taken in, m its largest element.  An element that is -inf adds nothing, a NaN makes s a NaN.
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

struct MaxSum {
    float m = kNegInf, s = 0.f;
    __device__ __forceinline__ void join(float m2, float s2, float c) {
        const float M = fmaxf(m, m2);
        s = s * (m == M ? 1.f : exp2_fast((m - M) * c)) + s2 * (m2 == M ? 1.f : exp2_fast((m2 - M) * c));
        m = M;
    }
};

// The same while it is taken in, with one multiply-add and one exp2 an element: s holds exp2(c z - shift), where shift is c m rounded,
// and what that rounding did to all terms alike is taken out at the end.  It is half a unit of c m at most: 64 below 2^31, and a sum of 2^31
// terms of 2^64 is still a number.  From there on (at scale 1 masks of -1.5e9 and below, the lowest value of a type among them, +inf) shift stays at the limit:
// a thread whose places are all far below it has a sum of 0, as they have in a row with an ordinary maximum; the sum of a row, or a
// piece of one, whose maximum is itself wild() is taken again by slow_sum.
constexpr float kWild = 0x1p31f;
__device__ __forceinline__ bool wild(float m, float c) { return m > kNegInf && !(fabsf(m * c) < kWild); }

struct Running {
    float m = kNegInf, s = 0.f, shift = -kWild;
    __device__ __forceinline__ void raise(float b, float c) {
        if (b > m) {
            const float sh = fminf(fmaxf(b * c, -kWild), kWild);
            s *= exp2_fast(shift - sh);
            m = b, shift = sh;
        }
    }
    template <int N> __device__ __forceinline__ void add(const float *f, float c) {
        float t[4] = {s, 0.f, 0.f, 0.f};                         // four sums: an addition need not wait for the one before
#pragma unroll
        for (int k = 0; k < N; ++k) t[k % 4] += exp2_fast(__builtin_fmaf(f[k], c, -shift));
        s = (t[0] + t[1]) + (t[2] + t[3]);
    }
    // N elements, b the largest
    template <int N> __device__ __forceinline__ void take(const float *f, float b, float c) {
        raise(b, c);
        add<N>(f, c);
    }
    __device__ __forceinline__ MaxSum sum(float c) const {
        MaxSum r;
        r.m = m;
        const float e = -__builtin_fmaf(m, c, -shift);            // what makes s relative to m: up to any size where shift is at its lower limit
        r.s = s * (e < 100.f ? exp2_fast(e) : 0.f);
        return r;
    }
};

// A logarithm of a sum in two parts, big + log(sum of exp(. - big)): where all terms are the lowest value of their type, or near it,
// the second part would be lost in one number.
struct Log {
    double big, rest;
    __device__ __forceinline__ bool none() const { return big == kNegInfD; }                      // of nothing
};
__device__ __forceinline__ Log make_log(double big, double sum) {
    Log l;
    l.big = big;
    l.rest = big == kNegInfD && !(sum != sum) ? 0.0 : log(sum);
    if (sum != sum) l.big = sum;
    return l;
}
// ln of a 32-bit sum, to about 2^-24 whatever its size: the exponent is taken off first.  0 gives -inf, a NaN itself.
__device__ __forceinline__ double log_of(float s) {
    const int e = s >= 0x1p-126f && s < __builtin_huge_valf() ? (int)(__float_as_uint(s) >> 23) - 127 : 0;
    const float m = __builtin_ldexpf(s, -e);                                   // 1 <= m < 2
    return ((double)e + (double)__builtin_amdgcn_logf(m)) * 0.6931471805599453;
}

// ---- reductions ---------------------------------------------------------------------------------------------
// Over a wavefront with data-parallel moves (lanes 1, 2, 4, 8 back in rows of 16, then row ends onto the rows behind them):
// the last lane ends up with everything, in one fixed order.  A lane that a move does not reach sees `none`.
template <int CTRL, int ROWS> __device__ __forceinline__ float dpp(float none, float v) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(none), __float_as_uint(v), CTRL, ROWS, 0xf, false));
}
template <class F> __device__ __forceinline__ float wave_reduce(float v, float none, F f) {
    v = f(v, dpp<0x111, 0xf>(none, v));
    v = f(v, dpp<0x112, 0xf>(none, v));
    v = f(v, dpp<0x114, 0xf>(none, v));
    v = f(v, dpp<0x118, 0xf>(none, v));
    v = f(v, dpp<0x142, 0xa>(none, v));
    v = f(v, dpp<0x143, 0xc>(none, v));
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}
struct Add { template <class X> __device__ __forceinline__ X operator()(X a, X b) const { return a + b; } };
struct Larger { __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); } };
struct Smaller { __device__ __forceinline__ float operator()(float a, float b) const { return fminf(a, b); } };
struct Max { __device__ __forceinline__ double operator()(double a, double b) const { return a != a || a > b ? a : b; } };   // a NaN on the left stays

template <int CTRL, int ROWS> __device__ __forceinline__ double dpp(double none, double v) {
    const int lo = __builtin_amdgcn_update_dpp(__double2loint(none), __double2loint(v), CTRL, ROWS, 0xf, false);
    const int hi = __builtin_amdgcn_update_dpp(__double2hiint(none), __double2hiint(v), CTRL, ROWS, 0xf, false);
    return __hiloint2double(hi, lo);
}
template <class F> __device__ __forceinline__ double wave_reduce(double v, double none, F f) {
    v = f(v, dpp<0x111, 0xf>(none, v));
    v = f(v, dpp<0x112, 0xf>(none, v));
    v = f(v, dpp<0x114, 0xf>(none, v));
    v = f(v, dpp<0x118, 0xf>(none, v));
    v = f(v, dpp<0x142, 0xa>(none, v));
    v = f(v, dpp<0x143, 0xc>(none, v));
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), 63), __builtin_amdgcn_readlane(__double2loint(v), 63));
}
__device__ __forceinline__ void wave_join(MaxSum &a, float c) {
    const float M = wave_reduce(a.m, kNegInf, Larger());
    a.s = wave_reduce(a.m == M ? a.s : a.s * exp2_fast((a.m - M) * c), 0.f, Add());
    a.m = M;
}
// over a workgroup of T threads; buf has a place for every wavefront and is free again after the call's last barrier
template <int T> __device__ __forceinline__ void block_join(MaxSum &a, float c, float2 *buf) {
    wave_join(a, c);
    if (T == kWave) return;
    if ((threadIdx.x & (kWave - 1)) == 0) buf[threadIdx.x / kWave] = make_float2(a.m, a.s);
    lds_barrier();
    a = MaxSum();
#pragma unroll
    for (int w = 0; w < T / kWave; ++w) a.join(buf[w].x, buf[w].y, c);
    lds_barrier();
}
// The sum over columns [begin, end) of a row whose maximum there is m, against m itself: what Running does not have where m is wild.  A column
// that `skip` names is left out.  Where m is +inf it is the number of its places, or a NaN.  By a workgroup of T threads.
template <int TYPE, int T, class SKIP>
__device__ __forceinline__ float slow_sum(const Row<TYPE> &row, int64_t begin, int64_t end, float m, float c, float2 *buf, SKIP skip) {
    MaxSum a;
    a.m = m;
    for (int64_t i = begin + threadIdx.x; i < end && i < row.n; i += T)
        if (!skip(i)) {
            const float z = Elem<TYPE>::one(row.p[i]);
            a.s += z == m ? 1.f : exp2_fast((z - m) * c);
        }
    block_join<T>(a, c, buf);
    return a.s;
}

// ---- order ------------------------------------------------------------------------------------------------------
// An unsigned number whose order is that of the float (-0 as 0).
__device__ __forceinline__ uint32_t order_of(float z) {
    const uint32_t u = __float_as_uint(z + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
    return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
// Larger value first, then lower column; 0 is less than every key of an element that can be kept.
__device__ __forceinline__ uint64_t key_of(float z, uint32_t column) { return (uint64_t)order_of(z) << 32 | (uint32_t)~column; }
__device__ __forceinline__ uint32_t column_of(uint64_t key) { return ~(uint32_t)key; }
__device__ __forceinline__ float value_of_key(uint64_t key) { return value_of((uint32_t)(key >> 32)); }

}  // namespace comet
