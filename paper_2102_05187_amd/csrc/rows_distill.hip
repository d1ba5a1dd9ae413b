// Distillation from a teacher's top logits: loss and gradient.
//
// With x = scale z, the student's places fall into the row's entries c and all others ("outside").  The dense pass takes in
//   without tail  all places:  S = sum exp(x_j - M),            lse = M + ln S
//   with tail     those outside: S_o, M_o, L_o = M_o + ln S_o,  lse = log(exp(L_o) + sum_c exp(x_c))
// so that neither the tail's mass nor its logarithm is a difference of nearly equal numbers, or lost where the entries' logits are
// far above it.  The gradient is  w scale (P q_c - p_c)  at the entries and  w scale A exp(x_j - M)  elsewhere, with
//   A = P / S                                   (P = sum p + rest: 1 up to rounding, 0 for an empty row)
//   A = (P exp(L_o - lse) - rest) / S_o         (r_j = exp(x_j - M_o) / S_o sums to 1 outside)
// What a row has once (logs, sums over its entries) is computed in 64 bits: the loss is a difference of logs.
//
// The entries' places are marked in LDS, a bit each.  The dense pass of the gradient leaves marked places alone, and the entries'
// gradients are written on their own: no order between the two is needed, also where dZ is Z.
#include "rows.hpp"
#include "rows_kernels.hpp"

namespace comet {

namespace {

constexpr double kNoTailBelow = 0x1p-20;

struct Stat { double m, A, P; Log lse, norm; };   // comet_distill_forward's stat
static_assert(sizeof(Stat) == COMET_DISTILL_STAT * sizeof(double), "stat");

// The entries of a row.
struct Entries {
    const int32_t *crd;
    const float *tvals;
    int64_t begin, end, V;
    double scale;
    __device__ __forceinline__ Entries(const DistillArgs &a, int64_t r)
        : crd(a.crd), tvals(a.tvals), begin(a.pos ? a.pos[r] : r * a.K), end(a.pos ? a.pos[r + 1] : begin + a.K), V(a.V), scale(a.scale) {}
    __device__ __forceinline__ bool at(int64_t e, int64_t *c) const {
        *c = crd[e];
        return *c >= 0 && *c < V;
    }
    __device__ __forceinline__ double a(int64_t e) const { return (double)tvals[e] * scale; }
};

template <int TYPE> __device__ __forceinline__ double student(const Row<TYPE> &row, int64_t c, double scale) {
    return (double)Elem<TYPE>::one(row.p[c]) * scale;
}

// What the entries alone give, with ta and xa the largest of the a and of the x:
//   S = sum exp(a - ta),  D = sum exp(a - ta) ((a - ta) - (x - xa)),  X = sum exp(x - xa)
struct Taught { double ta, xa, S, D, X; };

// By one wavefront.
template <int TYPE> __device__ Taught teach(const Row<TYPE> &row, const Entries &en) {
    const int lane = threadIdx.x & (kWave - 1);
    Taught t{kNegInfD, kNegInfD, 0, 0, 0};
    int64_t c;
    for (int64_t e = en.begin + lane; e < en.end; e += kWave)
        if (en.at(e, &c)) {
            t.ta = Max()(t.ta, en.a(e));
            t.xa = Max()(t.xa, student(row, c, en.scale));
        }
    t.ta = wave_reduce(t.ta, kNegInfD, Max());
    t.xa = wave_reduce(t.xa, kNegInfD, Max());
    for (int64_t e = en.begin + lane; e < en.end; e += kWave)
        if (en.at(e, &c)) {
            const double a = en.a(e), x = student(row, c, en.scale);
            const double p = a == kNegInfD ? 0.0 : exp(a - t.ta);
            t.S += p;
            if (p != 0) t.D += p * ((a - t.ta) - (x == kNegInfD ? x : x - t.xa));
            t.X += x == kNegInfD ? 0.0 : exp(x - t.xa);
        }
    t.S = wave_reduce(t.S, 0.0, Add());
    t.D = wave_reduce(t.D, 0.0, Add());
    t.X = wave_reduce(t.X, 0.0, Add());
    return t;
}

// Loss of a row (times its weight) and what its gradient needs, from the entries' sums and the dense pass's.
__device__ double finish(const Taught &t, MaxSum d, bool tail, double tlse, double scale, double w, Stat *out) {
    const Log dense = log_sum(d, scale);
    const bool some = t.ta != kNegInfD;                          // an entry has a probability
    Log norm = make_log(t.ta, t.S), lse = dense;
    double mass = some ? 1.0 : 0.0, share = mass;                // share: the factor of exp(a - ta)
    if (tail) {
        norm = Log{tlse, 0.0};
        share = some ? exp(t.ta - tlse) : 0.0;
        mass = tlse != tlse ? tlse : share * t.S;
        if (t.xa != kNegInfD) {
            const double m = dense.none() || t.xa != t.xa || t.xa > dense.big ? t.xa : dense.big;
            lse = make_log(m, t.X * exp(t.xa - m) + (dense.none() ? 0.0 : exp((dense.big - m) + dense.rest)));
        }
    } else if (some) share = 1.0 / t.S;
    double loss = 0;
    if (some) loss = share * t.D + mass * ((t.ta - norm.big) - norm.rest + (t.xa == kNegInfD ? 0.0 : (lse.big - t.xa) + lse.rest));
    const double outside = dense.none() ? kNegInfD : (dense.big - lse.big) + (dense.rest - lse.rest);      // log of the dense pass's share
    double rest = 0;
    if (tail) {
        rest = 1.0 - mass;
        if (rest < kNoTailBelow) rest = 0;
        if (rest != 0) loss += rest * (log(rest) - outside);
    }
    const double P = mass + rest;
    out->P = P;
    out->norm = norm;
    out->lse = lse;
    out->m = d.m == kNegInf ? 0.0 : (double)d.m;
    if (d.m == kNegInf) out->A = d.s != d.s ? (double)d.s : 0.0;   // nothing is left for the dense pass, or it is NaN
    else out->A = ((tail ? P * exp(outside) : P) - rest) / (double)d.s;
    const double bad = (lse.big + P) + t.S;                        // NaN and +inf in the row or its entries
    if (bad != bad) loss = out->A = bad;
    return w * loss;
}

// ---- marks --------------------------------------------------------------------------------------------------
// A bit for each of `columns` places from `base` on, a multiple of 32; all threads call this, and a barrier has to follow.
template <int T> __device__ __forceinline__ void clear_marks(uint32_t *marks, int columns) {
    for (int i = threadIdx.x; i < (columns + 31) / 32; i += T) marks[i] = 0;
    __syncthreads();
}
template <int T> __device__ __forceinline__ void set_marks(uint32_t *marks, const Entries &en, int64_t base, int columns) {
    int64_t c;
    for (int64_t e = en.begin + threadIdx.x; e < en.end; e += T)
        if (en.at(e, &c) && c >= base && c < base + columns) atomicOr(&marks[(c - base) >> 5], 1u << ((c - base) & 31));
}
// The marks of vector i of the piece.
template <int P> __device__ __forceinline__ uint32_t marks_at(const uint32_t *marks, int i) {
    const int c = i * P;
    return marks[c >> 5] >> (c & 31) & ((1u << P) - 1);
}
template <int P> __device__ __forceinline__ void leave_out(float *f, uint32_t mk) {
    if (mk) {
#pragma unroll
        for (int k = 0; k < P; ++k) if (mk >> k & 1) f[k] = kNegInf;
    }
}

// ---- forward --------------------------------------------------------------------------------------------------
constexpr int kThreads = 256;
constexpr int kPiece = 16384;             // vectors of a piece at most: its marks take 16 KB
constexpr int kAhead = 4;                 // vectors that a thread has in flight

struct Pieces {                           // how a row is cut: `count` pieces of `vectors` vectors
    int vectors, count;
};

template <int TYPE, bool TAIL>
__global__ void __launch_bounds__(kThreads) k_distill_forward(DistillArgs a, float c2, Pieces cut, float *__restrict__ loss, Stat *__restrict__ stat,
                                                              float2 *__restrict__ partial) {
    using E = Elem<TYPE>;
    constexpr int P = E::kPer, T = kThreads, U = kAhead;
    __shared__ float2 buf[T / kWave];
    extern __shared__ uint32_t marks[];
    const int64_t r = blockIdx.x / (unsigned)cut.count;
    const int piece = (int)(blockIdx.x - r * cut.count);
    const float w = a.weight ? a.weight[r] : 1.f;
    if (w == 0) {
        if (threadIdx.x == 0 && cut.count == 1) loss[r] = 0;
        return;
    }
    const Row<TYPE> row(a.Z, r, a.ldz, a.V);
    const int64_t v0 = (int64_t)piece * cut.vectors, full = a.V / P;
    const int own = (int)(full - v0 < cut.vectors ? full - v0 : cut.vectors);
    const bool ends_here = a.V % P != 0 && full >= v0 && full < v0 + cut.vectors;
    uint4 v[U];
    auto fetch = [&](int i0) {
        if (i0 + U * T <= own) {
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = row.raw(v0 + i0 + u * T + threadIdx.x);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * T + threadIdx.x;
                v[u] = make_uint4(E::kNone, E::kNone, E::kNone, E::kNone);
                if (i < own) v[u] = row.raw(v0 + i);
            }
        }
    };
    fetch(0);
    if (TAIL) {
        const Entries en(a, r);
        clear_marks<T>(marks, cut.vectors * P);
        set_marks<T>(marks, en, v0 * P, cut.vectors * P);
        __syncthreads();
    }
    Running run;
    for (int i0 = 0; i0 < own; i0 += U * T) {
        uint4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = v[u];
        if (i0 + U * T < own) fetch(i0 + U * T);
        float b = kNegInf;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[P];
            E::widen(x[u], f);
            if (TAIL) {
                const int i = i0 + u * T + threadIdx.x;
                const uint32_t mk = i < own ? marks_at<P>(marks, i) : 0;
                if (mk) {                                        // rare: the places' bits become -inf
                    leave_out<P>(f, mk);
                    x[u] = E::narrow(f);
                }
            }
#pragma unroll
            for (int k = 0; k < P; ++k) b = fmaxf(b, f[k]);
        }
        run.raise(b, c2);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[P];
            E::widen(x[u], f);
            run.template add<P>(f, c2);
        }
    }
    if (ends_here && threadIdx.x == 0) {
        float f[P], b = kNegInf;
        row.load(full, f);
        if (TAIL) leave_out<P>(f, marks_at<P>(marks, (int)(full - v0)));
#pragma unroll
        for (int k = 0; k < P; ++k) b = fmaxf(b, f[k]);
        run.template take<P>(f, b, c2);
    }
    MaxSum d = run.sum(c2);
    block_join<T>(d, c2, buf);
    if (cut.count > 1) {
        if (threadIdx.x == 0) partial[blockIdx.x] = make_float2(d.m, d.s);
    } else if (threadIdx.x < kWave) {
        const Taught t = teach(row, Entries(a, r));
        Stat s;
        const double l = finish(t, d, TAIL, TAIL ? a.tlse[r] : 0.0, a.scale, w, &s);
        if (threadIdx.x == 0) { loss[r] = (float)l; stat[r] = s; }
    }
}

// Joins the pieces of a row, a wavefront a row.
template <int TYPE>
__global__ void __launch_bounds__(kThreads) k_distill_finish(DistillArgs a, float c2, int count, const float2 *__restrict__ partial,
                                                             float *__restrict__ loss, Stat *__restrict__ stat) {
    const int64_t r = (int64_t)blockIdx.x * (kThreads / kWave) + threadIdx.x / kWave;
    const int lane = threadIdx.x & (kWave - 1);
    if (r >= a.N) return;
    const float w = a.weight ? a.weight[r] : 1.f;
    if (w == 0) {
        if (lane == 0) loss[r] = 0;
        return;
    }
    MaxSum d;
    for (int i = lane; i < count; i += kWave) {
        const float2 p = partial[r * count + i];
        d.join(p.x, p.y, c2);
    }
    const Row<TYPE> row(a.Z, r, a.ldz, a.V);
    const Taught t = teach(row, Entries(a, r));
    wave_join(d, c2);
    Stat s;
    const double l = finish(t, d, a.tlse != nullptr, a.tlse ? a.tlse[r] : 0.0, a.scale, w, &s);
    if (lane == 0) { loss[r] = (float)l; stat[r] = s; }
}

// ---- gradient ---------------------------------------------------------------------------------------------------
// exp2 of a probability's logarithm: its argument is computed in 64 bits
__device__ __forceinline__ float prob32(double x, const Log &l) {
    return x == kNegInfD ? 0.f : exp2_fast((float)(((x - l.big) - l.rest) * 1.4426950408889634));
}

// The gradients of the entries of [base, base + columns).
template <int TYPE, int T>
__device__ __forceinline__ void write_entries(const Row<TYPE> &row, const Entries &en, const Stat &s, double up, int64_t base, int64_t columns,
                                              typename Elem<TYPE>::T *out) {
    int64_t c;
    for (int64_t e = en.begin + threadIdx.x; e < en.end; e += T)
        if (en.at(e, &c) && c >= base && c < base + columns) {
            const double q = prob32(student(row, c, en.scale), s.lse), p = s.norm.none() ? 0.0 : (double)prob32(en.a(e), s.norm);
            out[c] = Elem<TYPE>::bits((float)(s.A != s.A ? s.A : up * (s.P * q - p)));
        }
}

// The dense pass of the gradient: g = A exp2(c2 (z - m)).
struct Dense {
    float A, m, c2, shift;
    bool plain;
    __device__ __forceinline__ Dense(const Stat &s, double up, float c2_) : m((float)s.m), c2(c2_), shift(m * c2_), plain(fabsf(shift) < 1e30f) {
        A = (float)(up * s.A);
        if (plain) A *= exp2_fast(-__builtin_fmaf(m, c2, -shift));
    }
    template <int N> __device__ __forceinline__ void of(const float *f, float *g) const {
        if (plain) {
#pragma unroll
            for (int k = 0; k < N; ++k) g[k] = A * exp2_fast(__builtin_fmaf(f[k], c2, -shift));
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) g[k] = A * exp2_fast((f[k] - m) * c2);
        }
    }
};

// Vector `first` .. of a row's gradient: as one where no place is marked.
template <int TYPE> __device__ __forceinline__ void write_vector(typename Elem<TYPE>::T *out, const float *g, uint32_t mk) {
    using E = Elem<TYPE>;
    if (mk == 0) {
        const uint4 n = E::narrow(g);
        typename Row<TYPE>::V4 q = {n.x, n.y, n.z, n.w};
        *(typename Row<TYPE>::V4 *)out = q;
    } else {
#pragma unroll
        for (int k = 0; k < E::kPer; ++k) if (!(mk >> k & 1)) out[k] = E::bits(g[k]);
    }
}

template <int TYPE, int T>
__device__ __forceinline__ void write_zeros(typename Elem<TYPE>::T *out, int64_t begin, int64_t end) {
    constexpr int P = Elem<TYPE>::kPer;
    const typename Row<TYPE>::V4 zero = {0, 0, 0, 0};
    const int64_t whole = (end - begin) / P * P;
    for (int64_t c = begin + threadIdx.x * P; c < begin + whole; c += T * P) *(typename Row<TYPE>::V4 *)(out + c) = zero;
    for (int64_t c = begin + whole + threadIdx.x; c < end; c += T) out[c] = 0;
}

// Vectors [piece * T * NV, ..) of a row, from its stat.
template <int TYPE, int T, int NV>
__global__ void __launch_bounds__(T) k_distill_backward(DistillArgs a, float c2, int count, const Stat *__restrict__ stat,
                                                        const float *__restrict__ dloss, void *dZ, int64_t lddz) {
    using E = Elem<TYPE>;
    constexpr int P = E::kPer;
    __shared__ uint32_t marks[T * NV * P / 32];
    const int64_t r = blockIdx.x / (unsigned)count;
    const int64_t v0 = (int64_t)(blockIdx.x - r * count) * T * NV, base = v0 * P;
    const float w = a.weight ? a.weight[r] : 1.f;
    typename E::T *out = (typename E::T *)dZ + r * lddz;
    if (w == 0) {
        write_zeros<TYPE, T>(out, base, base + T * NV * P < a.V ? base + T * NV * P : a.V);
        return;
    }
    const Row<TYPE> row(a.Z, r, a.ldz, a.V);
    const int64_t full = a.V / P;
    const int own = (int)(full - v0 < T * NV ? full - v0 : T * NV);
    uint4 v[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int i = j * T + threadIdx.x;
        v[j] = make_uint4(0, 0, 0, 0);
        if (i < own) v[j] = row.raw(v0 + i);
    }
    const Entries en(a, r);
    clear_marks<T>(marks, T * NV * P);
    set_marks<T>(marks, en, base, T * NV * P);
    const Stat s = stat[r];
    const double up = (double)w * a.scale * (dloss ? (double)dloss[r] : 1.0);
    write_entries<TYPE, T>(row, en, s, up, base, T * NV * P, out);
    __syncthreads();
    const Dense d(s, up, c2);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int i = j * T + threadIdx.x;
        if (i >= own) continue;
        float f[P], g[P];
        E::widen(v[j], f);
        d.of<P>(f, g);
        write_vector<TYPE>(out + (v0 + i) * P, g, marks_at<P>(marks, i));
    }
    if (a.V % P != 0 && full >= v0 && full < v0 + T * NV && threadIdx.x == 0) {
        float f[P], g[P];
        row.load(full, f);
        d.of<P>(f, g);
        const uint32_t mk = marks_at<P>(marks, (int)(full - v0));
        for (int k = 0; k < P; ++k) if (full * P + k < a.V && !(mk >> k & 1)) out[full * P + k] = E::bits(g[k]);
    }
}

// Loss and gradient of a row that a workgroup holds in registers: Z is read once.
template <int TYPE, int T, int NV, bool TAIL>
__global__ void __launch_bounds__(T, NV == 32 ? 2 : NV == 16 ? 3 : 4) k_distill_step(DistillArgs a, float c2, float *__restrict__ loss, void *dZ, int64_t lddz) {
    using E = Elem<TYPE>;
    constexpr int P = E::kPer;
    __shared__ uint32_t marks[T * NV * P / 32];
    __shared__ float2 buf[T / kWave];
    __shared__ Taught taught;
    const int64_t r = blockIdx.x;
    const float w = a.weight ? a.weight[r] : 1.f;
    typename E::T *out = (typename E::T *)dZ + r * lddz;
    if (w == 0) {
        write_zeros<TYPE, T>(out, 0, a.V);
        if (threadIdx.x == 0) loss[r] = 0;
        return;
    }
    const Row<TYPE> row(a.Z, r, a.ldz, a.V);
    const int full = (int)(a.V / P);
    const bool ends = a.V % P != 0;
    uint4 v[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int i = j * T + threadIdx.x;
        v[j] = make_uint4(E::kNone, E::kNone, E::kNone, E::kNone);
        if (i < full) v[j] = row.raw(i);
    }
    const Entries en(a, r);
    clear_marks<T>(marks, T * NV * P);
    set_marks<T>(marks, en, 0, T * NV * P);
    if (threadIdx.x >= T - kWave) {                              // one wavefront, while the row is on its way
        const Taught t = teach(row, en);
        if (threadIdx.x == T - 1) taught = t;
    }
    __syncthreads();
    Running run;
    constexpr int U = NV < 4 ? NV : 4;
#pragma unroll
    for (int j0 = 0; j0 < NV; j0 += U) {
        float b = kNegInf;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[P];
            E::widen(again(v[j0 + u]), f);
            if (TAIL) {
                const uint32_t mk = marks_at<P>(marks, (j0 + u) * T + threadIdx.x);
                if (mk) {
                    leave_out<P>(f, mk);
                    v[j0 + u] = E::narrow(f);
                }
            }
#pragma unroll
            for (int k = 0; k < P; ++k) b = fmaxf(b, f[k]);
        }
        run.raise(b, c2);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[P];
            E::widen(again(v[j0 + u]), f);
            run.template add<P>(f, c2);
        }
    }
    float last[P];                                               // the vector that the row ends in: thread 0's
    uint32_t last_marks = 0;
    if (ends && threadIdx.x == 0) {
        float f[P], b = kNegInf;
        row.load(full, f);
        last_marks = marks_at<P>(marks, full);
#pragma unroll
        for (int k = 0; k < P; ++k) last[k] = f[k];
        if (TAIL) leave_out<P>(f, last_marks);
#pragma unroll
        for (int k = 0; k < P; ++k) b = fmaxf(b, f[k]);
        run.template take<P>(f, b, c2);
    }
    MaxSum d = run.sum(c2);
    block_join<T>(d, c2, buf);
    const Taught t = taught;
    Stat s;
    const double l = finish(t, d, TAIL, TAIL ? a.tlse[r] : 0.0, a.scale, w, &s);
    if (threadIdx.x == 0) loss[r] = (float)l;
    const double up = (double)w * a.scale;
    write_entries<TYPE, T>(row, en, s, up, 0, a.V, out);
    const Dense g(s, up, c2);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int i = j * T + threadIdx.x;
        if (i >= full) continue;
        float f[P], o[P];
        E::widen(again(v[j]), f);
        g.of<P>(f, o);
        write_vector<TYPE>(out + (int64_t)i * P, o, marks_at<P>(marks, i));
    }
    if (ends && threadIdx.x == 0) {
        float o[P];
        g.of<P>(last, o);
        for (int k = 0; k < P; ++k) if ((int64_t)full * P + k < a.V && !(last_marks >> k & 1)) out[(int64_t)full * P + k] = E::bits(o[k]);
    }
}

int64_t vectors_of(int type, int64_t V) {
    const int64_t per = type == COMET_F32 ? 4 : 8;
    return (V + per - 1) / per;
}

// Pieces of the forward pass: as few as a row needs, more where the rows are too few for the device.
Pieces cut_forward(int type, int64_t N, int64_t V) {
    const int64_t nv = vectors_of(type, V);
    int64_t vectors = kPiece;
    while (vectors > 512 && N * ((nv + vectors - 1) / vectors) < 256) vectors /= 2;
    const int64_t count = nv > 0 ? (nv + vectors - 1) / vectors : 1;
    return Pieces{(int)(count == 1 ? (nv + 31) / 32 * 32 : vectors), (int)count};
}

int64_t round16(int64_t b) { return (b + 15) / 16 * 16; }
// the pieces' sums, behind the stat that the step keeps there
int64_t partial_bytes(const Pieces &c, int64_t N) { return c.count > 1 ? round16(N * c.count * (int64_t)sizeof(float2)) : 0; }

template <int TYPE> hipError_t forward(const DistillArgs &a, float c2, const Pieces &c, float *loss, Stat *stat, float2 *partial, hipStream_t st) {
    const size_t lds = a.tlse ? (size_t)c.vectors * Elem<TYPE>::kPer / 8 : 0;
    const auto kernel = a.tlse ? k_distill_forward<TYPE, true> : k_distill_forward<TYPE, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.N * c.count)), dim3(kThreads), lds, st, a, c2, c, loss, stat, partial);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || c.count == 1) return e;
    constexpr int rows = kThreads / kWave;
    hipLaunchKernelGGL(k_distill_finish<TYPE>, dim3((unsigned)((a.N + rows - 1) / rows)), dim3(kThreads), 0, st, a, c2, c.count, partial, loss, stat);
    return hipGetLastError();
}

template <int TYPE> hipError_t backward(const DistillArgs &a, float c2, const Stat *stat, const float *dloss, void *dZ, int64_t lddz, hipStream_t st) {
    const int64_t nv = vectors_of(TYPE, a.V);
    const bool big = a.N * ((nv + 2047) / 2048) >= 512;
    const int64_t piece = big ? 2048 : 512, count = (nv + piece - 1) / piece;
    const auto kernel = big ? k_distill_backward<TYPE, 256, 8> : k_distill_backward<TYPE, 256, 2>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.N * count)), dim3(256), 0, st, a, c2, (int)count, stat, dloss, dZ, lddz);
    return hipGetLastError();
}

template <int TYPE, int T, int NV> hipError_t launch_step(const DistillArgs &a, float c2, float *loss, void *dZ, int64_t lddz, hipStream_t st) {
    const auto kernel = a.tlse ? k_distill_step<TYPE, T, NV, true> : k_distill_step<TYPE, T, NV, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)a.N), dim3(T), 0, st, a, c2, loss, dZ, lddz);
    return hipGetLastError();
}
template <int TYPE> hipError_t step(const DistillArgs &a, float c2, float *loss, void *dZ, int64_t lddz, hipStream_t st) {
    const int64_t nv = vectors_of(TYPE, a.V);
    if (nv <= 256 * 4) return launch_step<TYPE, 256, 4>(a, c2, loss, dZ, lddz, st);
    if (nv <= 256 * 8) return launch_step<TYPE, 256, 8>(a, c2, loss, dZ, lddz, st);
    if (nv <= 256 * 16) return launch_step<TYPE, 256, 16>(a, c2, loss, dZ, lddz, st);
    if (nv <= 256 * 32) return launch_step<TYPE, 256, 32>(a, c2, loss, dZ, lddz, st);
    return launch_step<TYPE, 512, 32>(a, c2, loss, dZ, lddz, st);
}

float log2_scale(const DistillArgs &a) { return (float)(a.scale * 1.4426950408889634); }

}  // namespace

int64_t distill_work(int type, int64_t N, int64_t V) {
    return round16(N * (int64_t)sizeof(Stat)) + partial_bytes(cut_forward(type, N, V), N);
}

hipError_t distill_forward(const DistillArgs &a, float *loss, double *stat, void *work, hipStream_t st) {
    const float c2 = log2_scale(a);
    const Pieces c = cut_forward(a.type, a.N, a.V);
    float2 *partial = (float2 *)((char *)work + round16(a.N * (int64_t)sizeof(Stat)));
    return a.type == COMET_F32 ? forward<COMET_F32>(a, c2, c, loss, (Stat *)stat, partial, st)
         : a.type == COMET_BF16 ? forward<COMET_BF16>(a, c2, c, loss, (Stat *)stat, partial, st)
                                : forward<COMET_F16>(a, c2, c, loss, (Stat *)stat, partial, st);
}

hipError_t distill_backward(const DistillArgs &a, const double *stat, const float *dloss, void *dZ, int64_t lddz, hipStream_t st) {
    const float c2 = log2_scale(a);
    return a.type == COMET_F32 ? backward<COMET_F32>(a, c2, (const Stat *)stat, dloss, dZ, lddz, st)
         : a.type == COMET_BF16 ? backward<COMET_BF16>(a, c2, (const Stat *)stat, dloss, dZ, lddz, st)
                                : backward<COMET_F16>(a, c2, (const Stat *)stat, dloss, dZ, lddz, st);
}

hipError_t distill_step(const DistillArgs &a, float *loss, void *dZ, int64_t lddz, void *work, hipStream_t st) {
    const int64_t nv = vectors_of(a.type, a.V);
    if (nv <= 512 * 32 && (a.N >= 64 || nv <= 2048)) {
        const float c2 = log2_scale(a);
        return a.type == COMET_F32 ? step<COMET_F32>(a, c2, loss, dZ, lddz, st)
             : a.type == COMET_BF16 ? step<COMET_BF16>(a, c2, loss, dZ, lddz, st) : step<COMET_F16>(a, c2, loss, dZ, lddz, st);
    }
    const hipError_t e = distill_forward(a, loss, (double *)work, work, st);
    return e != hipSuccess || a.V == 0 ? e : distill_backward(a, (const double *)work, nullptr, dZ, lddz, st);
}

}  // namespace comet
