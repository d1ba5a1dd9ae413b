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

// What the entries alone give.  With ta and xa the largest of the a and of the x,
//   S = sum exp(a - ta),  D = sum exp(a - ta) ((a - ta) - (x - xa)),  X = sum exp(x - xa),
// norm the teacher's normaliser (ta + ln S, or tlse) and f = exp(ta - norm):
struct Taught {
    Log norm;
    double xa, X;
    double mass, rest;                    // f S, and what is missing to 1 where there is a tail
    double part;                          // the loss but for mass (lse - xa) - rest outside
};

// By one wavefront; the same in all its lanes.  A lane keeps its first entry.
template <int TYPE> __device__ Taught teach(const Row<TYPE> &row, const Entries &en, bool tail, double tlse) {
    const int lane = threadIdx.x & (kWave - 1);
    const int64_t e0 = en.begin + lane;
    int64_t c;
    double a0 = kNegInfD, x0 = kNegInfD, ta, xa, S = 0, D = 0, X = 0;
    const bool own = e0 < en.end && en.at(e0, &c);
    if (own) a0 = en.a(e0), x0 = student(row, c, en.scale);
    ta = a0, xa = x0;
    for (int64_t e = e0 + kWave; e < en.end; e += kWave)
        if (en.at(e, &c)) {
            ta = Max()(ta, en.a(e));
            xa = Max()(xa, student(row, c, en.scale));
        }
    ta = wave_reduce(ta, kNegInfD, Max());
    xa = wave_reduce(xa, kNegInfD, Max());
    const auto take = [&](double a, double x) {
        const double p = a == kNegInfD ? 0.0 : exp(a - ta);
        S += p;
        if (p != 0) D += p * ((a - ta) - (x == kNegInfD ? x : x - xa));
        X += x == kNegInfD ? 0.0 : exp(x - xa);
    };
    if (own) take(a0, x0);
    for (int64_t e = e0 + kWave; e < en.end; e += kWave)
        if (en.at(e, &c)) take(en.a(e), student(row, c, en.scale));
    S = wave_reduce(S, 0.0, Add());
    D = wave_reduce(D, 0.0, Add());
    X = wave_reduce(X, 0.0, Add());
    Taught t;
    const bool some = ta != kNegInfD;                            // an entry has a probability
    t.xa = xa, t.X = X;
    t.norm = tail ? Log{tlse, 0.0} : make_log(ta, S);
    const double f = !some ? 0.0 : tail ? exp(ta - tlse) : 1.0 / S;
    t.mass = tail ? f * S : some ? 1.0 : 0.0;
    if (t.norm.big != t.norm.big || S != S) t.mass = t.norm.big + S;            // NaN among the entries
    t.rest = tail ? 1.0 - t.mass : 0.0;
    if (t.rest < kNoTailBelow) t.rest = 0.0;
    t.part = 0;
    if (some) t.part = f * D + t.mass * ((ta - t.norm.big) - t.norm.rest);
    if (t.rest != 0) t.part += t.rest * log(t.rest);
    return t;
}

// Loss of a row (times its weight) and what its gradient needs, from the entries' sums and the dense pass's.
__device__ __forceinline__ double finish(const Taught &t, MaxSum d, bool tail, double scale, double w, Stat *out) {
    const double P = t.mass + t.rest, big = (double)d.m * scale;
    const bool none = d.m == kNegInf;                            // nothing is left for the dense pass
    Log lse;
    double tot = d.s, outside = 1;                               // sum of exp(x - lse.big), and of it the factor of the dense pass's sum
    lse.big = none ? kNegInfD : big;
    lse.rest = none ? 0.0 : log_of(d.s);
    double share = none ? kNegInfD : 0.0;                        // log of the dense pass's share
    if (tail && t.xa != kNegInfD) {
        const bool dense_first = !none && !(t.xa > big);
        const float other = none || t.xa != t.xa ? 0.f : exp2_fast((float)((dense_first ? t.xa - big : big - t.xa) * 1.4426950408889634));
        const double log_s = lse.rest;
        lse.big = dense_first ? big : t.xa;
        outside = dense_first ? 1.0 : (double)other;
        tot = t.X * (dense_first ? (double)other : 1.0) + outside * (none ? 0.0 : (double)d.s);
        lse.rest = log_of((float)tot);
        if (!none) share = (big - lse.big) + (log_s - lse.rest);
    }
    if (d.s != d.s) lse.big = d.s;
    double loss = t.part;
    if (t.mass != 0 && t.xa != kNegInfD) loss += t.mass * ((lse.big - t.xa) + lse.rest);
    if (t.rest != 0) loss -= t.rest * share;
    out->P = P;
    out->norm = t.norm;
    out->lse = lse;
    out->m = none ? 0.0 : (double)d.m;
    out->A = none ? 0.0 : tail ? P * outside / tot - t.rest / (double)d.s : P / (double)d.s;
    // NaN and +inf in the row, its entries, tlse or the weight
    if (lse.big + P != lse.big + P || lse.big == -kNegInfD || t.norm.big == -kNegInfD || w - w != 0) loss = out->A = __builtin_nan("");
    return w * loss;
}

// ---- marks --------------------------------------------------------------------------------------------------
// A piece of a row: `vectors` vectors from v0 on, vector j T + t of them thread t's j-th.  `own` of them are whole in the row; `ends` says that
// the row ends inside of the vector behind those.
template <int P> struct Piece {
    int64_t v0, vectors;
    int own;
    bool ends;
    __device__ __forceinline__ Piece(int64_t V, int64_t v0_, int64_t vectors_) : v0(v0_), vectors(vectors_) {
        const int64_t full = V / P;
        own = (int)(full - v0 < vectors ? full - v0 : vectors);                // below 1: none
        ends = V % P != 0 && full >= v0 && full < v0 + vectors;
    }
    __device__ __forceinline__ int64_t base() const { return v0 * P; }
    __device__ __forceinline__ int64_t columns() const { return vectors * P; }
};

// The places of the row's entries in a piece: a bit for each place (`bits`), and for each thread a word that names its vectors with such
// places (WORD has a bit for each of them).  Both are LDS.
template <int T, int P, class WORD> struct Marks {
    uint32_t *bits;
    WORD *words;
    __device__ __forceinline__ void clear(const Piece<P> &p) const {
        for (int i = threadIdx.x; i < (int)((p.columns() + 31) / 32); i += T) bits[i] = 0;
        words[threadIdx.x] = 0;
        lds_barrier();
    }
    // By `threads` threads, of which this is `thread`; a barrier has to follow.
    __device__ __forceinline__ void set(const Piece<P> &p, const Entries &en, int thread = threadIdx.x, int threads = T) const {
        int64_t c;
        for (int64_t e = en.begin + thread; e < en.end; e += threads)
            if (en.at(e, &c) && c >= p.base() && c < p.base() + p.columns()) {
                const int at = (int)(c - p.base()), i = at / P;
                atomicOr(&bits[at >> 5], 1u << (at & 31));
                atomicOr(&words[i % T], (WORD)1 << (i / T));
            }
    }
    __device__ __forceinline__ uint32_t of(int i) const {                                        // the marks of the piece's vector i
        const int c = i * P;
        return bits[c >> 5] >> (c & 31) & ((1u << P) - 1);
    }
    __device__ __forceinline__ bool at(int c) const { return bits[c >> 5] >> (c & 31) & 1; }
};

// The bit of the vector that the row ends in, for its thread.
template <int T, int P, class WORD> __device__ __forceinline__ WORD last_vector(const Piece<P> &p) {
    return p.ends && (int)threadIdx.x == p.own % T ? (WORD)1 << (p.own / T) : (WORD)0;
}

// The words of a piece of NV vectors a thread.
template <int NV> struct WordOf { using type = uint32_t; };
template <> struct WordOf<40> { using type = uint64_t; };

__device__ __forceinline__ int lowest(uint32_t w) { return __builtin_ctz(w); }
__device__ __forceinline__ int lowest(uint64_t w) { return __builtin_ctzll(w); }

// Takes in the vectors that `word` names, without the marked places where there is a tail.
template <int TYPE, int T, bool TAIL, class WORD>
__device__ __forceinline__ void take_some(Running &run, const Row<TYPE> &row, const Piece<Elem<TYPE>::kPer> &p, WORD word,
                                          const Marks<T, Elem<TYPE>::kPer, WORD> &marks, float c2) {
    constexpr int P = Elem<TYPE>::kPer;
    while (word) {
        const int i = lowest(word) * T + threadIdx.x;
        word &= word - 1;
        float f[P], b = kNegInf;
        row.load(p.v0 + i, f);
        const uint32_t mk = TAIL ? marks.of(i) : 0;
#pragma unroll
        for (int k = 0; k < P; ++k) {
            if (TAIL && mk >> k & 1) f[k] = kNegInf;
            b = fmaxf(b, f[k]);
        }
        run.template take<P>(f, b, c2);
    }
}

// ---- forward --------------------------------------------------------------------------------------------------
constexpr int kThreads = 256;
constexpr int kPiece = 64 * kThreads;     // vectors of a piece at most: a bit for each of a thread's, and marks of 16 KB
constexpr int kAhead = 4;                 // vectors that a thread has in flight

struct Pieces {                           // how a row is cut: `count` pieces of `vectors` vectors
    int vectors, count;
};

// Reads a piece once: the running maximum and sum of its places, without the marked ones where there is a tail.  Vectors with marks, and the
// one that the row ends in, are read again at the end, in part.  `mark` sets the marks, once the first loads are on their way.
template <int TYPE, int T, bool TAIL, class WORD, class MARK>
__device__ __forceinline__ MaxSum read_piece(const Row<TYPE> &row, const Piece<Elem<TYPE>::kPer> &p, const Marks<T, Elem<TYPE>::kPer, WORD> &marks,
                                             float c2, bool once, float2 *buf, MARK mark) {
    using E = Elem<TYPE>;
    constexpr int P = E::kPer, U = kAhead;
    uint4 v[U];
    auto fetch = [&](int i0) {
        if (i0 + U * T <= p.own && once) {
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = row.template stream<true>(p.v0 + i0 + u * T + threadIdx.x);
        } else if (i0 + U * T <= p.own) {
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = row.template stream<false>(p.v0 + i0 + u * T + threadIdx.x);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * T + threadIdx.x;
                v[u] = make_uint4(E::kNone, E::kNone, E::kNone, E::kNone);
                if (i < p.own) v[u] = row.template stream<false>(p.v0 + i);
            }
        }
    };
    const auto edge = row.template edges<T>(p.v0, p.own);
    fetch(0);
    mark();
    WORD word = TAIL ? marks.words[threadIdx.x] : (WORD)0;
    Running run;
    for (int i0 = 0, j0 = 0; i0 < p.own; i0 += U * T, j0 += U) {
        uint4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = v[u];
        if (i0 + U * T < p.own) fetch(i0 + U * T);
        if (row.odd) {
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = row.settle(x[u], edge, j0 + u, i0 + u * T + threadIdx.x, p.own);
        }
        if (TAIL && (word >> j0 & ((1 << U) - 1))) {
#pragma unroll
            for (int u = 0; u < U; ++u) if (word >> (j0 + u) & 1) x[u] = make_uint4(E::kNone, E::kNone, E::kNone, E::kNone);
        }
        float f[U * P], b = kNegInf;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            E::widen(x[u], f + u * P);
#pragma unroll
            for (int k = 0; k < P; ++k) b = fmaxf(b, f[u * P + k]);
        }
        run.template take<U * P>(f, b, c2);
    }
    take_some<TYPE, T, TAIL>(run, row, p, word | last_vector<T, P, WORD>(p), marks, c2);
    MaxSum d = run.sum(c2);
    block_join<T>(d, c2, buf);
    if (wild(d.m, c2))
        d.s = slow_sum<TYPE, T>(row, p.base(), p.base() + p.columns(), d.m, c2, buf, [&](int64_t c) { return TAIL && marks.at((int)(c - p.base())); });
    return d;
}

// One workgroup a row or a piece of one, four vectors a thread under way while four are taken in.  Bound by memory where rows are long and many
// (4096 x 131072 of 16 bits in 173 us: 6.2 TB/s) and by the exponentials and their additions where they are shorter: 2048 x 50021 of 16 bits
// 48 us in the kernel, 29 for its bytes alone at 7.1 TB/s.
template <int TYPE, bool TAIL>
__global__ void __launch_bounds__(kThreads) k_distill_forward(DistillArgs a, float c2, Pieces cut, float *__restrict__ loss, Stat *__restrict__ stat,
                                                              float2 *__restrict__ partial) {
    using E = Elem<TYPE>;
    constexpr int P = E::kPer, T = kThreads;
    __shared__ float2 buf[T / kWave];
    __shared__ uint64_t words[TAIL ? T : 1];
    __shared__ Taught taught;
    extern __shared__ uint32_t bits[];
    const int64_t r = blockIdx.x / (unsigned)cut.count;
    const float w = a.weight ? a.weight[r] : 1.f;
    if (w == 0) {
        if (threadIdx.x == 0 && cut.count == 1) loss[r] = 0;
        return;
    }
    const Row<TYPE> row(a.Z, r, a.ldz, a.V, a.shift);
    const Piece<P> p(a.V, (blockIdx.x - r * cut.count) * cut.vectors, cut.vectors);
    const Marks<T, P, uint64_t> marks{bits, words};
    // The last wavefront goes through the entries of a long row before it reads its part of it, while the others' parts keep the memory busy; of
    // a short one, when the row has been read (4096 rows of 8000 elements of 16 bits: 28 us so, 32 the other way; 2048 of 50021: 51 and 49).
    const bool teacher = cut.count == 1 && threadIdx.x >= T - kWave, early = p.own > 16 * T;
    const auto learn = [&] {
        const Taught t = teach(row, Entries(a, r), TAIL, TAIL ? a.tlse[r] : 0.0);
        if (threadIdx.x == T - 1) taught = t;
    };
    const MaxSum d = read_piece<TYPE, T, TAIL>(row, p, marks, c2, a.once, buf, [&] {
        if (TAIL) {
            marks.clear(p);
            marks.set(p, Entries(a, r));
            lds_barrier();
        }
        if (teacher && early) learn();
    });
    if (cut.count > 1) {
        if (threadIdx.x == 0) partial[blockIdx.x] = make_float2(d.m, d.s);
    } else if (teacher) {
        if (!early) learn();
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        Stat s;
        const double l = finish(taught, d, TAIL, a.scale, w, &s);
        if (threadIdx.x == T - 1) { loss[r] = (float)l; stat[r] = s; }
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
    const Taught t = teach(row, Entries(a, r), a.tlse != nullptr, a.tlse ? a.tlse[r] : 0.0);
    wave_join(d, c2);
    Stat s;
    const double l = finish(t, d, a.tlse != nullptr, a.scale, w, &s);
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

// The dense pass of the gradient: g = A exp2(c2 (z - m)), with one multiply-add, one exp2 and one product an element.  What rounding c2 m does
// to the exponentials is put into A: a factor of 2^16 at most below kFlat, which leaves every A a number that has one to round to.  Rows beyond
// it (masked throughout by -4e8 or less) are computed from z - m.
constexpr float kFlat = 0x1p29f;
struct Dense {
    float A, m, c2, shift;
    __device__ __forceinline__ Dense(const Stat &s, double up, float c2_) : A((float)(up * s.A)), m((float)s.m), c2(c2_), shift(m * c2_) {
        if (plain()) A *= exp2_fast(-__builtin_fmaf(m, c2, -shift));
    }
    __device__ __forceinline__ bool plain() const { return fabsf(shift) < kFlat; }
    __device__ __forceinline__ float of(float z) const { return A * exp2_fast(__builtin_fmaf(z, c2, -shift)); }        // where plain()
    __device__ __forceinline__ float slow(float z) const { return A * exp2_fast(plain() ? __builtin_fmaf(z, c2, -shift) : (z - m) * c2); }
};

// Vector i of the gradient element by element: those that are in the row and not marked.
template <int TYPE> __device__ __forceinline__ void write_some(const Row<TYPE> &row, int64_t i, const Dense &d, uint32_t mk, typename Elem<TYPE>::T *out) {
    constexpr int P = Elem<TYPE>::kPer;
    float f[P];
    row.load(i, f);
#pragma unroll
    for (int k = 0; k < P; ++k)
        if (i * P + k < row.n && !(mk >> k & 1)) out[i * P + k] = Elem<TYPE>::bits(d.slow(f[k]));
}

// A piece of the gradient, whose logits v[] holds.  The few vectors with marked places and the one that the row ends in are read again and written
// one element after the other.  So are, as vectors, those of a row that is not plain(), in a loop of its own: 4096 such rows of 131072 elements of
// 16 bits 379 us, 352 of plain ones; both computations in one loop over the registers took 358 for plain rows, and the step 620 for 455.
template <int TYPE, int T, int NV, class WORD>
__device__ __forceinline__ void write_piece(const Row<TYPE> &row, const uint4 (&v)[NV], const Piece<Elem<TYPE>::kPer> &p, const Dense &d,
                                            const Marks<T, Elem<TYPE>::kPer, WORD> &marks, typename Elem<TYPE>::T *out) {
    using E = Elem<TYPE>;
    constexpr int P = E::kPer;
    static_assert(NV <= 8 * sizeof(WORD), "a bit for each");
    const int n = p.own > (int)threadIdx.x ? (p.own - (int)threadIdx.x + T - 1) / T : 0;        // this thread's whole vectors
    const WORD whole = n >= 8 * (int)sizeof(WORD) ? ~(WORD)0 : ((WORD)1 << n) - 1;
    WORD left = marks.words[threadIdx.x] & whole;
    WORD now = whole & ~left;
    left |= last_vector<T, P, WORD>(p);
    const auto put = [&](const float *f, int64_t i0) {           // the vectors i0 + threadIdx.x of the piece
        const uint4 q = E::narrow(f);
        const typename Row<TYPE>::V4 q4 = {q.x, q.y, q.z, q.w};
        __builtin_nontemporal_store(q4, (typename Row<TYPE>::V4 *)(out + p.base() + i0 * P) + threadIdx.x);
    };
    if (d.plain()) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (now >> j & 1) {
                float f[P];
                E::widen(again(v[j]), f);
#pragma unroll
                for (int k = 0; k < P; ++k) f[k] = d.of(f[k]);
                put(f, j * T);
            }
    } else {
        while (now) {
            const int i0 = lowest(now) * T;
            now &= now - 1;
            float f[P];
            E::widen(row.raw(p.v0 + i0 + threadIdx.x), f);
#pragma unroll
            for (int k = 0; k < P; ++k) f[k] = d.slow(f[k]);
            put(f, i0);
        }
    }
    while (left) {
        const int i = lowest(left) * T + threadIdx.x;
        left &= left - 1;
        write_some(row, p.v0 + i, d, marks.of(i), out);
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

// Loads a piece into registers; nothing where the row has ended.
template <int TYPE, int T, int NV> __device__ __forceinline__ void hold(const Row<TYPE> &row, const Piece<Elem<TYPE>::kPer> &p, uint4 (&v)[NV]) {
    using E = Elem<TYPE>;
    using V4 = typename Row<TYPE>::V4;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const V4 *at = (const V4 *)(row.p + (p.v0 + j * T) * E::kPer - (row.odd ? 1 : 0));         // one address for all threads
        V4 x = {E::kNone, E::kNone, E::kNone, E::kNone};
        if ((j + 1) * T <= p.own || j * T + (int)threadIdx.x < p.own) x = at[threadIdx.x];
        v[j] = make_uint4(x.x, x.y, x.z, x.w);
    }
}

// Vectors [piece * T * NV, ..) of a row, from its stat.  Bound by memory, half of it stores, which go past the caches: nobody in the call reads
// them again.  4096 x 131072 of 16 bits, 2.1 GB read and written, 350 us (6.1 TB/s); pieces of 1024 vectors, and of 512 where those would be
// fewer than two workgroups a compute unit.  Rows of odd 16-bit elements are stored as they lie: shifted to whole words like their loads, with
// single elements at the ends of wavefronts, 2048 x 50021 took 82 us and not 79.
template <int TYPE, int T, int NV>
__global__ void __launch_bounds__(T) k_distill_backward(DistillArgs a, float c2, int count, const Stat *__restrict__ stat,
                                                        const float *__restrict__ dloss, void *dZ, int64_t lddz) {
    using E = Elem<TYPE>;
    constexpr int P = E::kPer;
    __shared__ uint32_t bits[T * NV * P / 32], words[T];
    const int64_t r = blockIdx.x / (unsigned)count;
    const Piece<P> p(a.V, (blockIdx.x - r * count) * T * NV, T * NV);
    const float w = a.weight ? a.weight[r] : 1.f;
    typename E::T *out = (typename E::T *)dZ + r * lddz;
    if (w == 0) {
        write_zeros<TYPE, T>(out, p.base(), p.base() + p.columns() < a.V ? p.base() + p.columns() : a.V);
        return;
    }
    const Row<TYPE> row(a.Z, r, a.ldz, a.V, a.shift);
    const Marks<T, P, uint32_t> marks{bits, words};
    uint4 v[NV];
    const auto edge = row.template edges<T>(p.v0, p.own);
    hold<TYPE, T>(row, p, v);
    const Entries en(a, r);
    marks.clear(p);
    marks.set(p, en);
    const Stat s = stat[r];
    const double up = (double)w * a.scale * (dloss ? (double)dloss[r] : 1.0);
    write_entries<TYPE, T>(row, en, s, up, p.base(), p.columns(), out);
    lds_barrier();
    if (row.odd) {
#pragma unroll
        for (int j = 0; j < NV; ++j) v[j] = row.settle(v[j], edge, j, j * T + threadIdx.x, p.own);
    }
    write_piece<TYPE, T>(row, v, p, Dense(s, up, c2), marks, out);
}

// Loss and gradient of a row that a workgroup holds in registers: Z is read once and dZ written once, where the two calls read Z twice.  Bound
// by memory, and for rows of more than 8192 vectors by there being one workgroup a compute unit: 160 KB to 320 KB of its 512 KB of registers
// are the row, so that one row's loads, sums and stores follow each other.  4096 x 131072 of 16 bits with a quarter of its rows ignored, 1.88 GB, 420 us
// (4.5 TB/s; a copy of that size by the same kind of loop 6.2); of 24001 107 us (3.7 TB/s).  Going from row to row in one workgroup, the next row's loads
// before the stores of the last, was no faster (425).  Three wavefronts a SIMD with a few registers spilled are better than two without (2048 x
// 50016: 100 us and 117).
template <int TYPE, int T, int NV, bool TAIL>
__global__ void __launch_bounds__(T, T == 512 ? 2 : NV >= 16 ? 3 : 4) k_distill_step(DistillArgs a, float c2, float *__restrict__ loss, void *dZ, int64_t lddz) {
    using E = Elem<TYPE>;
    constexpr int P = E::kPer, U = NV < 4 ? NV : 4;
    using WORD = typename WordOf<NV>::type;
    __shared__ uint32_t bits[T * NV * P / 32];
    __shared__ WORD words[T];
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
    const Row<TYPE> row(a.Z, r, a.ldz, a.V, a.shift);
    const Piece<P> p(a.V, 0, T * NV);
    const Marks<T, P, WORD> marks{bits, words};
    const Entries en(a, r);
    uint4 v[NV];
    // A wavefront's loads come back in their order.  Of a long row the last wavefront goes through the entries before it asks for its part, while
    // the others' parts keep the memory busy (4096 x 131072 of 16 bits: 450 us after it, 412 before it); of a short one all parts first.
    constexpr bool kLong = NV >= 16;
    const bool teacher = threadIdx.x >= T - kWave;
    if (!kLong) hold<TYPE, T>(row, p, v);
    marks.clear(p);
    if (teacher) {
        if (kLong) marks.set(p, en, threadIdx.x - (T - kWave), kWave);
        else marks.set(p, en);
        const Taught t = teach(row, en, TAIL, TAIL ? a.tlse[r] : 0.0);
        if (threadIdx.x == T - 1) taught = t;
    } else if (!kLong) marks.set(p, en);
    const auto edge = row.template edges<T>(0, p.own);
    if (kLong) hold<TYPE, T>(row, p, v);
    lds_barrier();
    Running run;
    const WORD word = TAIL ? words[threadIdx.x] : 0;
#pragma unroll
    for (int j0 = 0; j0 < NV; j0 += U) {
        if (j0 * T >= p.own) continue;                           // the row has ended
        if (row.odd) {
#pragma unroll
            for (int u = 0; u < U; ++u) v[j0 + u] = row.settle(v[j0 + u], edge, j0 + u, (j0 + u) * T + threadIdx.x, p.own);
        }
        float f[U * P], b = kNegInf;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (TAIL && (word >> (j0 + u) & 1)) v[j0 + u] = make_uint4(E::kNone, E::kNone, E::kNone, E::kNone);
            E::widen(v[j0 + u], f + u * P);
#pragma unroll
            for (int k = 0; k < P; ++k) b = fmaxf(b, f[u * P + k]);
        }
        run.template take<U * P>(f, b, c2);
        __builtin_amdgcn_sched_barrier(0);
    }
    take_some<TYPE, T, TAIL>(run, row, p, word | last_vector<T, P, WORD>(p), marks, c2);
    MaxSum d = run.sum(c2);
    block_join<T>(d, c2, buf);
    if (wild(d.m, c2)) d.s = slow_sum<TYPE, T>(row, 0, a.V, d.m, c2, buf, [&](int64_t c) { return TAIL && marks.at((int)c); });
    const Taught t = taught;
    Stat s;
    const double l = finish(t, d, TAIL, a.scale, w, &s);
    if (threadIdx.x == 0) loss[r] = (float)l;
    const double up = (double)w * a.scale;
    write_entries<TYPE, T>(row, en, s, up, 0, a.V, out);
    write_piece<TYPE, T>(row, v, p, Dense(s, up, c2), marks, out);
}

int64_t vectors_of(int type, int64_t V) {
    const int64_t per = type == COMET_F32 ? 4 : 8;
    return (V + per - 1) / per;
}

// Pieces of the forward pass: as few as a row needs, more where long rows are too few for the device: a second launch joins them, and
// costs more than a row of 8192 vectors takes one workgroup.
Pieces cut_forward(int type, int64_t N, int64_t V) {
    const int64_t nv = vectors_of(type, V);
    int64_t vectors = kPiece;
    if (nv > 8192)
        while (vectors > 512 && N * ((nv + vectors - 1) / vectors) < 256) vectors /= 2;
    const int64_t count = nv > 0 ? (nv + vectors - 1) / vectors : 1;
    return Pieces{(int)(((nv + count - 1) / count + 31) / 32 * 32), (int)count};           // of one length
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

// The call's rows from r0 on, n of them.
template <int TYPE> DistillArgs rows_from(const DistillArgs &a, int64_t r0, int64_t n) {
    DistillArgs b = a;
    b.Z = (const typename Elem<TYPE>::T *)a.Z + r0 * a.ldz;
    b.N = n;
    if (a.pos) b.pos += r0;
    else b.crd += r0 * a.K, b.tvals += r0 * a.K;
    if (a.tlse) b.tlse += r0;
    if (a.weight) b.weight += r0;
    return b;
}

template <int TYPE> hipError_t backward(const DistillArgs &a, float c2, const Stat *stat, const float *dloss, void *dZ, int64_t lddz, hipStream_t st) {
    const int64_t nv = vectors_of(TYPE, a.V);
    const bool big = a.N * ((nv + 1023) / 1024) >= 512;
    const int64_t piece = big ? 1024 : 512, count = (nv + piece - 1) / piece;
    const auto kernel = big ? k_distill_backward<TYPE, 256, 4> : k_distill_backward<TYPE, 256, 2>;
    const int64_t most = ((int64_t(1) << 24) - 1) / count;       // a launch has fewer than 2^32 threads
    for (int64_t r0 = 0; r0 < a.N; r0 += most) {
        const int64_t n = a.N - r0 < most ? a.N - r0 : most;
        hipLaunchKernelGGL(kernel, dim3((unsigned)(n * count)), dim3(256), 0, st, rows_from<TYPE>(a, r0, n), c2, (int)count, stat + r0,
                           dloss ? dloss + r0 : nullptr, (typename Elem<TYPE>::T *)dZ + r0 * lddz, lddz);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
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
    if (nv <= 512 * 32) return launch_step<TYPE, 512, 32>(a, c2, loss, dZ, lddz, st);
    return launch_step<TYPE, 512, 40>(a, c2, loss, dZ, lddz, st);
}

float log2_scale(const DistillArgs &a) { return (float)(a.scale * 1.4426950408889634); }

}  // namespace

// Whether a step holds its rows in registers; else it is the two calls, with the stat between them.  A row of more than 8192 vectors takes a
// compute unit to itself, so that it is not read while the one before it is computed on: 4096 rows of 66000 elements of 16 bits 321 us, the two
// calls 298; of 81920 334 and 347, of 131072 462 and 545, of 151936 554 and 644.
static bool held(int type, int64_t N, int64_t V) {
    const int64_t nv = vectors_of(type, V);
    return nv <= 256 * 32 || (N >= 64 && nv > 10240 && nv <= 512 * 40);
}
static int64_t stat_bytes(int type, int64_t N, int64_t V) { return held(type, N, V) ? 0 : round16(N * (int64_t)sizeof(Stat)); }

int64_t distill_work(int type, int64_t N, int64_t V) { return stat_bytes(type, N, V) + partial_bytes(cut_forward(type, N, V), N); }

hipError_t distill_forward(const DistillArgs &given, float *loss, double *stat, void *work, hipStream_t st) {
    DistillArgs a = given;
    a.once = read_once(a.type, a.N, a.V), a.shift = read_shifted(a.type, a.N, a.V);
    const float c2 = log2_scale(a);
    const Pieces c = cut_forward(a.type, a.N, a.V);
    float2 *partial = (float2 *)((char *)work + stat_bytes(a.type, a.N, a.V));
    return a.type == COMET_F32 ? forward<COMET_F32>(a, c2, c, loss, (Stat *)stat, partial, st)
         : a.type == COMET_BF16 ? forward<COMET_BF16>(a, c2, c, loss, (Stat *)stat, partial, st)
                                : forward<COMET_F16>(a, c2, c, loss, (Stat *)stat, partial, st);
}

hipError_t distill_backward(const DistillArgs &given, const double *stat, const float *dloss, void *dZ, int64_t lddz, hipStream_t st) {
    DistillArgs a = given;
    a.shift = read_shifted(a.type, a.N, a.V);
    const float c2 = log2_scale(a);
    return a.type == COMET_F32 ? backward<COMET_F32>(a, c2, (const Stat *)stat, dloss, dZ, lddz, st)
         : a.type == COMET_BF16 ? backward<COMET_BF16>(a, c2, (const Stat *)stat, dloss, dZ, lddz, st)
                                : backward<COMET_F16>(a, c2, (const Stat *)stat, dloss, dZ, lddz, st);
}

hipError_t distill_step(const DistillArgs &given, float *loss, void *dZ, int64_t lddz, void *work, hipStream_t st) {
    DistillArgs a = given;
    a.shift = read_shifted(a.type, a.N, a.V);
    if (held(a.type, a.N, a.V)) {
        const float c2 = log2_scale(a);
        return a.type == COMET_F32 ? step<COMET_F32>(a, c2, loss, dZ, lddz, st)
             : a.type == COMET_BF16 ? step<COMET_BF16>(a, c2, loss, dZ, lddz, st) : step<COMET_F16>(a, c2, loss, dZ, lddz, st);
    }
    const hipError_t e = distill_forward(a, loss, (double *)work, work, st);
    return e != hipSuccess || a.V == 0 ? e : distill_backward(a, (const double *)work, nullptr, dZ, lddz, st);
}

}  // namespace comet
