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
#include "rows.hpp"
#include "rows_kernels.hpp"

namespace comet {

namespace {

constexpr int kThreads = 256;
constexpr int kSpan = 32768;              // columns whose marks are in LDS at a time
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

// Loss of a row (times its weight) and what its gradient needs, by a whole workgroup, from the dense pass's maximum and sum.
template <int TYPE, int T>
__device__ double finish_row(const DistillArgs &a, int64_t r, const Row<TYPE> &row, const Entries &en, MaxSum d, double w, double *buf, Stat *out) {
    const bool tail = a.tlse != nullptr;
    int64_t c;
    const Log dense = log_sum(d, a.scale);
    // the teacher's normaliser
    Log norm{0.0, 0.0};
    if (tail) norm.big = a.tlse[r];
    else {
        double m = kNegInfD, s = 0;
        for (int64_t e = en.begin + threadIdx.x; e < en.end; e += T) if (en.at(e, &c)) m = Max()(m, en.a(e));
        m = block_reduce<T>(m, Max(), buf);
        if (m != kNegInfD) {                                     // the same for all threads
            for (int64_t e = en.begin + threadIdx.x; e < en.end; e += T) if (en.at(e, &c)) s += exp(en.a(e) - m);
            s = block_reduce<T>(s, Add(), buf);
        }
        norm = make_log(m, s);
    }
    // the student's
    Log lse = dense;
    if (tail) {
        double m = dense.value(), s = 0;
        for (int64_t e = en.begin + threadIdx.x; e < en.end; e += T) if (en.at(e, &c)) m = Max()(m, student(row, c, a.scale));
        m = block_reduce<T>(m, Max(), buf);
        if (m != kNegInfD) {
            for (int64_t e = en.begin + threadIdx.x; e < en.end; e += T) if (en.at(e, &c)) s += prob(student(row, c, a.scale), Log{m, 0.0});
            s = block_reduce<T>(s, Add(), buf);
            if (!dense.none()) s += exp((dense.big - m) + dense.rest);
        }
        lse = make_log(m, s);
    }
    const double outside = dense.none() ? kNegInfD : (dense.big - lse.big) + (dense.rest - lse.rest);      // log of the dense pass's share
    double mass = 0, loss = 0;
    if (!norm.none())                                            // else no entry has a probability
        for (int64_t e = en.begin + threadIdx.x; e < en.end; e += T)
            if (en.at(e, &c)) {
                const double p = prob(en.a(e), norm);
                mass += p;
                if (p != 0) loss += p * (minus(en.a(e), norm) - minus(student(row, c, a.scale), lse));
            }
    mass = block_reduce<T>(mass, Add(), buf);
    loss = block_reduce<T>(loss, Add(), buf);
    if (norm.big != norm.big) mass = norm.big;
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
    if (lse.big != lse.big || P != P) loss = out->A = lse.big + P;
    return w * loss;
}

// Marks the row's entries of [base, base + kSpan) in LDS.
template <int T> __device__ __forceinline__ void mark(uint32_t *marks, const Entries &en, int64_t base) {
    __syncthreads();
    for (int i = threadIdx.x; i < kSpan / 32; i += T) marks[i] = 0;
    __syncthreads();
    int64_t c;
    for (int64_t e = en.begin + threadIdx.x; e < en.end; e += T)
        if (en.at(e, &c) && c >= base && c < base + kSpan) atomicOr(&marks[(c - base) >> 5], 1u << ((c - base) & 31));
    __syncthreads();
}
// The marks of the N places from `c` on, a multiple of N.
template <int N> __device__ __forceinline__ uint32_t marks_at(const uint32_t *marks, int64_t c) {
    return marks[c >> 5] >> (c & 31) & ((1u << N) - 1);
}

template <int TYPE>
__global__ void __launch_bounds__(kThreads) k_distill_forward(DistillArgs a, float c2, float *__restrict__ loss, Stat *__restrict__ stat) {
    using E = Elem<TYPE>;
    __shared__ float2 buf[kThreads / kWave];
    __shared__ double dbuf[kThreads / kWave];
    __shared__ uint32_t marks[kSpan / 32];
    const int64_t r = blockIdx.x;
    const double w = a.weight ? a.weight[r] : 1.0;
    if (w == 0) { if (threadIdx.x == 0) loss[r] = 0; return; }
    const Row<TYPE> row(a.Z, r, a.ldz, a.V);
    const Entries en(a, r);
    Running run;
    const int64_t nv = row.nvec(), per = kSpan / E::kPer;
    for (int64_t v0 = 0; v0 < nv; v0 += per) {
        const int64_t base = row.first(v0);
        if (a.tlse) mark<kThreads>(marks, en, base);
        for (int64_t i = v0 + threadIdx.x; i < v0 + per && i < nv; i += kThreads) {
            float f[E::kPer];
            row.load(i, f);
            if (a.tlse) {
                const uint32_t m = marks_at<E::kPer>(marks, row.first(i) - base);
#pragma unroll
                for (int k = 0; k < E::kPer; ++k) if (m >> k & 1) f[k] = kNegInf;
            }
            float b = f[0];
#pragma unroll
            for (int k = 1; k < E::kPer; ++k) b = fmaxf(b, f[k]);
            run.take<E::kPer>(f, b, c2);
        }
    }
    MaxSum d = run.sum(c2);
    block_join<kThreads>(d, c2, buf);
    Stat s;
    const double l = finish_row<TYPE, kThreads>(a, r, row, en, d, w, dbuf, &s);
    if (threadIdx.x == 0) { loss[r] = (float)l; stat[r] = s; }
}

template <int TYPE>
__global__ void __launch_bounds__(kThreads) k_distill_backward(DistillArgs a, float c2, const Stat *__restrict__ stat,
                                                               const float *__restrict__ dloss, void *dZ, int64_t lddz) {
    using E = Elem<TYPE>;
    __shared__ uint32_t marks[kSpan / 32];
    const int64_t r = blockIdx.x;
    const double w = a.weight ? a.weight[r] : 1.0;
    const Row<TYPE> row(a.Z, r, a.ldz, a.V);
    typename E::T *out = (typename E::T *)dZ + r * lddz;
    if (w == 0) {
        for (int64_t c = threadIdx.x; c < a.V; c += kThreads) out[c] = 0;
        return;
    }
    const Entries en(a, r);
    const Stat s = stat[r];
    const double up = w * a.scale * (dloss ? (double)dloss[r] : 1.0);
    // the entries first: where dZ is Z their logits are still there, and the dense pass leaves marked places alone
    int64_t c;
    for (int64_t e = en.begin + threadIdx.x; e < en.end; e += kThreads)
        if (en.at(e, &c)) {
            const double q = prob(student(row, c, a.scale), s.lse), p = s.norm.none() ? 0.0 : prob(en.a(e), s.norm);
            out[c] = E::bits((float)(s.A != s.A ? s.A : up * (s.P * q - p)));
        }
    const float m = (float)s.m, A = (float)(up * s.A);
    const int64_t nv = row.nvec(), per = kSpan / E::kPer;
    for (int64_t v0 = 0; v0 < nv; v0 += per) {
        const int64_t base = row.first(v0);
        mark<kThreads>(marks, en, base);
        for (int64_t i = v0 + threadIdx.x; i < v0 + per && i < nv; i += kThreads) {
            float f[E::kPer];
            row.load(i, f);
            const int64_t c0 = row.first(i);
            const uint32_t mk = marks_at<E::kPer>(marks, c0 - base);
#pragma unroll
            for (int k = 0; k < E::kPer; ++k)
                if (c0 + k < a.V && !(mk >> k & 1)) out[c0 + k] = E::bits(A * exp2_fast((f[k] - m) * c2));
        }
    }
}

}  // namespace

int64_t distill_work(int, int64_t N, int64_t) { return N * (int64_t)sizeof(Stat); }

hipError_t distill_forward(const DistillArgs &a, float *loss, double *stat, void *, hipStream_t st) {
    const float c2 = (float)(a.scale * 1.4426950408889634);
    const auto kernel = a.type == COMET_F32 ? k_distill_forward<COMET_F32> : a.type == COMET_BF16 ? k_distill_forward<COMET_BF16> : k_distill_forward<COMET_F16>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)a.N), dim3(kThreads), 0, st, a, c2, loss, (Stat *)stat);
    return hipGetLastError();
}

hipError_t distill_backward(const DistillArgs &a, const double *stat, const float *dloss, void *dZ, int64_t lddz, hipStream_t st) {
    const float c2 = (float)(a.scale * 1.4426950408889634);
    const auto kernel = a.type == COMET_F32 ? k_distill_backward<COMET_F32> : a.type == COMET_BF16 ? k_distill_backward<COMET_BF16> : k_distill_backward<COMET_F16>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)a.N), dim3(kThreads), 0, st, a, c2, (const Stat *)stat, dloss, dZ, lddz);
    return hipGetLastError();
}

hipError_t distill_step(const DistillArgs &a, float *loss, void *dZ, int64_t lddz, void *work, hipStream_t st) {
    const hipError_t e = distill_forward(a, loss, (double *)work, nullptr, st);
    return e != hipSuccess || a.V == 0 ? e : distill_backward(a, (const double *)work, nullptr, dZ, lddz, st);
}

}  // namespace comet
