// Beam search: selection over beams and vocabulary, and the reordering of the beams' states.
#include "rows.hpp"
#include "rows_kernels.hpp"

namespace comet {

namespace {

constexpr int kThreads = 256;

// One workgroup a batch: the n best of the W lists of n keys (each in order), by counting.
__global__ void __launch_bounds__(kThreads) k_beam_merge(const uint64_t *__restrict__ keys, const Log *__restrict__ logs,
                                                         const float *__restrict__ score, int W, int n, float *__restrict__ out_score,
                                                         int32_t *__restrict__ out_parent, int32_t *__restrict__ out_token) {
    __shared__ double big[COMET_MAX_BEAMS], off[COMET_MAX_BEAMS];       // a candidate's score is (z - big) + off
    const int64_t b = blockIdx.x;
    for (int w = threadIdx.x; w < W; w += kThreads) {
        big[w] = logs[b * W + w].big;
        off[w] = (double)score[b * W + w] - logs[b * W + w].rest;
    }
    for (int i = threadIdx.x; i < n; i += kThreads) {
        out_score[b * n + i] = kNegInf;
        out_parent[b * n + i] = -1;
        out_token[b * n + i] = -1;
    }
    __syncthreads();
    const uint64_t *k = keys + b * W * n;
    const int total = W * n;
    for (int i = threadIdx.x; i < total; i += kThreads) {
        const double s = ((double)value_of_key(k[i]) - big[i / n]) + off[i / n];
        if (k[i] == 0 || !(s > kNegInfD)) continue;
        int at = 0;
        for (int j = 0; j < total && at < n; ++j) {
            const double t = ((double)value_of_key(k[j]) - big[j / n]) + off[j / n];
            at += k[j] != 0 && (t > s || (t == s && j < i));
        }
        if (at >= n) continue;
        out_score[b * n + at] = (float)s;
        out_parent[b * n + at] = i / n;
        out_token[b * n + at] = (int32_t)column_of(k[i]);
    }
}

constexpr int kStates = 64;               // state arrays of one launch
struct StatePointers { char *p[kStates]; };

// A thread moves the same unit of all beams of a batch: all are read into LDS before the first is written.
template <class U>
__global__ void __launch_bounds__(kThreads) k_beam_reorder(StatePointers states, StateLayout l, const int32_t *__restrict__ parent) {
    extern __shared__ __align__(16) char raw[];
    U *tile = (U *)raw + threadIdx.x;
    const int W = (int)l.W, T = blockDim.x;
    const int64_t b = blockIdx.y, units = l.inner / (int64_t)sizeof(U), all = units * l.outer;
    char *base = states.p[blockIdx.z] + b * l.batch_stride;
    const int32_t *par = parent + b * W;
    for (int64_t u = (int64_t)blockIdx.x * T + threadIdx.x; u < all; u += (int64_t)gridDim.x * T) {
        const int64_t o = u / units;
        char *at = base + o * l.outer_stride + (u - o * units) * (int64_t)sizeof(U);
        for (int w = 0; w < W; ++w) {
            const int p = par[w];
            if (p >= 0 && p < W && p != w) tile[w * T] = *(const U *)(at + p * l.beam_stride);
        }
        for (int w = 0; w < W; ++w) {
            const int p = par[w];
            if (p >= 0 && p < W && p != w) *(U *)(at + w * l.beam_stride) = tile[w * T];
        }
    }
}

}  // namespace

int64_t beam_select_work(int type, int64_t B, int64_t W, int64_t V, int64_t n) {
    return (B * W * (n * (int64_t)sizeof(uint64_t) + (int64_t)sizeof(Log)) + 15) / 16 * 16 + rows_top_keys_work(type, B * W, V, n);
}

hipError_t beam_select(const void *Z, int type, int64_t B, int64_t W, int64_t V, int64_t ldz, const float *score, const uint8_t *finished,
                       int32_t eos, int64_t n, float *out_score, int32_t *out_parent, int32_t *out_token, void *work, hipStream_t st) {
    Log *lse = (Log *)work;
    uint64_t *keys = (uint64_t *)(lse + B * W);
    const hipError_t e = rows_top_keys(Z, type, B * W, V, ldz, n, finished, eos, keys, lse,
                                     (char *)work + (B * W * (n * (int64_t)sizeof(uint64_t) + (int64_t)sizeof(Log)) + 15) / 16 * 16, st);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_beam_merge, dim3((unsigned)B), dim3(kThreads), 0, st, keys, lse, score, (int)W, (int)n, out_score, out_parent, out_token);
    return hipGetLastError();
}

hipError_t beam_reorder(void *const *states, int64_t nstates, const StateLayout &l, const int32_t *parent, hipStream_t st) {
    // the widest unit that divides every address and length
    uint64_t all = (uint64_t)l.inner;
    if (l.B > 1) all |= (uint64_t)l.batch_stride;
    if (l.W > 1) all |= (uint64_t)l.beam_stride;
    if (l.outer > 1) all |= (uint64_t)l.outer_stride;
    for (int64_t i = 0; i < nstates; ++i) all |= (uint64_t)(uintptr_t)states[i];
    int unit = all & 1 ? 1 : all & 2 ? 2 : all & 4 ? 4 : all & 8 ? 8 : 16;
    while (kWave * unit * l.W > 65536) unit /= 2;            // one wavefront's tile fits into LDS: 4 bytes at 256 beams
    const auto kernel = unit == 16 ? k_beam_reorder<uint4> : unit == 8 ? k_beam_reorder<uint2> : unit == 4 ? k_beam_reorder<uint32_t>
                      : unit == 2 ? k_beam_reorder<uint16_t> : k_beam_reorder<uint8_t>;
    int threads = kThreads;
    while (threads > kWave && threads * unit * l.W > 65536) threads /= 2;
    const int64_t lds = (int64_t)threads * unit * l.W;
    const int64_t units = l.inner / unit * l.outer;
    int64_t gx = (units + threads - 1) / threads;
    if (gx > 65536) gx = 65536;
    for (int64_t s0 = 0; s0 < nstates; s0 += kStates)
        for (int64_t b0 = 0; b0 < l.B; b0 += 65535) {
            StatePointers sp{};
            const int64_t ns = nstates - s0 < kStates ? nstates - s0 : kStates, nb = l.B - b0 < 65535 ? l.B - b0 : 65535;
            for (int64_t i = 0; i < ns; ++i) sp.p[i] = (char *)states[s0 + i] + b0 * l.batch_stride;
            hipLaunchKernelGGL(kernel, dim3((unsigned)gx, (unsigned)nb, (unsigned)ns), dim3(threads), (size_t)lds, st, sp, l, parent + b0 * l.W);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    return hipSuccess;
}

}  // namespace comet
