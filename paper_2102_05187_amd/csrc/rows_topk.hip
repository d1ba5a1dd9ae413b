// The K largest elements of dense rows.
#include "rows.hpp"
#include "rows_kernels.hpp"

namespace comet {

namespace {

constexpr int kThreads = 256;

// One workgroup a row.  The K-th largest key (value, then lower column; all different) is found bit by bit, the row being
// counted once for each; then the keys from there on are collected and put in order by counting.
template <int TYPE>
__global__ void __launch_bounds__(kThreads) k_rows_topk(const void *Z, int64_t V, int64_t ldz, float c2, double scale, int K, bool by_coordinate,
                                                        int32_t *__restrict__ crd, float *__restrict__ vals, float *__restrict__ lse,
                                                        const uint8_t *__restrict__ finished, int32_t eos,
                                                        uint64_t *__restrict__ out_keys, Log *__restrict__ logs) {
    using E = Elem<TYPE>;
    __shared__ float2 buf[kThreads / kWave];
    __shared__ double dbuf[kThreads / kWave];
    __shared__ uint64_t keys[COMET_MAX_TOP];
    __shared__ int found;
    const int64_t r = blockIdx.x;
    if (out_keys && finished && finished[r]) {               // an ended beam: one candidate, whatever its row holds
        for (int i = threadIdx.x; i < K; i += kThreads) out_keys[r * K + i] = i == 0 ? key_of(0.f, (uint32_t)eos) : 0;
        if (threadIdx.x == 0) logs[r] = Log{0.0, 0.0};
        return;
    }
    const Row<TYPE> row(Z, r, ldz, V);
    const int64_t nv = row.nvec();
    MaxSum a;
    double some = 0;                                         // elements that can be kept
    for (int64_t i = threadIdx.x; i < nv; i += kThreads) {
        float f[E::kPer];
        row.load(i, f);
        a.take<E::kPer>(f, c2);
#pragma unroll
        for (int k = 0; k < E::kPer; ++k) some += f[k] > kNegInf ? 1 : 0;
    }
    block_join<kThreads>(a, c2, buf);
    some = block_reduce<kThreads>(some, Add(), dbuf);
    if (lse && threadIdx.x == 0) lse[r] = a.m == -kNegInf ? a.m : (float)log_sum(a, scale).value();
    if (out_keys && threadIdx.x == 0) logs[r] = log_sum(a, scale);
    // the largest t with at least K keys >= t
    uint64_t t = 0;
    if (some > K)
        for (int bit = 63; bit >= 0; --bit) {
            const uint64_t mid = t | uint64_t(1) << bit;
            double n = 0;
            for (int64_t i = threadIdx.x; i < nv; i += kThreads) {
                float f[E::kPer];
                row.load(i, f);
#pragma unroll
                for (int k = 0; k < E::kPer; ++k) n += f[k] > kNegInf && key_of(f[k], (uint32_t)(row.first(i) + k)) >= mid ? 1 : 0;
            }
            n = block_reduce<kThreads>(n, Add(), dbuf);
            if (n >= K) t = mid;
            if (n == K) break;
        }
    if (threadIdx.x == 0) found = 0;
    __syncthreads();
    for (int64_t i = threadIdx.x; i < nv; i += kThreads) {
        float f[E::kPer];
        row.load(i, f);
#pragma unroll
        for (int k = 0; k < E::kPer; ++k) {
            const uint64_t key = key_of(f[k], (uint32_t)(row.first(i) + k));
            if (f[k] > kNegInf && key >= t) keys[atomicAdd(&found, 1)] = key;
        }
    }
    __syncthreads();
    const int n = found;
    for (int i = threadIdx.x; i < K; i += kThreads) {
        if (i >= n) {
            if (out_keys) out_keys[r * K + i] = 0;
            else crd[r * K + i] = -1, vals[r * K + i] = kNegInf;
            continue;
        }
        const uint64_t key = keys[i];
        int at = 0;
        for (int j = 0; j < n; ++j) at += by_coordinate ? column_of(keys[j]) < column_of(key) : keys[j] > key;
        if (out_keys) { out_keys[r * K + at] = key; continue; }
        crd[r * K + at] = (int32_t)column_of(key);
        vals[r * K + at] = value_of_key(key);
    }
}

}  // namespace

int64_t rows_topk_work(int, int64_t, int64_t, int64_t) { return 0; }

template <class... Args> static hipError_t launch(int type, int64_t N, hipStream_t st, Args... args) {
    const auto kernel = type == COMET_F32 ? k_rows_topk<COMET_F32> : type == COMET_BF16 ? k_rows_topk<COMET_BF16> : k_rows_topk<COMET_F16>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)N), dim3(kThreads), 0, st, args...);
    return hipGetLastError();
}

hipError_t rows_topk(const void *Z, int type, int64_t N, int64_t V, int64_t ldz, double scale, int64_t K, bool by_coordinate,
                     int32_t *crd, float *vals, float *lse, void *, hipStream_t st) {
    return launch(type, N, st, Z, V, ldz, (float)(scale * 1.4426950408889634), scale, (int)K, by_coordinate, crd, vals, lse,
                  (const uint8_t *)nullptr, 0, (uint64_t *)nullptr, (Log *)nullptr);
}

hipError_t rows_top_keys(const void *Z, int type, int64_t N, int64_t V, int64_t ldz, int64_t K, const uint8_t *finished, int32_t eos,
                         uint64_t *keys, void *logs, hipStream_t st) {
    return launch(type, N, st, Z, V, ldz, kLog2e, 1.0, (int)K, false, (int32_t *)nullptr, (float *)nullptr, (float *)nullptr, finished, eos,
                  keys, (Log *)logs);
}

}  // namespace comet
