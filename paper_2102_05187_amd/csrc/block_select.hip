// The blocks that each query is to read, by the score of its heads' sum with the block's mean key.
#include "cache.hpp"

namespace comet {

namespace {

struct SelectArgs {
    Queries q;
    const void *mean;
    int64_t blocks, mean_block, mean_head;
    int block, heads, size, group;
    int K, first, last;
    int32_t *sel;
};

constexpr int kSelect = 256;
constexpr uint64_t kAlways = ~0ull;          // above the order of every double

// One workgroup a token and head.  Scores in 64 bits: products of 16-bit elements are exact there, and a sum of a few hundred of
// them is off by 1e-14, so that it is the exact scores' order that decides.
template <int TYPE>
__global__ void __launch_bounds__(kSelect) k_select_one(SelectArgs a) {
    using E = Elem<TYPE>;
    extern __shared__ __align__(16) char raw[];
    uint64_t *key = (uint64_t *)raw;
    __shared__ double q[256];
    __shared__ int count[64 + 1];
    __shared__ int64_t scan[kSelect / kWave];
    const int64_t n = blockIdx.x / a.heads, h = blockIdx.x % a.heads;
    const int64_t b = request_of<kSelect>(a.q.pos, a.q.B, n, count);
    if (b < 0) return;
    int32_t *sel = a.sel + (n * a.heads + h) * a.K;
    const int64_t place = a.q.length[b] - ((int64_t)a.q.pos[b + 1] - n);
    const int64_t seen = place < 0 ? 0 : place / a.block + 1;
    const int C = (int)(seen < a.q.M ? seen : a.q.M);
    if (C <= a.K) {
        for (int i = threadIdx.x; i < a.K; i += kSelect) sel[i] = i < C ? i : -1;
        return;
    }
    for (int d = threadIdx.x; d < a.size; d += kSelect) {
        double s = 0;
        for (int g = 0; g < a.group; ++g) s += (double)E::one(((const typename E::T *)a.q.q)[n * a.q.row + (h * a.group + g) * a.q.head + d]);
        q[d] = s;
    }
    if (threadIdx.x < 65) count[threadIdx.x] = 0;
    __syncthreads();
    const int32_t *table = a.q.table + b * a.q.ldt;
    for (int j = threadIdx.x; j < C; j += kSelect) {
        uint64_t k = kAlways;
        if (j >= a.first && j < C - a.last) {
            const int64_t p = table[j];
            k = 0;
            if (p >= 0 && p < a.blocks) {
                const typename E::T *m = (const typename E::T *)a.mean + p * a.mean_block + h * a.mean_head;
                double s = 0;
                for (int d = 0; d < a.size; d += E::kPer) {
                    float f[E::kPer];
                    E::widen(*(const uint4 *)(m + d), f);
#pragma unroll
                    for (int e = 0; e < E::kPer; ++e) s = __builtin_fma(q[d + e], (double)f[e], s);
                }
                k = order_of_double(s);
            }
        }
        key[j] = k;
    }
    __syncthreads();
    // the K-th largest key: bits from the highest on, each kept where K keys reach it
    uint64_t bar = 0;
    for (int bit = 63; bit >= 0; --bit) {
        const uint64_t t = bar | 1ull << bit;
        int c = 0;
        for (int j = threadIdx.x; j < C; j += kSelect) c += key[j] >= t ? 1 : 0;
        if (c) atomicAdd(&count[bit], c);
        __syncthreads();
        if (count[bit] >= a.K) bar = t;
        if (count[bit] == a.K) break;
    }
    int more = 0;
    for (int j = threadIdx.x; j < C; j += kSelect) more += key[j] > bar ? 1 : 0;
    if (more) atomicAdd(&count[64], more);
    __syncthreads();
    const int equal = a.K - count[64];                       // of those that are at the bar, the lowest j
    int64_t before = 0, ties = 0, all;
    for (int j0 = 0; j0 < C; j0 += kSelect) {
        const int j = j0 + threadIdx.x;
        const uint64_t k = j < C ? key[j] : 0;
        const int64_t tie = ties + block_scan<kSelect>(j < C && k == bar ? 1 : 0, scan, all);
        ties += all;
        const bool in = j < C && (k > bar || (k == bar && tie <= equal));
        const int64_t at = before + block_scan<kSelect>(in ? 1 : 0, scan, all);
        before += all;
        if (in) sel[at - 1] = j;
    }
}

}  // namespace

int64_t block_select_work(const comet_cache &, int64_t, int64_t, int64_t, int64_t, int64_t) { return 0; }

hipError_t block_select(const comet_cache &c, const Queries &q, int64_t K, int64_t first, int64_t last, int32_t *sel, void *, hipStream_t st) {
    const SelectArgs a{q, c.mean, c.blocks, c.mean_stride[0], c.mean_stride[1], (int)c.block, (int)c.heads, (int)c.size, (int)(q.Q / c.heads),
                       (int)K, (int)first, (int)last, sel};
    const dim3 grid((unsigned)(q.N * c.heads));
    const size_t lds = (size_t)q.M * 8;
    const auto kernel = c.type == COMET_F32 ? k_select_one<COMET_F32> : c.type == COMET_BF16 ? k_select_one<COMET_BF16> : k_select_one<COMET_F16>;
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, grid, dim3(kSelect), lds, st, a);
    return hipGetLastError();
}

}  // namespace comet
