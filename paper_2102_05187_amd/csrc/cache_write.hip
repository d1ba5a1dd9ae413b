// New keys and values into the slots of a cache, and the means of the blocks that become whole.
#include "cache.hpp"

namespace comet {

namespace {

struct WriteArgs {
    const char *k, *v;
    char *keys, *values, *mean;
    int64_t N, slots;
    int block, heads, per_head;                  // per_head: 16-byte vectors of a head
    int64_t k_row, k_head, v_row, v_head;        // all in bytes
    int64_t key_stride[3], value_stride[3], mean_stride[2];
    const int64_t *slot;
};

constexpr int kWrite = 256;

template <int TYPE>
__global__ void __launch_bounds__(kWrite) k_cache_write(WriteArgs a, int rows) {
    using E = Elem<TYPE>;
    __shared__ float part[kWrite * E::kPer];
    __shared__ int run;
    const int columns = a.heads * a.per_head;
    const int64_t i0 = (int64_t)blockIdx.x * rows;
    const int64_t here = a.N - i0 < rows ? a.N - i0 : rows;
    for (int64_t x = threadIdx.x; x < here * columns * 2; x += kWrite) {
        const int64_t r = x / (2 * columns);
        int c = (int)(x - r * 2 * columns);
        const bool value = c >= columns;
        if (value) c -= columns;
        const int64_t s = a.slot[i0 + r];
        if (s < 0 || s >= a.slots) continue;
        const int64_t p = s / a.block, in = s - p * a.block, h = c / a.per_head, d = (int64_t)(c - h * a.per_head) * 16;
        if (value) *(uint4 *)(a.values + p * a.value_stride[0] + in * a.value_stride[1] + h * a.value_stride[2] + d) = *(const uint4 *)(a.v + (i0 + r) * a.v_row + h * a.v_head + d);
        else *(uint4 *)(a.keys + p * a.key_stride[0] + in * a.key_stride[1] + h * a.key_stride[2] + d) = *(const uint4 *)(a.k + (i0 + r) * a.k_row + h * a.k_head + d);
    }
    if (!a.mean) return;
    for (int64_t i = i0; i < i0 + here; ++i) {
        const int64_t s = a.slot[i];
        if (s < 0 || s >= a.slots || s % a.block != a.block - 1) continue;           // the same for all threads
        // how many rows before this one fill the places before its own: those are read from k, where another workgroup may be copying them
        if (threadIdx.x == 0) run = a.block;
        __syncthreads();
        for (int j = threadIdx.x + 1; j < a.block; j += kWrite)
            if (j > i || a.slot[i - j] != s - j) atomicMin(&run, j);
        __syncthreads();
        const int old = a.block - run;                                                // places that the cache has already
        const int64_t p = s / a.block;
        // columns side by side, places in groups: each thread adds up a column's places o, o + groups, ..
        for (int c0 = 0; c0 < columns; c0 += kWrite) {
            const int width = columns - c0 < kWrite ? columns - c0 : kWrite, groups = kWrite / width;
            const int g = threadIdx.x / width, c = c0 + threadIdx.x - g * width;
            const int64_t h = c / a.per_head, d = (int64_t)(c - h * a.per_head) * 16;
            float sum[E::kPer] = {};
            if (g < groups) {
#pragma unroll 4
                for (int o = g; o < a.block; o += groups) {
                    const char *from = o < old ? a.keys + p * a.key_stride[0] + o * a.key_stride[1] + h * a.key_stride[2] + d
                                               : a.k + (i - (a.block - 1 - o)) * a.k_row + h * a.k_head + d;
                    float f[E::kPer];
                    E::widen(*(const uint4 *)from, f);
#pragma unroll
                    for (int e = 0; e < E::kPer; ++e) sum[e] += f[e];
                }
            }
#pragma unroll
            for (int e = 0; e < E::kPer; ++e) part[threadIdx.x * E::kPer + e] = sum[e];
            __syncthreads();
            if (g == 0) {
                for (int o = 1; o < groups; ++o)
#pragma unroll
                    for (int e = 0; e < E::kPer; ++e) sum[e] += part[(o * width + threadIdx.x) * E::kPer + e];
#pragma unroll
                for (int e = 0; e < E::kPer; ++e) sum[e] /= (float)a.block;
                *(uint4 *)(a.mean + p * a.mean_stride[0] + h * a.mean_stride[1] + d) = E::narrow(sum);
            }
            __syncthreads();
        }
    }
}

}  // namespace

hipError_t cache_write(const comet_cache &c, int64_t N, const void *k, const int64_t k_stride[2], const void *v, const int64_t v_stride[2],
                       const int64_t *slot, hipStream_t st) {
    const int64_t e = c.type == COMET_F32 ? 4 : 2;
    WriteArgs a{(const char *)k, (const char *)v, (char *)c.keys, (char *)c.values, (char *)c.mean, N, c.blocks * c.block, (int)c.block, (int)c.heads,
                (int)(c.size * e / 16), k_stride[0] * e, k_stride[1] * e, v_stride[0] * e, v_stride[1] * e, {}, {}, {}, slot};
    for (int i = 0; i < 3; ++i) a.key_stride[i] = c.key_stride[i] * e, a.value_stride[i] = c.value_stride[i] * e;
    for (int i = 0; i < 2; ++i) a.mean_stride[i] = c.mean_stride[i] * e;
    const int rows = N > 4096 ? 8 : 1;
    const dim3 grid((unsigned)((N + rows - 1) / rows));
    if (c.type == COMET_F32) hipLaunchKernelGGL(k_cache_write<COMET_F32>, grid, dim3(kWrite), 0, st, a, rows);
    else if (c.type == COMET_BF16) hipLaunchKernelGGL(k_cache_write<COMET_BF16>, grid, dim3(kWrite), 0, st, a, rows);
    else hipLaunchKernelGGL(k_cache_write<COMET_F16>, grid, dim3(kWrite), 0, st, a, rows);
    return hipGetLastError();
}

}  // namespace comet
