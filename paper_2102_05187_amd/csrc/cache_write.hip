// New keys and values into the slots of a cache, and the means of the blocks that become whole.
#include "cache.hpp"

namespace comet {

namespace {

typedef uint32_t V4 __attribute__((ext_vector_type(4)));

struct WriteArgs {
    const char *k, *v;
    char *keys, *values, *mean;
    int64_t N, slots;
    int block, heads, per_head;                  // per_head: 16-byte vectors of a head
    int64_t k_row, k_head, v_row, v_head;        // all in bytes
    int64_t key_block, key_place, key_head, value_block, value_place, value_head, mean_block, mean_head;
    const int64_t *slot;
};

constexpr int kWrite = 256, kSlice = 32;      // threads of a workgroup; columns of one that takes means

// Block and place of a slot; false where it is none.  In 32 bits where the cache has fewer slots.
template <class I> __device__ __forceinline__ bool find(const WriteArgs &a, int64_t s, int64_t &p, int &in) {
    if (s < 0 || s >= a.slots) return false;
    const I b = (I)s / (I)a.block;
    p = b, in = (int)((I)s - b * (I)a.block);
    return true;
}

// Rows i0 .. i0 + here - 1 to their slots: a thread a 16-byte column of the keys or the values, four rows under way.
template <class I> __device__ __forceinline__ void copy_rows(const WriteArgs &a, int64_t i0, int here) {
    const int columns = a.heads * a.per_head, both = 2 * columns;
    const auto column = [&](int x, int r0, int step) {
        const bool value = x >= columns;
        const int c = value ? x - columns : x, h = c / a.per_head, d = (c - h * a.per_head) * 16;
        const char *from = (value ? a.v : a.k) + h * (value ? a.v_head : a.k_head) + d;
        char *to = (value ? a.values : a.keys) + h * (value ? a.value_head : a.key_head) + d;
        const int64_t line = value ? a.v_row : a.k_row, block = value ? a.value_block : a.key_block, place = value ? a.value_place : a.key_place;
        for (int r = r0; r < here; r += 4 * step) {
            V4 y[4];
            int64_t s[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t i = i0 + (r + u * step < here ? r + u * step : here - 1);
                y[u] = *(const V4 *)(from + i * line);
                s[u] = a.slot[i];
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                int64_t p;
                int in;
                if (r + u * step < here && find<I>(a, s[u], p, in)) *(V4 *)(to + p * block + in * place) = y[u];
            }
        }
    };
    if (both >= kWrite) {
        for (int x = threadIdx.x; x < both; x += kWrite) column(x, 0, 1);        // the rows' slots are the same for all threads
    } else {
        const int step = kWrite / both, r0 = threadIdx.x / both;
        if (r0 < step) column(threadIdx.x - r0 * both, r0, step);
    }
}

// The means of the blocks whose last place is that of one of `here` rows from i0 on, at 16-byte columns c0 .. c0 + kSlice - 1.  Eight threads a column, which
// add up every eighth place.
template <int TYPE, class I> __device__ __forceinline__ void means(const WriteArgs &a, int64_t i0, int here, int c0) {
    using E = Elem<TYPE>;
    constexpr int GROUPS = kWrite / kSlice;
    __shared__ float part[kWrite * E::kPer];
    __shared__ int ends[COMET_MAX_BLOCK], count, run;
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
    for (int r = threadIdx.x; r < here; r += kWrite) {
        int64_t p;
        int in;
        if (find<I>(a, a.slot[i0 + r], p, in) && in == a.block - 1) ends[atomicAdd(&count, 1)] = r;
    }
    __syncthreads();
    const int some = count, g = threadIdx.x / kSlice, c = c0 + threadIdx.x % kSlice, columns = a.heads * a.per_head;
    const int64_t h = c / a.per_head, d = (int64_t)(c - h * a.per_head) * 16;
    for (int n = 0; n < some; ++n) {
        const int64_t i = i0 + ends[n], s = a.slot[i];
        // how many rows before this one fill the places before its own: those are read from k, where another workgroup may be copying them
        if (threadIdx.x == 0) run = a.block;
        __syncthreads();
        for (int j = threadIdx.x + 1; j < a.block; j += kWrite)
            if (j > i || a.slot[i - j] != s - j) atomicMin(&run, j);
        __syncthreads();
        const int old = a.block - run;                                                // places that the cache has already
        int64_t p;
        int in;
        find<I>(a, s, p, in);
        float sum[E::kPer] = {};
        if (c < columns) {
            const char *key = a.keys + p * a.key_block + h * a.key_head + d, *row = a.k + (i - a.block + 1) * a.k_row + h * a.k_head + d;
#pragma unroll 8
            for (int o = g; o < a.block; o += GROUPS) {
                const V4 y = *(const V4 *)(o < old ? key + o * a.key_place : row + o * a.k_row);
                float f[E::kPer];
                E::widen(make_uint4(y.x, y.y, y.z, y.w), f);
#pragma unroll
                for (int e = 0; e < E::kPer; ++e) sum[e] += f[e];
            }
        }
#pragma unroll
        for (int e = 0; e < E::kPer; ++e) part[e * kWrite + threadIdx.x] = sum[e];
        __syncthreads();
        if (g == 0 && c < columns) {
            for (int o = 1; o < GROUPS; ++o)
#pragma unroll
                for (int e = 0; e < E::kPer; ++e) sum[e] += part[e * kWrite + o * kSlice + threadIdx.x];
#pragma unroll
            for (int e = 0; e < E::kPer; ++e) sum[e] /= (float)a.block;
            *(uint4 *)(a.mean + p * a.mean_block + h * a.mean_head + d) = E::narrow(sum);
        }
        __syncthreads();
    }
}

// The first workgroups take means, of `block` rows and a slice of the columns each, the others copy four rows.  Bound by memory where rows are many (8191 rows of
// 2 x 2 KB: 14 to 16 us, 13 without means, and two copies of half the size 20; a row a workgroup 18), by one read after the other where they are few.  Means
// taken by the workgroups that copy the blocks' last rows, behind the copy, were 26.
template <int TYPE, class I>
__global__ void __launch_bounds__(kWrite) k_cache_write(WriteArgs a, int64_t from, int rows, unsigned slices, unsigned for_means) {
    if (blockIdx.x < for_means) {
        const int64_t i0 = from + (int64_t)(blockIdx.x / slices) * a.block;
        means<TYPE, I>(a, i0, (int)(a.N - i0 < a.block ? a.N - i0 : a.block), (int)(blockIdx.x % slices) * kSlice);
    } else {
        const int64_t i0 = from + (int64_t)(blockIdx.x - for_means) * rows;
        copy_rows<I>(a, i0, (int)(a.N - i0 < rows ? a.N - i0 : rows));
    }
}

template <int TYPE, class I> hipError_t launch(const WriteArgs &a, hipStream_t st) {
    const int64_t rows = 4, slices = (a.heads * a.per_head + kSlice - 1) / kSlice;
    // as many rows, of whole blocks' number, as a launch has threads for: fewer than 2^32
    const int64_t most = ((int64_t(1) << 32) / kWrite - 1) / (a.block / rows + slices) * a.block;
    for (int64_t from = 0; from < a.N; from += most) {
        const int64_t n = a.N - from < most ? a.N - from : most, for_means = a.mean ? (n + a.block - 1) / a.block * slices : 0;
        hipLaunchKernelGGL((k_cache_write<TYPE, I>), dim3((unsigned)(for_means + (n + rows - 1) / rows)), dim3(kWrite), 0, st, a, from, (int)rows, (unsigned)slices,
                           (unsigned)for_means);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <int TYPE> hipError_t launch(const WriteArgs &a, hipStream_t st) {
    return a.slots < (int64_t(1) << 31) ? launch<TYPE, uint32_t>(a, st) : launch<TYPE, int64_t>(a, st);
}

}  // namespace

hipError_t cache_write(const comet_cache &c, int64_t N, const void *k, const int64_t k_stride[2], const void *v, const int64_t v_stride[2],
                       const int64_t *slot, hipStream_t st) {
    const int64_t e = c.type == COMET_F32 ? 4 : 2;
    const WriteArgs a{(const char *)k, (const char *)v, (char *)c.keys, (char *)c.values, (char *)c.mean, N, c.blocks * c.block, (int)c.block, (int)c.heads,
                      (int)(c.size * e / 16), k_stride[0] * e, k_stride[1] * e, v_stride[0] * e, v_stride[1] * e,
                      c.key_stride[0] * e, c.key_stride[1] * e, c.key_stride[2] * e, c.value_stride[0] * e, c.value_stride[1] * e, c.value_stride[2] * e,
                      c.mean_stride[0] * e, c.mean_stride[1] * e, slot};
    return c.type == COMET_F32 ? launch<COMET_F32>(a, st) : c.type == COMET_BF16 ? launch<COMET_BF16>(a, st) : launch<COMET_F16>(a, st);
}

}  // namespace comet
