// Attention over the blocks that are chosen for each query.
#include "cache.hpp"

namespace comet {

namespace {

struct AttendArgs {
    Queries q;
    const void *keys, *values;
    int64_t blocks;
    int block, heads, size, group;
    int64_t key_stride[3], value_stride[3];
    const int32_t *sel;
    int K;
    float c;                                  // scale * log2 e
    void *out;
    float *lse;
};

constexpr int kAttend = 256;

// One workgroup a token and query head: the simplest form.
template <int TYPE>
__global__ void __launch_bounds__(kAttend) k_attend_simple(AttendArgs a) {
    using E = Elem<TYPE>;
    using T = typename E::T;
    extern __shared__ __align__(16) char raw[];
    uint32_t *bits = (uint32_t *)raw;
    __shared__ float q[256], p[kAttend];
    __shared__ float2 red[kAttend / kWave];
    __shared__ int count;
    const int64_t n = blockIdx.x / a.q.Q;
    const int x = (int)(blockIdx.x % a.q.Q), h = x / a.group;
    const int64_t b = request_of<kAttend>(a.q.pos, a.q.B, n, &count);
    if (b < 0) return;
    const int64_t place = a.q.length[b] - ((int64_t)a.q.pos[b + 1] - n);
    const int64_t seen = place < 0 ? 0 : place / a.block + 1;
    const int C = (int)(seen < a.q.M ? seen : a.q.M), words = (C + 31) / 32;
    for (int w = threadIdx.x; w < words; w += kAttend) bits[w] = 0;
    for (int d = threadIdx.x; d < a.size; d += kAttend) q[d] = E::one(((const T *)a.q.q)[n * a.q.row + x * a.q.head + d]);
    __syncthreads();
    for (int i = threadIdx.x; i < a.K; i += kAttend) {
        const int j = a.sel[(n * a.heads + h) * a.K + i];
        if (j >= 0 && j < C) atomicOr(&bits[j >> 5], 1u << (j & 31));
    }
    __syncthreads();
    float m = kNegInf, l = 0.f, o = 0.f;
    for (int j = 0; j < C; ++j) {
        if (!(bits[j >> 5] >> (j & 31) & 1)) continue;
        const int64_t id = a.q.table[b * a.q.ldt + j];
        if (id < 0 || id >= a.blocks) continue;
        const int64_t left = place + 1 - (int64_t)j * a.block;
        const int there = (int)(left < a.block ? left : a.block);
        for (int i0 = 0; i0 < there; i0 += kAttend) {
            const int i = i0 + threadIdx.x;
            float s = kNegInf;
            if (i < there) {
                const T *k = (const T *)a.keys + id * a.key_stride[0] + i * a.key_stride[1] + h * a.key_stride[2];
                s = 0.f;
                for (int d = 0; d < a.size; d += E::kPer) {
                    float f[E::kPer];
                    E::widen(*(const uint4 *)(k + d), f);
#pragma unroll
                    for (int e = 0; e < E::kPer; ++e) s = __builtin_fmaf(q[d + e], f[e], s);
                }
                s *= a.c;
            }
            MaxSum top;
            top.m = s;
            block_join<kAttend>(top, 1.f, red);
            const float M = fmaxf(m, top.m), safe = M == kNegInf ? 0.f : M;
            const float w = i < there ? exp2_fast(s - safe) : 0.f;
            const float back = exp2_fast(m - safe);
            p[threadIdx.x] = w;
            top.m = 0.f, top.s = w;
            block_join<kAttend>(top, 1.f, red);              // a barrier behind p's last write among it
            l = l * back + top.s;
            o *= back;
            m = M;
            if ((int)threadIdx.x < a.size) {
                const T *v = (const T *)a.values + id * a.value_stride[0] + h * a.value_stride[2] + threadIdx.x;
                for (int k = 0; k < kAttend && i0 + k < there; ++k) o = __builtin_fmaf(p[k], E::one(v[(i0 + k) * a.value_stride[1]]), o);
            }
            __syncthreads();
        }
    }
    const bool any = m > kNegInf || l != l;
    if ((int)threadIdx.x < a.size) ((T *)a.out)[(n * a.q.Q + x) * a.size + threadIdx.x] = (T)E::bits(any ? o / l : 0.f);
    if (threadIdx.x == 0 && a.lse) a.lse[n * a.q.Q + x] = any ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : kNegInf;
}

}  // namespace

int64_t block_attend_work(const comet_cache &, int64_t, int64_t, int64_t, int64_t, int64_t) { return 0; }

hipError_t block_attend(const comet_cache &c, const Queries &q, const int32_t *sel, int64_t K, double scale, void *out, float *lse, void *, hipStream_t st) {
    AttendArgs a{q, c.keys, c.values, c.blocks, (int)c.block, (int)c.heads, (int)c.size, (int)(q.Q / c.heads), {}, {}, sel, (int)K,
                 (float)(scale * 1.4426950408889634), out, lse};
    for (int i = 0; i < 3; ++i) a.key_stride[i] = c.key_stride[i], a.value_stride[i] = c.value_stride[i];
    const dim3 grid((unsigned)(q.N * q.Q));
    const size_t lds = (size_t)(q.M + 31) / 32 * 4;
    const auto kernel = c.type == COMET_F32 ? k_attend_simple<COMET_F32> : c.type == COMET_BF16 ? k_attend_simple<COMET_BF16> : k_attend_simple<COMET_F16>;
    hipLaunchKernelGGL(kernel, grid, dim3(kAttend), lds, st, a);
    return hipGetLastError();
}

}  // namespace comet
