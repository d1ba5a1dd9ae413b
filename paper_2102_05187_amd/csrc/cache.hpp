// What the kernels over a cache in blocks share, and their launchers (cache_map.hip, cache_write.hip, block_select.hip, block_attend.hip).
// Arguments are checked by the entry points (cache_api.hip); every launcher only enqueues work on `st`.
#pragma once

#include "rows.hpp"

namespace comet {

struct MapArgs {
    int64_t B, M, block;
    const int32_t *add;
    const uint8_t *ended;
    int32_t *length, *held, *table;
    int64_t ldt;
    int32_t *spare;
    int64_t S;
    int32_t *count;
    int64_t N;
    int32_t *pos;
    int64_t *slot;
    int32_t *place;
};
int64_t cache_map_work(int64_t B, int64_t M, int64_t N);
hipError_t cache_map(const MapArgs &a, void *work, hipStream_t st);

hipError_t cache_write(const comet_cache &c, int64_t N, const void *k, const int64_t k_stride[2], const void *v, const int64_t v_stride[2],
                       const int64_t *slot, hipStream_t st);

// The packed queries of B requests, and where their blocks are.
struct Queries {
    const void *q;
    int64_t N, Q, row, head;             // rows, heads, and their strides in elements
    int64_t B;
    const int32_t *pos, *length, *table;
    int64_t M, ldt;
};
int64_t block_select_work(const comet_cache &c, int64_t N, int64_t Q, int64_t B, int64_t M, int64_t K);
hipError_t block_select(const comet_cache &c, const Queries &q, int64_t K, int64_t first, int64_t last, int32_t *sel, void *work, hipStream_t st);

int64_t block_attend_work(const comet_cache &c, int64_t N, int64_t Q, int64_t B, int64_t M, int64_t K);
hipError_t block_attend(const comet_cache &c, const Queries &q, const int32_t *sel, int64_t K, double scale, void *out, float *lse, void *work,
                        hipStream_t st);

// ---- many workgroups -------------------------------------------------------------------------------------------------
// A launch has fewer than 2^32 threads.  More workgroups are enqueued in several, launch(first, count) each: a multiple of 8, so that the eight dies get as many.
template <class F> hipError_t in_launches(int64_t groups, int threads, F launch) {
    const int64_t most = (int64_t(1) << 32) / threads - 8;
    for (int64_t first = 0; first < groups; first += most) {
        launch((uint32_t)first, (unsigned)(groups - first < most ? groups - first : most));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// ---- sums over a workgroup, in the order of the threads ------------------------------------------------------------
__device__ __forceinline__ int64_t wave_scan(int64_t x) {
    const int lane = threadIdx.x & (kWave - 1);
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const int64_t y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    return x;
}
// The sum up to and with each thread's x; `total` becomes that of all.  buf: a place for each wavefront, free again afterwards.
template <int T> __device__ __forceinline__ int64_t block_scan(int64_t x, int64_t *buf, int64_t &total) {
    const int64_t up = wave_scan(x);
    if ((threadIdx.x & (kWave - 1)) == kWave - 1) buf[threadIdx.x / kWave] = up;
    __syncthreads();
    int64_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < T / kWave; ++w) {
        if (w < (int)(threadIdx.x / kWave)) before += buf[w];
        total += buf[w];
    }
    __syncthreads();
    return before + up;
}

// ---- requests of packed rows ---------------------------------------------------------------------------------------
// The request that a row belongs to, or -1: the number of requests that end at it or before it.  By a whole workgroup; count: one place of LDS.
template <int T> __device__ __forceinline__ int64_t request_of(const int32_t *pos, int64_t B, int64_t row, int *count) {
    if (threadIdx.x == 0) *count = 0;
    __syncthreads();
    int n = 0;
    for (int64_t b = threadIdx.x; b < B; b += T) n += pos[b + 1] <= row ? 1 : 0;
    if (n) atomicAdd(count, n);
    __syncthreads();
    const int b = *count;
    __syncthreads();
    return b < B && row >= pos[b] ? b : -1;
}

// Which tokens a workgroup has, and the first one's place in its request.
struct Tile { int64_t b, first; int n; int64_t place; };

// The sum over the lanes up to and with each.
__device__ __forceinline__ int lanes_scan(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}

// Tile `tile` of those that cut every request's tokens into pieces of `tokens`; n = 0 where there are not as many.
template <int T> __device__ __forceinline__ Tile find_tile(const Queries &q, int tokens, int tile, int64_t *buf, int64_t *where) {
    Tile t{0, 0, 0, 0};
    const auto cut = [&](int64_t b, int begin, int end, int length, int number) {
        const int n = end - begin, i = number * tokens;
        if (begin < 0) return;
        t.b = b, t.first = (int64_t)begin + i, t.n = n - i < tokens ? n - i : tokens, t.place = (int64_t)length - n + i;
        if (t.first + t.n > q.N) t.n = t.first < q.N ? (int)(q.N - t.first) : 0;
    };
    // One token a request, as decoding has them, or few requests: what is needed comes by scalar loads, which do not wait behind other workgroups' data.
    if (tokens == 1 && tile < q.B && q.pos[tile] == tile && q.pos[tile + 1] == tile + 1) {
        cut(tile, tile, tile + 1, q.length[tile], 0);
        return t;
    }
    if (q.B <= 4) {
        int at[5], length[4], left = tile;
#pragma unroll
        for (int b = 0; b < 5; ++b) at[b] = q.pos[b < q.B ? b : q.B];
#pragma unroll
        for (int b = 0; b < 4; ++b) length[b] = q.length[b < q.B ? b : 0];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int pieces = at[b + 1] > at[b] ? (at[b + 1] - at[b] + tokens - 1) / tokens : 0;
            if (left >= 0 && left < pieces) cut(b, at[b], at[b + 1], length[b], left);
            left -= pieces;
        }
        return t;
    }
    if (q.B <= 4 * kWave) {
        // every wavefront by itself: a request a lane, all that is needed of it with one wait
        const int lane = threadIdx.x & (kWave - 1);
        int begin[4], end[4], length[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int b = i * kWave + lane;
            begin[i] = end[i] = length[i] = 0;
            if (b < q.B) begin[i] = q.pos[b], end[i] = q.pos[b + 1], length[i] = q.length[b];
        }
        int before = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i * kWave >= q.B) break;
            const int mine = end[i] > begin[i] ? (end[i] - begin[i] + tokens - 1) / tokens : 0, upto = before + lanes_scan(mine);
            const uint64_t hit = __ballot(tile < upto);
            if (hit) {
                const int l = __builtin_ctzll(hit);
                cut(i * kWave + l, __builtin_amdgcn_readlane(begin[i], l), __builtin_amdgcn_readlane(end[i], l), __builtin_amdgcn_readlane(length[i], l),
                    tile - __builtin_amdgcn_readlane(upto - mine, l));
                return t;
            }
            before = __builtin_amdgcn_readlane(upto, kWave - 1);
        }
        return t;
    }
    if (threadIdx.x == 0) where[0] = -1;
    const int64_t each = (q.B + T - 1) / T, b0 = threadIdx.x * each, b1 = b0 + each < q.B ? b0 + each : q.B;
    int64_t mine = 0, total;
    const auto pieces = [&](int64_t b) { return q.pos[b + 1] > q.pos[b] ? (q.pos[b + 1] - q.pos[b] + tokens - 1) / tokens : 0; };
    for (int64_t b = b0; b < b1; ++b) mine += pieces(b);
    const int64_t upto = block_scan<T>(mine, buf, total);
    if (tile >= upto - mine && tile < upto) {
        int64_t left = tile - (upto - mine), b = b0;
        for (; left >= pieces(b); ++b) left -= pieces(b);
        where[0] = b, where[1] = left;
    }
    __syncthreads();
    const int64_t b = where[0];
    if (b >= 0) cut(b, q.pos[b], q.pos[b + 1], q.length[b], (int)where[1]);
    return t;
}

// An unsigned number whose order is that of the double: NaN is lowest, -0 is 0.
__device__ __forceinline__ uint64_t order_of_double(double x) {
    if (x != x) return 0;
    const uint64_t u = (uint64_t)__double_as_longlong(x + 0.0);
    return u >> 63 ? ~u : u | 0x8000000000000000ull;
}

}  // namespace comet
