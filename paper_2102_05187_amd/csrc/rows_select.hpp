// Choosing the K largest of what a workgroup's threads hold in registers.
#pragma once

#include "rows.hpp"

namespace comet {

constexpr int kCandidates = 2048;         // keys that a workgroup keeps in LDS
constexpr int kTries = 64;                // halvings of a threshold's range

// One count over the workgroup: every thread's n, added up (n is up to a few dozen; `slot` was 0).
template <int T> __device__ __forceinline__ int block_count(int n, int *slot) {
    if (__ballot(n != 0)) {
        const int sum = (int)wave_reduce((float)n, 0.f, Add());               // whole numbers far below 2^24
        if ((threadIdx.x & (kWave - 1)) == 0) atomicAdd(slot, sum);
    }
    __syncthreads();
    return *slot;
}
template <int T> __device__ __forceinline__ int block_count(bool yes, int *slot) {
    const uint64_t b = __ballot(yes);
    if (b && (threadIdx.x & (kWave - 1)) == 0) atomicAdd(slot, (int)__popcll(b));
    __syncthreads();
    return *slot;
}

// A bound that at least K of the held numbers reach and not many more than K: the range between `lo` and `hi` (the largest) is
// halved by value, a few times, then by the numbers' order, until K to K + K/4 + 4 reach its lower end or nothing is left to halve.
// `lo` comes back where no more than that reach it.  Elements below the bound cannot be among the K largest of the workgroup's elements where each
// held number is one of them.  COUNT(t) says how many of a thread's numbers have an order of t or more.  All threads return the same.
// `tries`: kTries places of LDS that hold 0.
template <int T, class COUNT> __device__ __forceinline__ uint32_t bound(uint32_t lo, uint32_t hi, int K, COUNT count, int *tries) {
    const int most = K + K / 4 + 4;
    if (block_count<T>(count(lo), &tries[0]) <= most) return lo;
    for (int i = 1; i < kTries && lo < hi; ++i) {
        uint32_t mid = 0;
        if (i <= 12) {
            const float a = value_of(lo), b = value_of(hi);
            mid = order_of(0.5f * a + 0.5f * b);
        }
        if (!(mid > lo && mid <= hi)) mid = lo + (hi - lo + 1) / 2;
        const int n = block_count<T>(count(mid), &tries[i]);
        if (n >= K) {
            lo = mid;
            if (n <= most) break;
        } else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ float finite(float x) { return fminf(fmaxf(x, -3.402823466e38f), 3.402823466e38f); }
// An unsigned number whose order is that of the score.
__device__ __forceinline__ uint64_t order64(double s) {
    const uint64_t u = __builtin_bit_cast(uint64_t, s + 0.0);
    return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ __forceinline__ double score_of(uint64_t o) { return __builtin_bit_cast(double, o >> 63 ? o & ~(1ull << 63) : ~o); }

// Things that sort_items() puts in order: plain keys, largest first ...
struct Keys {
    using Item = uint64_t;
    uint64_t *keys;
    __device__ __forceinline__ Item get(int i) const { return keys[i]; }
    __device__ __forceinline__ void put(int i, Item v) const { keys[i] = v; }
    static __device__ __forceinline__ bool before(Item a, Item b) { return a > b; }
    static __device__ __forceinline__ Item none() { return 0; }
    static __device__ __forceinline__ float rough(Item a) { return finite(value_of((uint32_t)(a >> 32))); }
};
// ... keys whose upper half is a number ...
struct NumberKeys : Keys {
    static __device__ __forceinline__ float rough(Item a) { return (float)(uint32_t)(a >> 32); }
};
// ... and keys of 128 bits, the upper half a score.
struct WideKey { uint64_t high, low; };
struct WideKeys {
    using Item = WideKey;
    uint64_t *high, *low;
    __device__ __forceinline__ Item get(int i) const { return Item{high[i], low[i]}; }
    __device__ __forceinline__ void put(int i, Item v) const { high[i] = v.high, low[i] = v.low; }
    static __device__ __forceinline__ bool before(Item a, Item b) { return a.high > b.high || (a.high == b.high && a.low > b.low); }
    static __device__ __forceinline__ Item none() { return Item{0, 0}; }
    static __device__ __forceinline__ float rough(Item a) { return finite((float)score_of(a.high)); }
};

constexpr int kBins = 512;
constexpr int kCrowd = 48;                // more than these in one bin: the bins are of no use
struct SortSpace {
    int count[kBins];                     // also the ranks of few
    int head[kBins];
    uint16_t next[kCandidates];
    float ends[2][16];
    int crowd;
};

// Puts n different items in LDS in order (n <= kCandidates; places up to the next power of two are used too).  An item's place is its
// rank.  Few are compared with all others, several threads counting for each.  More are put into bins by their rough value, which are as wide
// as each other from the least to the largest, and compared with the others of their bin.  Where the values crowd in a few bins
// (outliers), a bitonic network sorts them.
template <int T, class S> __device__ __forceinline__ void sort_items(const S &s, int n, SortSpace &sp) {
    constexpr int E = kCandidates / T;                                         // items of a thread
    using Item = typename S::Item;
    if (n <= 2 * kWave) {
        const int wide = n <= kWave ? kWave : 2 * kWave, parts = T / wide;     // threads of one part
        const int part = threadIdx.x / wide, i = threadIdx.x - part * wide, per = (n + parts - 1) / parts;
        const int j0 = part * per, j1 = j0 + per < n ? j0 + per : n;
        if (threadIdx.x < 2 * kWave) sp.count[threadIdx.x] = 0;
        Item mine{};
        if (i < n) mine = s.get(i);
        __syncthreads();
        if (i < n) {
            int at = 0;
#pragma unroll 4
            for (int j = j0; j < j1; ++j) at += S::before(s.get(j), mine) ? 1 : 0;
            if (at) atomicAdd(&sp.count[i], at);
        }
        __syncthreads();
        if (part == 0 && i < n) s.put(sp.count[i], mine);
        __syncthreads();
        return;
    }
    for (int i = threadIdx.x; i < kBins; i += T) sp.count[i] = 0, sp.head[i] = -1;
    if (threadIdx.x == 0) sp.crowd = 0;
    Item mine[E];
    float least = -kNegInf, most = kNegInf;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int i = e * T + threadIdx.x;
        if (i >= n) continue;
        mine[e] = s.get(i);
        least = fminf(least, S::rough(mine[e])), most = fmaxf(most, S::rough(mine[e]));
    }
    least = wave_reduce(least, -kNegInf, Smaller());
    most = wave_reduce(most, kNegInf, Larger());
    if ((threadIdx.x & (kWave - 1)) == 0) sp.ends[0][threadIdx.x / kWave] = least, sp.ends[1][threadIdx.x / kWave] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < T / kWave; ++w) least = fminf(least, sp.ends[0][w]), most = fmaxf(most, sp.ends[1][w]);
    const float per = (kBins - 1) / fmaxf(0.5f * most - 0.5f * least, 1e-30f);  // bins for half the distance: the whole one may overflow
    int bin[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int i = e * T + threadIdx.x;
        if (i >= n) continue;
        const float b = (0.5f * S::rough(mine[e]) - 0.5f * least) * per;
        bin[e] = b < (float)(kBins - 1) ? (int)b : kBins - 1;
        atomicAdd(&sp.count[bin[e]], 1);
        sp.next[i] = (uint16_t)atomicExch(&sp.head[bin[e]], i);                // 65535: none
    }
    __syncthreads();
    if (threadIdx.x < kWave) {                                                 // count[b]: items in the bins above b
        constexpr int B = kBins / kWave;
        const int last = kBins - 1 - (int)threadIdx.x * B;
        int c[B], sum = 0;
#pragma unroll
        for (int k = 0; k < B; ++k) {
            c[k] = sp.count[last - k], sum += c[k];
            if (c[k] > kCrowd) sp.crowd = 1;
        }
        int before = sum;
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) {
            const int x = __shfl_up(before, d);
            if ((int)threadIdx.x >= d) before += x;
        }
        before -= sum;
#pragma unroll
        for (int k = 0; k < B; ++k) sp.count[last - k] = before, before += c[k];
    }
    __syncthreads();
    if (sp.crowd) {
        int N = 4 * kWave;
        while (N < n) N *= 2;
        for (int i = n + threadIdx.x; i < N; i += T) s.put(i, S::none());
        __syncthreads();
        // steps over distances of up to 64 stay inside of a wavefront's 128 items and need no barrier
        for (int k = 2; k <= N; k *= 2)
            for (int j = k / 2; j > 0; j /= 2) {
                for (int t = threadIdx.x; t < N / 2; t += T) {
                    const int i = 2 * t - (t & (j - 1)), o = i + j;            // t's pair, j apart
                    const Item a = s.get(i), b = s.get(o);
                    if (S::before(b, a) == ((i & k) == 0)) { s.put(i, b); s.put(o, a); }
                }
                if (j > kWave || (j == 1 && k >= 2 * kWave)) __syncthreads();
                else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            }
        return;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if (e * T + (int)threadIdx.x >= n) continue;
        int at = sp.count[bin[e]];
        for (int m = sp.head[bin[e]]; m >= 0 && m != 65535; m = sp.next[m]) at += S::before(s.get(m), mine[e]) ? 1 : 0;
        bin[e] = at;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (e * T + (int)threadIdx.x < n) s.put(bin[e], mine[e]);
    __syncthreads();
}

// Adds the wavefront's chosen elements to a list in LDS: each lane has `mine` of them, and is told where its first one goes.
__device__ __forceinline__ int append(int mine, int *found) {
    int upto = mine;
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x111, 0xf, 0xf, false);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x112, 0xf, 0xf, false);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x114, 0xf, 0xf, false);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x118, 0xf, 0xf, false);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x142, 0xa, 0xf, false);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x143, 0xc, 0xf, false);
    int base = 0;
    if ((threadIdx.x & (kWave - 1)) == kWave - 1) base = atomicAdd(found, upto);
    return __builtin_amdgcn_readlane(base, kWave - 1) + upto - mine;
}

// The K-th largest of different numbers of 64 bits between lo and hi, of which K at least are `lo` or more: COUNT(t) says how many of a thread's
// are t or more.  `tries` has kTries places that hold 0, and is left so.
template <int T, class COUNT> __device__ __forceinline__ uint64_t kth(uint64_t lo, uint64_t hi, int K, COUNT count, int *tries) {
    for (int i = 0; lo < hi; ++i) {
        const uint64_t mid = lo + (hi - lo) / 2 + 1;
        const int reach = block_count<T>(count(mid), &tries[i % kTries]);
        if (threadIdx.x == 0) tries[(i + kTries - 1) % kTries] = 0;            // the one before, which all have read
        if (reach >= K) lo = mid;
        else hi = mid - 1;
        if (reach == K) break;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kTries; i += T) tries[i] = 0;
    __syncthreads();
    return lo;
}

}  // namespace comet
