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

// Things that sort_items() puts in order: plain keys, largest first ...
struct Keys {
    using Item = uint64_t;
    uint64_t *keys;
    __device__ __forceinline__ Item get(int i) const { return keys[i]; }
    __device__ __forceinline__ void put(int i, Item v) const { keys[i] = v; }
    static __device__ __forceinline__ bool before(Item a, Item b) { return a > b; }
    static __device__ __forceinline__ Item none() { return 0; }
};
// ... and keys of 128 bits.
struct WideKey { uint64_t high, low; };
struct WideKeys {
    using Item = WideKey;
    uint64_t *high, *low;
    __device__ __forceinline__ Item get(int i) const { return Item{high[i], low[i]}; }
    __device__ __forceinline__ void put(int i, Item v) const { high[i] = v.high, low[i] = v.low; }
    static __device__ __forceinline__ bool before(Item a, Item b) { return a.high > b.high || (a.high == b.high && a.low > b.low); }
    static __device__ __forceinline__ Item none() { return Item{0, 0}; }
};

// Puts n different items in LDS in order; places up to the next power of two (256 at least where n > 128) are used too.  Few
// are moved to their rank, counted by several threads each; more go through a bitonic network, whose steps over distances of up to 64
// stay inside of a wavefront's 128 items and need no barrier.  `ranks`: 128 places.
template <int T, class S> __device__ __forceinline__ void sort_items(const S &s, int n, int *ranks) {
    static_assert(T >= 2 * kWave, "ranks are counted by two wavefronts or more");
    if (n <= 2 * kWave) {
        const int wide = n <= kWave ? kWave : 2 * kWave, parts = T / wide;     // threads of one part
        const int part = threadIdx.x / wide, i = threadIdx.x - part * wide, per = (n + parts - 1) / parts;
        const int j0 = part * per, j1 = j0 + per < n ? j0 + per : n;
        if (threadIdx.x < 2 * kWave) ranks[threadIdx.x] = 0;
        const typename S::Item mine = i < n ? s.get(i) : S::none();
        __syncthreads();
        if (i < n) {
            int at = 0;
#pragma unroll 4
            for (int j = j0; j < j1; ++j) at += S::before(s.get(j), mine) ? 1 : 0;
            if (at) atomicAdd(&ranks[i], at);
        }
        __syncthreads();
        if (part == 0 && i < n) s.put(ranks[i], mine);
        __syncthreads();
        return;
    }
    int N = 4 * kWave;
    while (N < n) N *= 2;
    for (int i = n + threadIdx.x; i < N; i += T) s.put(i, S::none());
    __syncthreads();
    for (int k = 2; k <= N; k *= 2)
        for (int j = k / 2; j > 0; j /= 2) {
            for (int t = threadIdx.x; t < N / 2; t += T) {
                const int i = 2 * t - (t & (j - 1)), o = i + j;                // t's pair, j apart
                const typename S::Item a = s.get(i), b = s.get(o);
                if (S::before(b, a) == ((i & k) == 0)) { s.put(i, b); s.put(o, a); }
            }
            if (j > kWave || (j == 1 && k >= 2 * kWave)) __syncthreads();
            else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
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
