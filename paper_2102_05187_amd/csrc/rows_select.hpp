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

// The rank of every key among n in LDS (all different), each counted by one or several threads; ranks[] is LDS too.
template <int T> __device__ __forceinline__ void rank_keys(const uint64_t *keys, int n, int *ranks) {
    const int wide = n > 0 ? (n + kWave - 1) & ~(kWave - 1) : kWave;          // threads of one part
    const int parts = wide >= T ? 1 : T / wide;
    for (int i = threadIdx.x; i < n; i += T) ranks[i] = 0;
    __syncthreads();
    if (parts == 1) {
        for (int i = threadIdx.x; i < n; i += T) {
            const uint64_t key = keys[i];
            int at = 0;
#pragma unroll 8
            for (int j = 0; j < n; ++j) at += keys[j] > key;
            ranks[i] = at;
        }
    } else {
        const int part = threadIdx.x / wide, i = threadIdx.x - part * wide, per = (n + parts - 1) / parts;
        const int j0 = part * per, j1 = j0 + per < n ? j0 + per : n;
        if (part < parts && i < n) {
            const uint64_t key = keys[i];
            int at = 0;
#pragma unroll 8
            for (int j = j0; j < j1; ++j) at += keys[j] > key;
            if (at) atomicAdd(&ranks[i], at);
        }
    }
    __syncthreads();
}

}  // namespace comet
