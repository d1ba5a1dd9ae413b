// Choosing the K largest of what a workgroup's threads hold in registers.
#pragma once

#include "rows.hpp"

namespace comet {

constexpr int kCandidates = 2048;         // keys that a workgroup keeps in LDS
constexpr int kTries = 64;                // counts of halvings of a range

// One count over the workgroup: every thread's n, added up (n is up to a few dozen; `slot` was 0).
template <int T> __device__ __forceinline__ int block_count(int n, int *slot) {
    if (__ballot(n != 0)) {
        const int sum = (int)wave_reduce((float)n, 0.f, Add());               // whole numbers far below 2^24
        if ((threadIdx.x & (kWave - 1)) == 0) atomicAdd(slot, sum);
    }
    lds_barrier();
    return *slot;
}

constexpr int kBins = 512;

// A value that at least K of the held numbers reach and not many more: those between `lo` and `hi` (the largest) are counted in 256 bins, by
// value first, where the bins' width and its inverse are ordinary numbers, then, while more than 1.25 K + 4 reach the bin that the K-th largest
// is in, by their order inside of that bin (each time a 256th of the range, so that outliers do no harm).  EACH(f) calls f with every number of
// the thread; those below lo are not counted.  Elements below the value that comes back cannot be among the K largest of the workgroup's where
// each number is one of them.  Where fewer than K numbers are counted it is the lowest there is.  The same for all threads.  `bins`: kBins
// places of LDS that hold 0 and have been since a barrier.
template <int T, class EACH> __device__ __forceinline__ float bound(float lo, float hi, int K, EACH each, int *bins) {
    constexpr int B = kBins / 2;
    const int lane = threadIdx.x & (kWave - 1), most = K + K / 4 + 4;
    const float everything = -3.402823466e38f;
    uint32_t from = order_of(lo), to = order_of(hi);
    bool by_value = hi - lo > 1e-30f && hi - lo < __builtin_huge_valf();
    for (int round = 0; round < 6; ++round) {
        int *bin = bins + (round & 1) * B;
        const float per = (float)B / (hi - lo);
        const int shift = to - from < (uint32_t)B ? 0 : 24 - __builtin_clz(to - from);
        if (round > 0) {
            lds_barrier();                                                   // the other half has been read
            for (int i = threadIdx.x; i < B; i += T) bin[i] = 0;
            lds_barrier();
        }
        each([&](float x) {
            if (!(x >= lo)) return;
            const float at = (x - lo) * per;
            const uint32_t step = (order_of(x) - from) >> shift;
            const int i = by_value ? (at < (float)(B - 1) ? (int)at : B - 1) : (step < (uint32_t)B ? (int)step : B - 1);
            atomicAdd(&bin[i], 1);
        });
        lds_barrier();
        // every wavefront by itself, the highest bins first
        const int4 c = ((const int4 *)bin)[kWave - 1 - lane];
        const int sum = c.x + c.y + c.z + c.w;
        int upto = sum;
        upto += __builtin_amdgcn_update_dpp(0, upto, 0x111, 0xf, 0xf, false);
        upto += __builtin_amdgcn_update_dpp(0, upto, 0x112, 0xf, 0xf, false);
        upto += __builtin_amdgcn_update_dpp(0, upto, 0x114, 0xf, 0xf, false);
        upto += __builtin_amdgcn_update_dpp(0, upto, 0x118, 0xf, 0xf, false);
        upto += __builtin_amdgcn_update_dpp(0, upto, 0x142, 0xa, 0xf, false);
        upto += __builtin_amdgcn_update_dpp(0, upto, 0x143, 0xc, 0xf, false);
        const uint64_t hit = __ballot(upto >= K);
        if (!hit) return round == 0 ? everything : lo;
        int reach = upto - sum + c.w, k = 3;
        if (reach < K) reach += c.z, k = 2;
        if (reach < K) reach += c.y, k = 1;
        if (reach < K) reach += c.x, k = 0;
        const int first = __builtin_ctzll(hit);
        reach = __builtin_amdgcn_readlane(reach, first);
        const int b = 4 * (kWave - 1 - first) + __builtin_amdgcn_readlane(k, first);
        if (by_value) {
            // a hundredth of a bin more on either side: (x - lo) * per rounds
            const float width = (hi - lo) / (float)B, top = hi;
            if (b < B - 1) hi = fminf(lo + ((float)b + 1.01f) * width, top);
            lo = fmaxf(lo, lo + ((float)b - 0.01f) * width);
            from = order_of(lo), to = order_of(hi);
            by_value = false;
        } else {
            if (b < B - 1) to = from + ((uint32_t)b << shift) + ((1u << shift) - 1);
            from += (uint32_t)b << shift;
            lo = value_of(from), hi = value_of(to);
        }
        if (reach <= most || from >= to) break;
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
    static __device__ __forceinline__ Item of_lane(Item a, int lane) {
        return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(a >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)a, lane);
    }
    static constexpr bool kEven = false;  // whether rough values are spread evenly
    static __device__ __forceinline__ float rough(Item a) { return finite(value_of((uint32_t)(a >> 32))); }
};
// ... keys whose upper half is a number ...
struct NumberKeys : Keys {
    static constexpr bool kEven = true;
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
    static __device__ __forceinline__ Item of_lane(Item a, int lane) { return Item{Keys::of_lane(a.high, lane), Keys::of_lane(a.low, lane)}; }
    static constexpr bool kEven = false;
    static __device__ __forceinline__ float rough(Item a) { return finite((float)score_of(a.high)); }
};

constexpr int kCrowd = 64;                // more than these in one bin: the bins are of no use
struct SortSpace {
    int count[kBins];                     // items of a bin, then the items in the bins above it
    int size[kBins];
    uint16_t order[kCandidates];          // items bin by bin
    float ends[3][16];
    int crowd;
};

// Calls emit(rank, item) once for each of n different items in LDS (n <= kCandidates; places up to the next power of two are used too), when
// all have been read.  Up to 16 are compared with each other by one wavefront, up to 128 by several threads for each.  More are put
// into 512 bins by their rough value, and compared with the others of their bin; of the largest of many numbers the number falls off exponentially with the value, so the
// bins are even in 1 - exp(-(value - least) / mean).  That this never puts a larger value below a smaller one rests on the device's exp2 never
// being larger for a smaller argument: it is not, for any two neighbouring 32-bit arguments up to 0.  Where the values crowd in a bin (equal
// ones, outliers), a bitonic network sorts them.
template <int T, class S, class EMIT> __device__ __forceinline__ void sort_items(const S &s, int n, SortSpace &sp, EMIT emit) {
    constexpr int E = kCandidates / T;                                         // items of a thread
    using Item = typename S::Item;
    if (n <= 16) {
        if (threadIdx.x < kWave) {
            const bool there = (int)threadIdx.x < n;
            Item mine{};
            if (there) mine = s.get(threadIdx.x);
            int at = 0;
            for (int j = 0; j < n; ++j) at += S::before(S::of_lane(mine, j), mine) ? 1 : 0;
            if (there) emit(at, mine);
        }
        return;
    }
    if (n <= 2 * kWave) {
        const int wide = n <= kWave ? kWave : 2 * kWave, parts = T / wide;     // threads of one part
        const int part = threadIdx.x / wide, i = threadIdx.x - part * wide, per = (n + parts - 1) / parts;
        const int j0 = part * per, j1 = j0 + per < n ? j0 + per : n;
        if (threadIdx.x < 2 * kWave) sp.count[threadIdx.x] = 0;
        Item mine{};
        if (i < n) mine = s.get(i);
        lds_barrier();
        if (i < n) {
            int at = 0;
#pragma unroll 4
            for (int j = j0; j < j1; ++j) at += S::before(s.get(j), mine) ? 1 : 0;
            if (at) atomicAdd(&sp.count[i], at);
        }
        lds_barrier();
        if (part == 0 && i < n) emit(sp.count[i], mine);
        return;
    }
    for (int i = threadIdx.x; i < kBins; i += T) sp.count[i] = 0;
    if (threadIdx.x == 0) sp.crowd = 0;
    Item mine[E];
    float least = -kNegInf, most = kNegInf, sum = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int i = e * T + threadIdx.x;
        if (i >= n) continue;
        mine[e] = s.get(i);
        const float x = S::rough(mine[e]);
        least = fminf(least, x), most = fmaxf(most, x), sum += x * (1.f / kCandidates);
    }
    least = wave_reduce(least, -kNegInf, Smaller());
    most = wave_reduce(most, kNegInf, Larger());
    sum = wave_reduce(sum, 0.f, Add());
    if ((threadIdx.x & (kWave - 1)) == 0) {
        const int w = threadIdx.x / kWave;
        sp.ends[0][w] = least, sp.ends[1][w] = most, sp.ends[2][w] = sum;
    }
    lds_barrier();
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < T / kWave; ++w) least = fminf(least, sp.ends[0][w]), most = fmaxf(most, sp.ends[1][w]), sum += sp.ends[2][w];
    const float mean = sum * ((float)kCandidates / (float)n) - least;
    const float per = S::kEven ? (float)(kBins - 1) / fmaxf(most - least, 1e-30f) : -kLog2e / fmaxf(mean, 1e-30f);
    int bin[E], slot[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int i = e * T + threadIdx.x;
        if (i >= n) continue;
        const float x = (S::rough(mine[e]) - least) * per;
        const float b = S::kEven ? x : (float)kBins * (1.f - exp2_fast(x));
        bin[e] = b < (float)(kBins - 1) ? (int)b : kBins - 1;                  // NaN: the last one
        slot[e] = atomicAdd(&sp.count[bin[e]], 1);
    }
    lds_barrier();
    if (threadIdx.x < kWave) {                                                 // count[b]: items in the bins above b
        constexpr int B = kBins / kWave;
        const int last = kBins - 1 - (int)threadIdx.x * B;
        int c[B], mine_sum = 0, crowd = 0;
#pragma unroll
        for (int k = 0; k < B; ++k) c[k] = sp.count[last - k], mine_sum += c[k], crowd |= c[k] > kCrowd;
        int before = mine_sum;
        before += __builtin_amdgcn_update_dpp(0, before, 0x111, 0xf, 0xf, false);
        before += __builtin_amdgcn_update_dpp(0, before, 0x112, 0xf, 0xf, false);
        before += __builtin_amdgcn_update_dpp(0, before, 0x114, 0xf, 0xf, false);
        before += __builtin_amdgcn_update_dpp(0, before, 0x118, 0xf, 0xf, false);
        before += __builtin_amdgcn_update_dpp(0, before, 0x142, 0xa, 0xf, false);
        before += __builtin_amdgcn_update_dpp(0, before, 0x143, 0xc, 0xf, false);
        before -= mine_sum;
#pragma unroll
        for (int k = 0; k < B; ++k) sp.count[last - k] = before, sp.size[last - k] = c[k], before += c[k];
        if (crowd) sp.crowd = 1;
    }
    lds_barrier();
    if (sp.crowd) {
        int N = 4 * kWave;
        while (N < n) N *= 2;
        for (int i = n + threadIdx.x; i < N; i += T) s.put(i, S::none());
        lds_barrier();
        // steps over distances of up to 64 stay inside of a wavefront's 128 items and need no barrier
        for (int k = 2; k <= N; k *= 2)
            for (int j = k / 2; j > 0; j /= 2) {
                for (int t = threadIdx.x; t < N / 2; t += T) {
                    const int i = 2 * t - (t & (j - 1)), o = i + j;            // t's pair, j apart
                    const Item a = s.get(i), b = s.get(o);
                    if (S::before(b, a) == ((i & k) == 0)) { s.put(i, b); s.put(o, a); }
                }
                if (j > kWave || (j == 1 && k >= 2 * kWave)) lds_barrier();
                else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            }
#pragma unroll
        for (int e = 0; e < E; ++e) if (e * T + (int)threadIdx.x < n) mine[e] = s.get(e * T + threadIdx.x), bin[e] = e * T + threadIdx.x;
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int i = e * T + threadIdx.x;
            if (i >= n) continue;
            sp.order[sp.count[bin[e]] + slot[e]] = (uint16_t)i;
        }
        lds_barrier();
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (e * T + (int)threadIdx.x >= n) continue;
            const int first = sp.count[bin[e]], end = first + sp.size[bin[e]];
            int at = first;
#pragma unroll 4
            for (int p = first; p < end; ++p) at += S::before(s.get(sp.order[p]), mine[e]) ? 1 : 0;
            bin[e] = at;
        }
    }
    lds_barrier();
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (e * T + (int)threadIdx.x < n) emit(bin[e], mine[e]);
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
    lds_barrier();
    for (int i = threadIdx.x; i < kTries; i += T) tries[i] = 0;
    lds_barrier();
    return lo;
}

}  // namespace comet
