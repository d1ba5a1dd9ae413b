// The K largest elements of dense rows, with the rows' log-sum-exp.
//
// A workgroup reads a piece of a row once (up to 256 KB; rows beyond that, and those of beams that are too few to fill the device, are cut
// into several pieces whose results a second kernel joins) and keeps of every vector of 16 bytes its largest element in a register.
// From these:
//   1. a bound that K to 1.25 K of the threads' largest elements reach (bound()): of a row in no particular order about
//      K (1 + K / 2T) elements reach it, of T threads; all others are out;
//   2. the vectors whose largest element reaches it are listed and read again, K or so of them, and their elements that do go
//      into LDS as 64-bit keys (value, then lower column);
//   3. the keys are put in order (sort_items()).
// Bound by memory where rows are long and many: top 64 of 2048 x 131072 of 16 bits in 95.6 us, 5.6 TB/s (a plain read of
// that size 7.1).  Few rows are bound by the latency of these steps: 8 us of one row of 32000 32-bit elements, 13 of 131072 of 16 bits.  Of a
// workgroup's time over a row of 60013 of 16 bits with K = 500, reading and summing take 37 %, the bound 10 %, the list 5 %, reading its 600 vectors
// again 23 %, the order 25 %; of 32000 of 32 bits with K = 50 58, 15, 7, 8 and 12 %.  Shapes of more threads with fewer vectors each were
// slower throughout (1024 threads: 146 us, and 13 for 11.5 with 4 rows).
// Where more than 2048 reach the bound (equal elements, or the large ones next to each other in a few threads) the K-th largest key is
// found exactly, by halving, with the vectors that matter read again each time.  That is slow: rows of equal elements take 2.8 ms for 0.1 at 2048 x
// 131072 with K = 64, 0.34 ms for 0.01 at 1 x 32000; and so do rows with fewer than K allowed elements above a finite mask (2.7 and 0.28 ms), which
// a mask of -inf does not (0.097 and 0.01).
#include "rows_kernels.hpp"
#include "rows_select.hpp"

namespace comet {

namespace {

struct TopArgs {
    const void *Z;
    int64_t V, ldz;
    float c2;                             // scale log2(e)
    double scale;
    int K, splits;
    bool by_coordinate, once, shift;      // once, shift: how rows are read
    int32_t *crd;                         // results, where a row is one piece and no keys are asked for
    float *vals, *lse;
    const uint8_t *finished;
    int32_t eos;
    uint64_t *keys;                       // [rows x splits x K], largest first, 0 where there are fewer
    float2 *sums;                         // [rows x splits] running maximum and sum
};

struct TopShared {
    uint64_t keys[kCandidates];
    SortSpace sort;
    int tries[kTries];
    float2 buf[16];
    float ends[16];
    int found, listed;
};

// The n keys that were found become the row's result: places 0 .. K-1 of the row, by value or by coordinate.
template <int T> __device__ __forceinline__ void write_row(TopShared &sh, int n, int K, bool by_coordinate, int32_t *crd, float *vals) {
    const int kept = n < K ? n : K;
    if (by_coordinate) {
        // the kept keys again, with the coordinate as the order: its complement is a key's low half
        if (n > K || K > kWave) {
            sort_items<T>(Keys{sh.keys}, n, sh.sort, [&](int rank, uint64_t key) { if (rank < K) sh.keys[rank] = key << 32 | key >> 32; });
        } else if (threadIdx.x < kWave && (int)threadIdx.x < n) sh.keys[threadIdx.x] = sh.keys[threadIdx.x] << 32 | sh.keys[threadIdx.x] >> 32;
        lds_barrier();
        sort_items<T>(NumberKeys{sh.keys}, kept, sh.sort, [&](int rank, uint64_t key) {
            crd[rank] = (int32_t)column_of(key >> 32);
            vals[rank] = value_of((uint32_t)key);
        });
    } else {
        sort_items<T>(Keys{sh.keys}, n, sh.sort, [&](int rank, uint64_t key) {
            if (rank >= K) return;
            crd[rank] = (int32_t)column_of(key);
            vals[rank] = value_of_key(key);
        });
    }
    for (int i = kept + threadIdx.x; i < K; i += T) crd[i] = -1, vals[i] = kNegInf;
}
// ... or a list of K keys, 0 at its end where there are fewer.
template <int T> __device__ __forceinline__ void write_keys(TopShared &sh, int n, int K, uint64_t *keys) {
    sort_items<T>(Keys{sh.keys}, n, sh.sort, [&](int rank, uint64_t key) { if (rank < K) keys[rank] = key; });
    for (int i = n + threadIdx.x; i < K; i += T) keys[i] = 0;
}
// A row's log-sum-exp.
__device__ __forceinline__ float lse_of(const MaxSum &a, double scale) {
    if (fabsf(a.m) == -kNegInf && a.s == a.s) return a.m;
    return (float)((double)a.m * scale + log_of(a.s));
}

// A piece of a row: vectors [piece * T * NV, ..), vector j of thread t at j * T + t.
template <int TYPE, int T, int NV>
__global__ void __launch_bounds__(T, 4) k_rows_topk(TopArgs a) {
    using E = Elem<TYPE>;
    constexpr int P = E::kPer, U = NV < 4 ? NV : 4;          // vectors that a thread has in flight
    __shared__ TopShared sh;
    const int64_t piece = blockIdx.x, r = piece / a.splits;
    const int split = (int)(piece - r * a.splits), K = a.K;
    if (a.keys && a.finished && a.finished[r]) {             // an ended beam: one candidate, whatever its row holds
        for (int i = threadIdx.x; i < K; i += T) a.keys[piece * K + i] = i == 0 && split == 0 ? key_of(0.f, (uint32_t)a.eos) : 0;
        if (threadIdx.x == 0) a.sums[piece] = make_float2(split == 0 ? 0.f : kNegInf, split == 0 ? 1.f : 0.f);
        return;
    }
    const Row<TYPE> row(a.Z, r, a.ldz, a.V, a.shift);
    const int64_t v0 = (int64_t)split * T * NV, full = row.n / P;
    const int own = (int)(full - v0 < T * NV ? full - v0 : T * NV);           // whole vectors of this piece
    const bool ends_here = row.n % P != 0 && full >= v0 && full < v0 + T * NV;    // ... and the one that the row ends in: thread 0's
    for (int i = threadIdx.x; i < kBins; i += T) sh.sort.count[i] = 0;
    if (threadIdx.x < kTries) sh.tries[threadIdx.x] = 0;
    if (threadIdx.x == 0) sh.found = 0, sh.listed = 0;
    float top[NV], last = kNegInf;                           // `last`: of the row's last, shorter vector
    Running run;
    uint4 v[U];
    auto fetch = [&](int j0) {
        if ((j0 + U) * T <= own && a.once) {
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = row.template stream<true>(v0 + (j0 + u) * T + threadIdx.x);
        } else if ((j0 + U) * T <= own) {
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = row.template stream<false>(v0 + (j0 + u) * T + threadIdx.x);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = (j0 + u) * T + threadIdx.x;
                v[u] = make_uint4(E::kNone, E::kNone, E::kNone, E::kNone);
                if (i < own) v[u] = row.template stream<false>(v0 + i);
            }
        }
    };
    const auto edge = row.template edges<T>(v0, own);
    fetch(0);
#pragma unroll
    for (int j0 = 0; j0 < NV; j0 += U) {
        if (j0 * T >= own) {                                 // the row has ended
#pragma unroll
            for (int u = 0; u < U; ++u) top[j0 + u] = kNegInf;
            continue;
        }
        uint4 w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = v[u];
        if (j0 + U < NV && (j0 + U) * T < own) fetch(j0 + U);
        if (row.odd) {
#pragma unroll
            for (int u = 0; u < U; ++u) w[u] = row.settle(w[u], edge, j0 + u, (j0 + u) * T + threadIdx.x, own);
        }
        if constexpr (NV <= U) {                             // kept for later
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = w[u];
        }
        float f[U * P], b = kNegInf;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            E::widen(w[u], f + u * P);
            float t = f[u * P];
#pragma unroll
            for (int k = 1; k < P; ++k) t = fmaxf(t, f[u * P + k]);
            top[j0 + u] = t;
            b = fmaxf(b, t);
        }
        run.template take<U * P>(f, b, a.c2);
    }
    if (ends_here && threadIdx.x == 0) {
        float f[P];
        row.load(full, f);
        last = f[0];
#pragma unroll
        for (int k = 1; k < P; ++k) last = fmaxf(last, f[k]);
        run.template take<P>(f, last, a.c2);
    }
    const float m = run.m;
    MaxSum sum = run.sum(a.c2);
    // 1: the bound, from the threads' largest elements, or those of eighths of their vectors where K is more than half of the threads
    constexpr int G = NV < 8 ? NV : 8;
    const bool few = K <= T / 2;
    const auto numbers = [&](auto f) {
        if (few) f(m);
        else {
#pragma unroll
            for (int g = 0; g < G; ++g) {
                float t = top[g];
#pragma unroll
                for (int j = g + G; j < NV; j += G) t = fmaxf(t, top[j]);
                f(t);
            }
            f(last);
        }
    };
    float least = -kNegInf;
    numbers([&](float x) { least = fminf(least, x > kNegInf ? x : -kNegInf); });
    least = wave_reduce(least, -kNegInf, Smaller());
    if ((threadIdx.x & (kWave - 1)) == 0) sh.ends[threadIdx.x / kWave] = least;
    block_join<T>(sum, a.c2, sh.buf);                        // also makes bins, tries, found and ends visible
    if (wild(sum.m, a.c2)) sum.s = slow_sum<TYPE, T>(row, v0 * P, (v0 + T * NV) * P, sum.m, a.c2, sh.buf, [](int64_t) { return false; });
    if (threadIdx.x == 0) {
        if (a.sums) a.sums[piece] = make_float2(sum.m, sum.s);
        else if (a.lse) a.lse[r] = lse_of(sum, a.scale);
    }
#pragma unroll
    for (int w = 0; w < T / kWave; ++w) least = fminf(least, sh.ends[w]);
    float from = -3.402823466e38f;                           // nothing that can be kept is below it
    if (sum.m > kNegInf && (few || T * NV * P > kCandidates)) from = bound<T>(least, sum.m, K, [&](auto f) { numbers([&](float x) { if (x > kNegInf) f(x); }); }, sh.sort.count);
    // 2: every vector with an element from a value (above -inf) on; whole wavefronts, the next vector on its way while one is looked at
    auto each = [&](float from, auto use) {
        uint32_t which = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j) which |= top[j] >= from ? 1u << j : 0u;
        bool end = last >= from;
        const auto next = [&](int64_t &i, uint4 &x) {
            i = -1;
            x = make_uint4(E::kNone, E::kNone, E::kNone, E::kNone);
            if (which) {
                i = v0 + __builtin_ctz(which) * T + threadIdx.x;
                which &= which - 1;
                x = row.raw(i);
            } else if (end) {
                i = full;
                end = false;
                float f[P];
                row.load(full, f);
                x = E::narrow(f);
            }
        };
        int64_t i, i2;
        uint4 x, x2;
        next(i, x);
        while (__ballot(i >= 0)) {
            next(i2, x2);
            float f[P];
            E::widen(x, f);
            use(f, (uint32_t)(i * P));
            i = i2, x = x2;
        }
    };
    // The elements of a vector that WANTED names go into LDS.
    const auto keep = [&](const float *f, uint32_t column, auto wanted) {
        int mine = 0;
#pragma unroll
        for (int k = 0; k < P; ++k) mine += wanted(f[k], column + k) ? 1 : 0;
        if (!__ballot(mine != 0)) return;
        int at = append(mine, &sh.found);
#pragma unroll
        for (int k = 0; k < P; ++k)
            if (wanted(f[k], column + k)) {
                if (at < kCandidates) sh.keys[at] = key_of(f[k], column + k);
                ++at;
            }
    };
    const auto reaches = [&](float x, uint32_t) { return x >= from; };
    // The vectors that matter are listed first and then shared out: a thread may hold several of them, and most hold none.  Of a small
    // piece all are still in registers.
    if constexpr (NV <= U) {
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            float f[P];
            E::widen(v[u], f);
            keep(f, (uint32_t)((v0 + u * T + threadIdx.x) * P), reaches);
        }
        if (ends_here && threadIdx.x < kWave) {
            float f[P];
            row.load(full, f);
#pragma unroll
            for (int k = 0; k < P; ++k) f[k] = threadIdx.x == 0 ? f[k] : kNegInf;
            keep(f, (uint32_t)(full * P), reaches);
        }
        lds_barrier();
    } else {
        uint16_t *list = sh.sort.order;
        uint32_t which = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j) which |= top[j] >= from ? 1u << j : 0u;
        int at = append(__popc(which), &sh.listed);
        for (; which; which &= which - 1, ++at)
            if (at < kCandidates) list[at] = (uint16_t)(__builtin_ctz(which) * T + threadIdx.x);
        lds_barrier();
        const int listed = sh.listed;
        if (listed <= kCandidates) {
            constexpr int A = 2;                             // vectors on their way
            for (int i0 = 0; i0 < listed; i0 += A * T) {
                uint4 x[A];
                uint32_t column[A];
#pragma unroll
                for (int q = 0; q < A; ++q) {
                    const int i = i0 + q * T + threadIdx.x;
                    x[q] = make_uint4(E::kNone, E::kNone, E::kNone, E::kNone);
                    column[q] = 0;
                    if (i < listed) {
                        column[q] = (uint32_t)((v0 + list[i]) * P);
                        x[q] = row.raw(v0 + list[i]);
                    }
                }
#pragma unroll
                for (int q = 0; q < A; ++q) {
                    if (i0 + q * T >= listed) break;
                    float f[P];
                    E::widen(x[q], f);
                    keep(f, column[q], reaches);
                }
            }
            if (ends_here && threadIdx.x < kWave) {
                float f[P];
                row.load(full, f);
#pragma unroll
                for (int k = 0; k < P; ++k) f[k] = threadIdx.x == 0 ? f[k] : kNegInf;
                keep(f, (uint32_t)(full * P), reaches);
            }
        } else if (threadIdx.x == 0) sh.found = kCandidates + 1;
        lds_barrier();
    }
    int n = sh.found;
    if (n > kCandidates) {
        // the K-th largest key: all keys are different, so exactly K reach it
        const uint64_t lo = kth<T>((uint64_t)order_of(from) << 32, (uint64_t)order_of(sum.m) << 32 | 0xffffffffu, K, [&](uint64_t t) {
            const float from = value_of((uint32_t)(t >> 32));
            int c = 0;
            each(from, [&](const float *f, uint32_t column) {
#pragma unroll
                for (int k = 0; k < P; ++k) c += f[k] >= from && key_of(f[k], column + k) >= t ? 1 : 0;
            });
            return c;
        }, sh.tries);
        if (threadIdx.x == 0) sh.found = 0;
        lds_barrier();
        const float least = value_of((uint32_t)(lo >> 32));
        each(least, [&](const float *f, uint32_t column) { keep(f, column, [&](float x, uint32_t c) { return x >= least && key_of(x, c) >= lo; }); });
        lds_barrier();
        n = sh.found < kCandidates ? sh.found : kCandidates;
    }
    // 3
    if (a.keys) write_keys<T>(sh, n, K, a.keys + piece * K);
    else write_row<T>(sh, n, K, a.by_coordinate, a.crd + r * K, a.vals + r * K);
}

// Joins the pieces of a row: `splits` lists of K keys, at most T * PER in all, and as many sums.
constexpr int kMerge = 16384;

template <int T, int PER>
__global__ void __launch_bounds__(T) k_topk_merge(TopArgs a, uint64_t *__restrict__ out_keys, float2 *__restrict__ out_sums) {
    __shared__ TopShared sh;
    const int64_t r = blockIdx.x;
    const int K = a.K, total = a.splits * K;
    const uint64_t *from = a.keys + r * total;
    uint64_t key[PER], most = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int i = j * T + threadIdx.x;
        key[j] = i < total ? from[i] : 0;
        most = key[j] > most ? key[j] : most;
    }
    MaxSum sum;
    for (int i = threadIdx.x; i < a.splits; i += T) {
        const float2 p = a.sums[r * a.splits + i];
        sum.join(p.x, p.y, a.c2);
    }
    for (int i = threadIdx.x; i < kBins; i += T) sh.sort.count[i] = 0;
    if (threadIdx.x < kTries) sh.tries[threadIdx.x] = 0;
    if (threadIdx.x == 0) sh.found = 0;
    const float top = most ? value_of_key(most) : kNegInf;
    float least = wave_reduce(most ? top : -kNegInf, -kNegInf, Smaller());
    if ((threadIdx.x & (kWave - 1)) == 0) sh.ends[threadIdx.x / kWave] = least;
    block_join<T>(sum, a.c2, sh.buf);
    if (threadIdx.x == 0) {
        if (out_sums) out_sums[r] = make_float2(sum.m, sum.s);
        else if (a.lse) a.lse[r] = lse_of(sum, a.scale);
    }
#pragma unroll
    for (int w = 0; w < T / kWave; ++w) least = fminf(least, sh.ends[w]);
    float bar = -3.402823466e38f;
    if (sum.m > kNegInf) bar = bound<T>(least, sum.m, K, [&](auto f) { if (most) f(top); }, sh.sort.count);
    uint64_t lo = (uint64_t)order_of(bar) << 32;
    for (int pass = 0;; ++pass) {
        int chosen = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) chosen += key[j] && key[j] >= lo ? 1 : 0;
        int at = append(chosen, &sh.found);
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (key[j] && key[j] >= lo) {
                if (at < kCandidates) sh.keys[at] = key[j];
                ++at;
            }
        lds_barrier();
        if (pass == 1 || sh.found <= kCandidates) break;
        lo = kth<T>(lo, (uint64_t)order_of(sum.m) << 32 | 0xffffffffu, K, [&](uint64_t t) {
            int c = 0;
#pragma unroll
            for (int j = 0; j < PER; ++j) c += key[j] >= t ? 1 : 0;
            return c;
        }, sh.tries);
        if (threadIdx.x == 0) sh.found = 0;
        lds_barrier();
    }
    const int n = sh.found < kCandidates ? sh.found : kCandidates;
    if (out_keys) write_keys<T>(sh, n, K, out_keys + r * K);
    else write_row<T>(sh, n, K, a.by_coordinate, a.crd + r * K, a.vals + r * K);
}

hipError_t merge(const TopArgs &a, int64_t N, uint64_t *out_keys, float2 *out_sums, hipStream_t st) {
    const int total = a.splits * a.K;
    if (total <= 2048) hipLaunchKernelGGL((k_topk_merge<256, 8>), dim3((unsigned)N), dim3(256), 0, st, a, out_keys, out_sums);
    else hipLaunchKernelGGL((k_topk_merge<1024, 16>), dim3((unsigned)N), dim3(1024), 0, st, a, out_keys, out_sums);
    return hipGetLastError();
}

// How rows are cut: workgroups of `threads` with `vectors` vectors in each thread's registers, `splits` of them for a row.
struct Cut { int threads, vectors, splits; };

// The smallest piece that holds a row whole; one workgroup takes a row of 16384 vectors in 13 us alone (131072 elements of 16 bits), and a second
// launch that joins pieces costs 4 to 5 more than pieces save: 16 such rows take 15 us whole and 17 to 25 cut, one row of 32000
// 32-bit elements 9 whole and 13 or more cut.
Cut cut_rows(int type, int64_t V) {
    const int64_t per = type == COMET_F32 ? 4 : 8, nv = (V + per - 1) / per;
    const int sizes[][2] = {{256, 1}, {256, 2}, {256, 4}, {256, 8}, {256, 16}, {256, 32}, {512, 32}};
    for (const auto &s : sizes)
        if (nv <= s[0] * s[1]) return Cut{s[0], s[1], 1};
    // Of the two largest pieces the smaller where fewer of its places stay empty (4096 x 131074 of 16 bits: 214 us in 3 pieces, 294 in 2).  Of
    // many pieces the larger: their number times K, 1024 at most, has to stay below kMerge.
    const int64_t large = (nv + 16383) / 16384, small = (nv + 8191) / 8192;
    return small < 2 * large && small <= 16 ? Cut{256, 32, (int)small} : Cut{512, 32, (int)large};
}

// Where a row's pieces are joined with those of other rows anyway, a cut costs nothing: pieces get smaller until 512 of them are there, or
// `together` rows' lists are more than the 1024 keys that are joined fastest.
Cut cut_lists(int type, int64_t N, int64_t V, int64_t K, int64_t together) {
    const int64_t per = type == COMET_F32 ? 4 : 8, nv = (V + per - 1) / per;
    Cut best = cut_rows(type, V);
    const int sizes[][2] = {{256, 32}, {256, 16}, {256, 8}, {256, 4}, {256, 2}, {256, 1}};
    for (const auto &s : sizes) {
        const int64_t piece = (int64_t)s[0] * s[1], splits = (nv + piece - 1) / piece;
        if (piece >= (int64_t)best.threads * best.vectors) continue;
        if (N * best.splits >= 512 || together * splits * K > 1024) break;
        best = Cut{s[0], s[1], (int)splits};
    }
    return best;
}

template <int TYPE> hipError_t launch(const Cut &c, const TopArgs &a, int64_t N, hipStream_t st) {
    const auto kernel = c.threads == 512 ? k_rows_topk<TYPE, 512, 32> : c.vectors == 32 ? k_rows_topk<TYPE, 256, 32>
                      : c.vectors == 16 ? k_rows_topk<TYPE, 256, 16> : c.vectors == 8 ? k_rows_topk<TYPE, 256, 8>
                      : c.vectors == 4 ? k_rows_topk<TYPE, 256, 4> : c.vectors == 2 ? k_rows_topk<TYPE, 256, 2> : k_rows_topk<TYPE, 256, 1>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(N * a.splits)), dim3(c.threads), 0, st, a);
    return hipGetLastError();
}
hipError_t launch(int type, const Cut &c, const TopArgs &a, int64_t N, hipStream_t st) {
    return type == COMET_F32 ? launch<COMET_F32>(c, a, N, st) : type == COMET_BF16 ? launch<COMET_BF16>(c, a, N, st) : launch<COMET_F16>(c, a, N, st);
}

int64_t round16(int64_t b) { return (b + 15) / 16 * 16; }

}  // namespace

int64_t rows_topk_work(int type, int64_t N, int64_t V, int64_t K) {
    const Cut c = cut_rows(type, V);
    return c.splits == 1 ? 0 : round16(N * c.splits * (int64_t)sizeof(float2)) + N * c.splits * K * (int64_t)sizeof(uint64_t);
}

hipError_t rows_topk(const void *Z, int type, int64_t N, int64_t V, int64_t ldz, double scale, int64_t K, bool by_coordinate,
                     int32_t *crd, float *vals, float *lse, void *work, hipStream_t st) {
    const Cut c = cut_rows(type, V);
    TopArgs a{Z, V, ldz, (float)(scale * 1.4426950408889634), scale, (int)K, c.splits, by_coordinate, read_once(type, N, V), read_shifted(type, N, V), crd, vals, lse, nullptr, 0, nullptr, nullptr};
    if (c.splits > 1) {
        a.sums = (float2 *)work;
        a.keys = (uint64_t *)((char *)work + round16(N * c.splits * (int64_t)sizeof(float2)));
    }
    const hipError_t e = launch(type, c, a, N, st);
    if (e != hipSuccess || c.splits == 1) return e;
    return merge(a, N, nullptr, nullptr, st);
}

TopLists rows_top_lists(int type, int64_t N, int64_t V, int64_t K, int64_t together) {
    TopLists l;
    l.lists = cut_lists(type, N, V, K, together).splits;
    l.joined = l.lists > 1 && together * l.lists * K > kMerge;
    const int64_t pieces = N * l.lists;
    l.sums = round16(pieces * (int64_t)sizeof(float2));
    l.bytes = l.sums + pieces * K * (int64_t)sizeof(uint64_t);
    if (l.joined) {
        l.at = round16(l.bytes);
        l.lists = 1;
        l.sums = round16(N * (int64_t)sizeof(float2));
        l.bytes = l.at + l.sums + N * K * (int64_t)sizeof(uint64_t);
    }
    return l;
}

hipError_t rows_top_keys(const void *Z, int type, int64_t N, int64_t V, int64_t ldz, int64_t K, int64_t together, const TopLists &l, const uint8_t *finished, int32_t eos,
                         void *work, hipStream_t st) {
    const Cut c = cut_lists(type, N, V, K, together);
    const TopArgs a{Z, V, ldz, kLog2e, 1.0, (int)K, c.splits, false, read_once(type, N, V), read_shifted(type, N, V), nullptr, nullptr, nullptr, finished, eos,
                    (uint64_t *)((char *)work + round16(N * c.splits * (int64_t)sizeof(float2))), (float2 *)work};
    const hipError_t e = launch(type, c, a, N, st);
    if (e != hipSuccess || !l.joined) return e;
    char *to = (char *)work + l.at;
    return merge(a, N, (uint64_t *)(to + l.sums), (float2 *)to, st);
}

}  // namespace comet
