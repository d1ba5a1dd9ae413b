// Beam search: selection over beams and vocabulary, and the reordering of the beams' states.
#include "rows_kernels.hpp"
#include "rows_select.hpp"

namespace comet {

namespace {

// A candidate as a number of 128 bits whose order is that of the candidates: the score; then the lower beam, the larger logit, the lower
// token.
__device__ __forceinline__ uint64_t rest_of(uint64_t key, int beam) {
    return (uint64_t)(~beam & 0xff) << 56 | key >> 32 << 24 | ((uint32_t)key & 0xffffff);
}
// The score in 32 bits, above -inf.
__device__ __forceinline__ float rough(uint64_t o) { return finite((float)score_of(o)); }

struct BeamArgs {
    const uint64_t *keys;                 // [B x W x lists x n], each list in order, 0 where there are fewer
    const float2 *sums;                   // [B x W x lists]
    const float *score;
    int W, lists, n;
    float *out_score;
    int32_t *out_parent, *out_token;
};

// One workgroup a batch: the n best of all its lists' keys, T * PER at most, which the threads hold as scores.  Bound by the latency of its steps, one
// after the other (two reads, log-sum-exps, bound, list, order): 5 us for up to 1024 keys, whatever their number and that of the batches, of the 16
// that the call takes; the kernel before it takes 5 to 12, the host the rest.
template <int T, int PER>
__global__ void __launch_bounds__(T) k_beam_join(BeamArgs a) {
    __shared__ double big[COMET_MAX_BEAMS], off[COMET_MAX_BEAMS];       // a candidate's score is (z - big) + off
    __shared__ uint64_t high[kCandidates], low[kCandidates];
    __shared__ SortSpace sort;
    __shared__ int tries[kTries], found;
    __shared__ float ends[2][T / kWave];
    const int64_t b = blockIdx.x;
    const int n = a.n, total = a.W * a.lists * n, per_beam = a.lists * n;
    const uint64_t *keys = a.keys + b * total;
    uint64_t key[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int i = j * T + threadIdx.x;
        key[j] = i < total ? keys[i] : 0;
    }
    for (int w = threadIdx.x; w < a.W; w += T) {
        MaxSum sum;
#pragma unroll 4
        for (int l = 0; l < a.lists; ++l) {
            const float2 p = a.sums[(b * a.W + w) * a.lists + l];
            sum.join(p.x, p.y, kLog2e);
        }
        big[w] = sum.s != sum.s ? (double)sum.s : (double)sum.m;
        off[w] = (double)a.score[b * a.W + w] - log_of(sum.s);
    }
    for (int i = threadIdx.x; i < kBins; i += T) sort.count[i] = 0;
    if (threadIdx.x < kTries) tries[threadIdx.x] = 0;
    if (threadIdx.x == 0) found = 0;
    lds_barrier();
    uint64_t s[PER], most = 0;                                           // orders of the scores, 0: no candidate
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int w = (j * T + (int)threadIdx.x) / per_beam;
        const double x = key[j] ? ((double)value_of_key(key[j]) - big[w]) + off[w] : kNegInfD;
        s[j] = x > kNegInfD ? order64(x) : 0;
        most = s[j] > most ? s[j] : most;
    }
    const float best = most ? rough(most) : kNegInf;
    const float least = wave_reduce(most ? best : -kNegInf, -kNegInf, Smaller());
    const float largest = wave_reduce(best, kNegInf, Larger());
    if ((threadIdx.x & (kWave - 1)) == 0) ends[0][threadIdx.x / kWave] = least, ends[1][threadIdx.x / kWave] = largest;
    lds_barrier();
    float from = ends[0][0], to = ends[1][0];
#pragma unroll
    for (int w = 1; w < T / kWave; ++w) from = fminf(from, ends[0][w]), to = fmaxf(to, ends[1][w]);
    float bar = kNegInf;                                                 // scores below it are out
    if (to > kNegInf) bar = bound<T>(from, to, n, [&](auto f) { if (most) f(best); }, sort.count);
    uint64_t bar64 = 0, bar_rest = 0;                                    // ... and those below this one, once it is known
    for (int pass = 0;; ++pass) {
        const auto chosen = [&](int j, uint64_t rest) {
            return s[j] && rough(s[j]) >= bar && (s[j] > bar64 || (s[j] == bar64 && rest >= bar_rest));
        };
        int mine = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) mine += chosen(j, rest_of(key[j], (j * T + (int)threadIdx.x) / per_beam)) ? 1 : 0;
        int at = append(mine, &found);
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const uint64_t rest = rest_of(key[j], (j * T + (int)threadIdx.x) / per_beam);
            if (chosen(j, rest)) {
                if (at < kCandidates) high[at] = s[j], low[at] = rest;
                ++at;
            }
        }
        lds_barrier();
        if (pass == 1 || found <= kCandidates) break;
        // many equal ones: the n-th largest score exactly, and of the candidates that have it as many as are missing
        bar64 = kth<T>(1, order64(-kNegInfD), n, [&](uint64_t t) {
            int c = 0;
#pragma unroll
            for (int j = 0; j < PER; ++j) c += s[j] >= t ? 1 : 0;
            return c;
        }, tries);
        int above = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) above += s[j] > bar64 ? 1 : 0;
        above = block_count<T>(above, &tries[0]);
        lds_barrier();
        if (threadIdx.x == 0) tries[0] = 0;
        lds_barrier();
        bar_rest = kth<T>(0, ~0ull, n - above, [&](uint64_t t) {
            int c = 0;
#pragma unroll
            for (int j = 0; j < PER; ++j) c += s[j] == bar64 && rest_of(key[j], (j * T + (int)threadIdx.x) / per_beam) >= t ? 1 : 0;
            return c;
        }, tries);
        if (threadIdx.x == 0) found = 0;
        lds_barrier();
    }
    const int some = found < kCandidates ? found : kCandidates;
    sort_items<T>(WideKeys{high, low}, some, sort, [&](int rank, const WideKey &c) {
        if (rank >= n) return;
        a.out_score[b * n + rank] = (float)score_of(c.high);
        a.out_parent[b * n + rank] = (int32_t)(~(c.low >> 56) & 0xff);
        a.out_token[b * n + rank] = (int32_t)(~(uint32_t)c.low & 0xffffff);
    });
    for (int i = some + threadIdx.x; i < n; i += T) {
        a.out_score[b * n + i] = kNegInf;
        a.out_parent[b * n + i] = -1;
        a.out_token[b * n + i] = -1;
    }
}

constexpr int kStates = 64;               // state arrays of one launch
struct StatePointers { char *p[kStates]; };

template <class U> __device__ __forceinline__ void put_once(char *to, const U &u) { *(U *)to = u; }
template <> __device__ __forceinline__ void put_once<uint4>(char *to, const uint4 &u) {
    typedef uint32_t v4 __attribute__((ext_vector_type(4)));
    const v4 v = {u.x, u.y, u.z, u.w};
    __builtin_nontemporal_store(v, (v4 *)to);
}

// A thread moves the same unit of all beams of a batch: all are read into LDS before the first is written.  Bound by memory; what it has in
// flight is set by LDS, and less of it is better than more: beams lie at large powers of two from each other, and the more of their
// rows are open at once the worse.  8 batches of 8 beams, 5 of them moved, 4.7 GB read and written: 128 threads (16 KB) with stores past the
// caches 803 us, 256 threads 820, 512 threads 854, stores through the caches 823, units in registers at full occupancy 921.
constexpr int kMoveThreads = 128;
template <class U>
__global__ void __launch_bounds__(kMoveThreads) k_beam_reorder(StatePointers states, StateLayout l, const int32_t *__restrict__ parent) {
    extern __shared__ __align__(16) char raw[];
    U *tile = (U *)raw + threadIdx.x;
    const int W = (int)l.W, T = blockDim.x;
    const int64_t b = blockIdx.y, units = l.inner / (int64_t)sizeof(U), all = units * l.outer;
    char *base = states.p[blockIdx.z] + b * l.batch_stride;
    const int32_t *par = parent + b * W;
    for (int64_t u = (int64_t)blockIdx.x * T + threadIdx.x; u < all; u += (int64_t)gridDim.x * T) {
        const int64_t o = l.outer == 1 ? 0 : u / units;
        char *at = base + o * l.outer_stride + (u - o * units) * (int64_t)sizeof(U);
        for (int w = 0; w < W; ++w) {
            const int p = par[w];
            if (p >= 0 && p < W && p != w) tile[w * T] = *(const U *)(at + p * l.beam_stride);
        }
        for (int w = 0; w < W; ++w) {
            const int p = par[w];
            if (p >= 0 && p < W && p != w) put_once<U>(at + w * l.beam_stride, tile[w * T]);
        }
    }
}

}  // namespace

int64_t beam_select_work(int type, int64_t B, int64_t W, int64_t V, int64_t n) { return rows_top_lists(type, B * W, V, n, W).bytes; }

hipError_t beam_select(const void *Z, int type, int64_t B, int64_t W, int64_t V, int64_t ldz, const float *score, const uint8_t *finished,
                       int32_t eos, int64_t n, float *out_score, int32_t *out_parent, int32_t *out_token, void *work, hipStream_t st) {
    const TopLists l = rows_top_lists(type, B * W, V, n, W);
    const hipError_t e = rows_top_keys(Z, type, B * W, V, ldz, n, W, l, finished, eos, work, st);
    if (e != hipSuccess) return e;
    const char *lists = (const char *)work + l.at;
    const BeamArgs a{(const uint64_t *)(lists + l.sums), (const float2 *)lists, score, (int)W, (int)l.lists, (int)n, out_score, out_parent, out_token};
    const int64_t total = W * l.lists * n;
    if (total <= 1024) hipLaunchKernelGGL((k_beam_join<256, 4>), dim3((unsigned)B), dim3(256), 0, st, a);
    else if (total <= 4096) hipLaunchKernelGGL((k_beam_join<512, 8>), dim3((unsigned)B), dim3(512), 0, st, a);
    else hipLaunchKernelGGL((k_beam_join<1024, 16>), dim3((unsigned)B), dim3(1024), 0, st, a);
    return hipGetLastError();
}

hipError_t beam_reorder(void *const *states, int64_t nstates, const StateLayout &l, const int32_t *parent, hipStream_t st) {
    // the widest unit that divides every address and length
    uint64_t all = (uint64_t)l.inner;
    if (l.B > 1) all |= (uint64_t)l.batch_stride;
    if (l.W > 1) all |= (uint64_t)l.beam_stride;
    if (l.outer > 1) all |= (uint64_t)l.outer_stride;
    for (int64_t i = 0; i < nstates; ++i) all |= (uint64_t)(uintptr_t)states[i];
    int unit = all & 1 ? 1 : all & 2 ? 2 : all & 4 ? 4 : all & 8 ? 8 : 16;
    while (kWave * unit * l.W > 65536) unit /= 2;            // one wavefront's tile fits into LDS: 4 bytes at 256 beams
    const auto kernel = unit == 16 ? k_beam_reorder<uint4> : unit == 8 ? k_beam_reorder<uint2> : unit == 4 ? k_beam_reorder<uint32_t>
                      : unit == 2 ? k_beam_reorder<uint16_t> : k_beam_reorder<uint8_t>;
    const int threads = kMoveThreads * unit * l.W > 65536 ? kWave : kMoveThreads;
    const int64_t lds = (int64_t)threads * unit * l.W;
    const int64_t units = l.inner / unit * l.outer;
    int64_t gx = (units + threads - 1) / threads;
    if (gx > 65536) gx = 65536;
    for (int64_t s0 = 0; s0 < nstates; s0 += kStates)
        for (int64_t b0 = 0; b0 < l.B; b0 += 65535) {
            StatePointers sp{};
            const int64_t ns = nstates - s0 < kStates ? nstates - s0 : kStates, nb = l.B - b0 < 65535 ? l.B - b0 : 65535;
            for (int64_t i = 0; i < ns; ++i) sp.p[i] = (char *)states[s0 + i] + b0 * l.batch_stride;
            hipLaunchKernelGGL(kernel, dim3((unsigned)gx, (unsigned)nb, (unsigned)ns), dim3(threads), (size_t)lds, st, sp, l, parent + b0 * l.W);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    return hipSuccess;
}

}  // namespace comet
