// The blocks that each query is to read, by the score of its heads' sum with the block's mean key.
#include "cache.hpp"

namespace comet {

namespace {

struct SelectArgs {
    Queries q;
    const void *mean;
    int64_t blocks, mean_block, mean_head;
    int block, heads, size, group;
    int K, first, last;
    int32_t *sel;
    int tokens, candidates;                  // tokens of a workgroup at most; room for a token's keys
};

constexpr uint64_t kAlways = ~0ull;          // above the order of every double
constexpr int kHeld = 16;                    // candidates of a lane, where a wavefront chooses

struct Choice { int32_t *sel; int C; };      // where a token's blocks go, and how many it sees

// What a token sees, of which it takes the K with the largest keys, equal ones by their number: by a wavefront, the keys in registers, HELD a lane.
// The K-th largest is found bit by bit, from the highest on, until as many as are wanted reach it: about 25 bits, of which the upper 32 are
// compared by themselves.  One count is a few instructions a register; the number of registers is fixed so that there is nothing else.
template <int HELD> __device__ __forceinline__ void choose_held(const uint64_t *key, const Choice &t, int K) {
    const int lane = threadIdx.x & (kWave - 1);
    uint64_t x[HELD];
    uint32_t high[HELD];
#pragma unroll
    for (int r = 0; r < HELD; ++r) {
        x[r] = 0;
        if (r * kWave + lane < t.C) x[r] = key[r * kWave + lane];
        high[r] = (uint32_t)(x[r] >> 32);
    }
    const auto there = [&](int r) { return r * kWave + lane < t.C; };
    uint32_t bar_high = 0, bar_low = 0;
    int reach = t.C;
    for (int bit = 31; bit >= 0 && reach != K; --bit) {
        const uint32_t y = bar_high | 1u << bit;
        int n = 0;
#pragma unroll
        for (int r = 0; r < HELD; ++r) n += __builtin_popcountll(__ballot(high[r] >= y));
        if (n >= K) bar_high = y, reach = n;
    }
    for (int bit = 31; bit >= 0 && reach != K; --bit) {
        const uint64_t y = (uint64_t)bar_high << 32 | bar_low | 1u << bit;
        int n = 0;
#pragma unroll
        for (int r = 0; r < HELD; ++r) n += __builtin_popcountll(__ballot(x[r] >= y));
        if (n >= K) bar_low |= 1u << bit, reach = n;
    }
    const uint64_t bar = (uint64_t)bar_high << 32 | bar_low;
    int over = 0;
#pragma unroll
    for (int r = 0; r < HELD; ++r) over += __builtin_popcountll(__ballot(there(r) && x[r] > bar));
    const uint64_t below = (1ull << lane) - 1;
    int at = 0, equal = K - over;                        // of those at the bar, the lowest
#pragma unroll
    for (int r = 0; r < HELD; ++r) {
        const uint64_t ties = __ballot(there(r) && x[r] == bar);
        const bool in = there(r) && (x[r] > bar || (x[r] == bar && __builtin_popcountll(ties & below) < equal));
        const uint64_t taken = __ballot(in);
        if (in) t.sel[at + __builtin_popcountll(taken & below)] = r * kWave + lane;
        at += __builtin_popcountll(taken);
        const int n = __builtin_popcountll(ties);
        equal -= n < equal ? n : equal;
    }
}
__device__ __forceinline__ void choose_held(const uint64_t *key, const Choice &t, int K) {
    if (t.C <= 2 * kWave) choose_held<2>(key, t, K);
    else if (t.C <= 4 * kWave) choose_held<4>(key, t, K);
    else if (t.C <= 8 * kWave) choose_held<8>(key, t, K);
    else choose_held<kHeld>(key, t, K);
}

// The same by a workgroup of T threads, the keys in LDS.
template <int T> __device__ __forceinline__ void choose_all(const uint64_t *key, const Choice &t, int K, int *count, int64_t *scan) {
    if (threadIdx.x < 65) count[threadIdx.x] = 0;
    __syncthreads();
    uint64_t bar = 0;
    for (int bit = 63; bit >= 0; --bit) {
        const uint64_t y = bar | 1ull << bit;
        int c = 0;
        for (int j = threadIdx.x; j < t.C; j += T) c += key[j] >= y ? 1 : 0;
        if (c) atomicAdd(&count[bit], c);
        __syncthreads();
        if (count[bit] >= K) bar = y;
        if (count[bit] == K) break;
    }
    int more = 0;
    for (int j = threadIdx.x; j < t.C; j += T) more += key[j] > bar ? 1 : 0;
    if (more) atomicAdd(&count[64], more);
    __syncthreads();
    const int equal = K - count[64];
    int64_t before = 0, ties = 0, all;
    for (int j0 = 0; j0 < t.C; j0 += T) {
        const int j = j0 + threadIdx.x;
        const uint64_t k = j < t.C ? key[j] : 0;
        const int64_t tie = ties + block_scan<T>(j < t.C && k == bar ? 1 : 0, scan, all);
        ties += all;
        const bool in = j < t.C && (k > bar || (k == bar && tie <= equal));
        const int64_t at = before + block_scan<T>(in ? 1 : 0, scan, all);
        before += all;
        if (in) t.sel[at - 1] = j;
    }
}

typedef double D4 __attribute__((ext_vector_type(4)));

// One workgroup a head and TOKENS tokens of a request that follow each other.  Scores in 64 bits: off by (size + G) 2^-53
// times the sum of the products' sizes at most (products of 16-bit elements are exact), so that the exact scores' order decides but for blocks that are closer; the
// lanes and the matrix instructions add in different orders.  Sixteen blocks at a time, a lane a block and a quarter
// of its 16-byte pieces: the fragment of a 64-bit matrix instruction whose columns are 16 tokens' sums over their heads; a single token's
// products are added up by the lanes themselves, which is less work than columns that are not used.  4093 tokens of 4 heads, contexts of up to 256 blocks: 43 us,
// of which the matrix instructions are 10, the rest counts and waits; a token at a time, a thread a block, took 159.  16 tokens of 8 heads, up to
// 512 blocks: 12 us, all of it latency (25 that way).
template <int TYPE, int WIDE, int TOKENS, int WAVES>
__global__ void __launch_bounds__(WAVES * kWave) k_select(SelectArgs a, uint32_t from) {
    using E = Elem<TYPE>;
    using T = typename E::T;
    constexpr int THREADS = WAVES * kWave, CH = E::kPer, NK = WIDE / (4 * CH);
    extern __shared__ __align__(16) uint64_t keys[];
    __shared__ int64_t buf[WAVES], where[2];
    __shared__ int count[65];
    const uint32_t item = from + blockIdx.x;
    const int tile = (int)(item / (unsigned)a.heads), h = (int)(item - (unsigned)tile * a.heads);
    const Tile t = find_tile<THREADS>(a.q, a.tokens, tile, buf, where);
    if (t.n == 0) return;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, col = lane & 15, g = lane >> 4;
    const auto seen = [&](int i) {
        const int64_t place = t.place + i, c = place < 0 ? 0 : (int64_t)((uint32_t)place / (uint32_t)a.block) + 1;
        return (int)(c < a.q.M ? c : a.q.M);
    };
    const auto choice = [&](int i) { return Choice{a.sel + ((t.first + i) * a.heads + h) * a.K, seen(i)}; };
    const int most = seen(t.n - 1), stride = a.candidates;
    const bool scored = most > a.K;                                // else there is nothing to choose
    if (scored) {
        const int32_t *table = a.q.table + t.b * a.q.ldt;
        // the heads' sums, a thread a token and 16-byte piece, to where each lane finds its own, and the keys go afterwards
        constexpr int PIECES = 4 * NK, LINE = WIDE + 2;
        double *const sums = (double *)keys;
        for (int x = threadIdx.x; x < TOKENS * PIECES; x += THREADS) {
            const int i = x / PIECES, d = x % PIECES * CH;
            double s[CH] = {};
            if (i < t.n && d < a.size) {
                const T *from = (const T *)a.q.q + (t.first + i) * a.q.row + (int64_t)h * a.group * a.q.head + d;
#pragma unroll 4
                for (int y = 0; y < a.group; ++y) {
                    float f[CH];
                    E::widen(*(const uint4 *)(from + y * a.q.head), f);
#pragma unroll
                    for (int e = 0; e < CH; ++e) s[e] += (double)f[e];
                }
            }
#pragma unroll
            for (int e = 0; e < CH; ++e) sums[i * LINE + d + e] = s[e];
        }
        __syncthreads();
        double q[NK][CH];
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
            for (int e = 0; e < CH; ++e) q[k][e] = sums[(TOKENS == 1 ? 0 : col) * LINE + (4 * k + g) * CH + e];
        __syncthreads();
        const int mine = TOKENS == 1 ? most : col < t.n ? seen(col) : 0;          // blocks that the lane's token sees
        // A step's numbers of the table are asked for while the steps before it are computed; where a wavefront has the SIMD to itself, its means too.
        constexpr int STEP = THREADS / 4;
        const auto number = [&](int j0) {
            int p = -1;
            if (j0 + col < most) p = table[j0 + col];
            return p >= 0 && p < a.blocks ? p : -1;
        };
        const auto read = [&](int p, uint4 (&v)[NK]) {
            const T *m = (const T *)a.mean + (int64_t)(p < 0 ? 0 : p) * a.mean_block + h * a.mean_head;
#pragma unroll
            for (int k = 0; k < NK; ++k) {
                const int d = (4 * k + g) * CH;
                v[k] = make_uint4(0, 0, 0, 0);
                if (p >= 0 && d < a.size) v[k] = *(const uint4 *)(m + d);
            }
        };
        // a block's key for a token; blocks of the table that are none have NaN's
        const auto put = [&](int i, int block, double s, bool is) {
            if (block < mine) keys[i * stride + block] = block < a.first || block >= mine - a.last ? kAlways : is ? order_of_double(s) : 0;
        };
        int now = number(wave * 16), then = number(wave * 16 + STEP);
        uint4 v[NK];
        if (TOKENS == 1) read(now, v);
        for (int j0 = wave * 16; j0 < most; j0 += STEP) {
            const int later = number(j0 + 2 * STEP);
            uint4 w[NK];
            if (TOKENS == 1) read(then, w);
            else read(now, v);
            if constexpr (TOKENS == 1) {
                double s = 0, s2 = 0;
#pragma unroll
                for (int k = 0; k < NK; ++k) {
                    float f[CH];
                    E::widen(v[k], f);
#pragma unroll
                    for (int e = 0; e < CH; e += 2) s = __builtin_fma(q[k][e], (double)f[e], s), s2 = __builtin_fma(q[k][e + 1], (double)f[e + 1], s2);
                }
                s += s2;
                s += __shfl_xor(s, 16);
                s += __shfl_xor(s, 32);
                if (g == 0) put(0, j0 + col, s, now >= 0);
            } else {
                D4 s = {0, 0, 0, 0};
#pragma unroll
                for (int k = 0; k < NK; ++k) {
                    if (4 * k * CH >= a.size) continue;
                    float f[CH];
                    E::widen(v[k], f);
#pragma unroll
                    for (int e = 0; e < CH; ++e) s = __builtin_amdgcn_mfma_f64_16x16x4f64((double)f[e], q[k][e], s, 0, 0, 0);
                }
                const uint32_t is = (uint32_t)(__ballot(now >= 0) & 0xffff);
#pragma unroll
                for (int r = 0; r < 4; ++r) put(col, j0 + 4 * r + g, s[r], is >> (4 * r + g) & 1);
            }
            now = then, then = later;
            if (TOKENS == 1)
#pragma unroll
                for (int k = 0; k < NK; ++k) v[k] = w[k];
        }
        __syncthreads();
    }
    for (int i = TOKENS == 1 ? 0 : wave; i < t.n; i += TOKENS == 1 ? 1 : WAVES) {
        const Choice c = choice(i);
        if (c.C <= a.K) {
            for (int k = TOKENS == 1 ? threadIdx.x : lane; k < a.K; k += TOKENS == 1 ? THREADS : kWave) c.sel[k] = k < c.C ? k : -1;
        } else if (TOKENS > 1 || a.q.M <= kHeld * kWave) {
            if (TOKENS > 1 || wave == 0) choose_held(keys + i * stride, c, a.K);
        } else if constexpr (TOKENS == 1) {
            choose_all<THREADS>(keys, c, a.K, count, buf);
        }
    }
}

template <int TYPE, int WIDE> hipError_t launch(SelectArgs a, hipStream_t st) {
    // Tokens share their blocks' means where requests have four of them or more, and a wavefront's registers hold a token's candidates.  64 requests of 3, 4, 8
    // and 16 tokens, 4 heads, up to 250 blocks: 16.7, 16.8, 19.3 and 25.7 us together, 16.5, 18.2, 32.3 and 60.2 one by one.
    const int64_t B = a.q.B < a.q.N ? a.q.B : a.q.N, each = (a.q.N + B - 1) / B;
    // Where the table has more columns than a wavefront holds, every token goes by itself, however few blocks it sees.
    const bool many = each >= 4 && a.q.M <= kHeld * kWave;
    const auto kernel = many ? k_select<TYPE, WIDE, 16, 4> : k_select<TYPE, WIDE, 1, 8>;
    a.tokens = many ? 16 : 1;
    int64_t tiles = a.q.N / a.tokens + B;
    if (tiles > a.q.N) tiles = a.q.N;
    const size_t lds = (size_t)(a.candidates > WIDE + 2 ? a.candidates : WIDE + 2) * 8 * a.tokens;
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    const int threads = many ? 256 : 512;
    return in_launches(tiles * a.heads, threads, [&](uint32_t from, unsigned n) { hipLaunchKernelGGL(kernel, dim3(n), dim3(threads), lds, st, a, from); });
}
template <int TYPE> hipError_t launch(const SelectArgs &a, hipStream_t st) {
    return a.size <= 64 ? launch<TYPE, 64>(a, st) : a.size <= 128 ? launch<TYPE, 128>(a, st) : launch<TYPE, 256>(a, st);
}

}  // namespace

int64_t block_select_work(const comet_cache &, int64_t, int64_t, int64_t, int64_t, int64_t) { return 0; }

hipError_t block_select(const comet_cache &c, const Queries &q, int64_t K, int64_t first, int64_t last, int32_t *sel, void *, hipStream_t st) {
    // a token's keys lie 16 bytes off those of the one before it: 16 tokens' writes meet in few banks
    const SelectArgs a{q, c.mean, c.blocks, c.mean_stride[0], c.mean_stride[1], (int)c.block, (int)c.heads, (int)c.size, (int)(q.Q / c.heads),
                       (int)K, (int)first, (int)last, sel, 0, (int)((q.M + 15) / 16 * 16 + 2)};
    return c.type == COMET_F32 ? launch<COMET_F32>(a, st) : c.type == COMET_BF16 ? launch<COMET_BF16>(a, st) : launch<COMET_F16>(a, st);
}

}  // namespace comet
