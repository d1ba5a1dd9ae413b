// Attention over the blocks that are chosen for each query: the kernels.
//
// out = softmax(scale q K^T) V, with a running maximum and sum, over the places of the chosen blocks.  The rows of a matrix instruction are the
// heads of a few tokens that share a head of the cache: G query heads of one token, or of up to 32 neighbouring tokens, which mostly choose
// the same blocks.  A workgroup takes the union of its tokens' blocks, each block with a mask of the tokens that chose it, and reads keys
// and values once for all of them.  Its wavefronts take different places, each with a maximum, a sum and an output of its own, and are
// joined at the end: nothing is handed from wavefront to wavefront on the way, and no barrier waits.
//
// Both products are turned around, S^T = K Q^T and O^T = V^T P^T: then a lane of the first one's result holds four places of one row, which is
// how the second one wants P, and no element has to move.  V^T's fragments come from LDS, which turns 16-bit elements around as it is read.
//
// Bound by memory where tokens are single (64 tokens, 8 heads, 2048 places each, 537 MB: 92 us, 5.9 TB/s; the same loads alone 6.6 to 7.0), by the dies'
// caches where they are neighbours (4093 tokens, 4 heads, 1024 places each: 318 us, 216 TFLOP/s; keys and values are read by every fourth
// token, 5.8 GB, at 19 TB/s of 31).  Every wavefront holds all of the workgroup's rows.  Four tiles of them in a wavefront would read less, but leave registers for
// one wavefront a SIMD: 547 us with eight tokens.  Rows spread over the wavefronts, all of which would read one tile of keys, have not been measured.
#pragma once

#include "cache.hpp"

namespace comet {

struct AttendArgs {
    Queries q;
    const char *keys, *values;
    int64_t blocks;
    int block, heads, size, group;            // group: query heads of a head of the cache
    int64_t key_stride[3], value_stride[3];   // in bytes
    const int32_t *sel;
    int K;
    float c;                                  // scale * log2 e
    void *out;
    float *lse;
    int tokens, chunk, chunks;                // of a workgroup: tokens at most, query heads; chunks of them in a group
    int64_t tiles;                            // at most
    int splits, words, entries;               // workgroups that share a tile's places; sizes of the list
    bool once;                                // what is read does not stay in the last cache: it is read past it
    float *part;                              // splits > 1: [item x splits x rows x (DT + 2)]
};

typedef float F4 __attribute__((ext_vector_type(4)));
typedef __bf16 B8 __attribute__((ext_vector_type(8)));
typedef _Float16 H8 __attribute__((ext_vector_type(8)));
typedef uint32_t U4 __attribute__((ext_vector_type(4)));
typedef short S4 __attribute__((ext_vector_type(4)));

// What the types do differently.  A step of a wavefront takes HALVES times 16 places: of 16 bits 32, which one matrix instruction of the second
// product adds up, of 32 bits 16.
template <int TYPE, int DT> struct Shape {
    static constexpr int CH = Elem<TYPE>::kPer;                // elements of 16 bytes
    static constexpr int HALVES = TYPE == COMET_F32 ? 1 : 2;
    static constexpr int CHUNKS = DT / CH;                     // 16-byte pieces of a key
    static constexpr int NK = CHUNKS / 4;                      // of them in a lane: piece 4 kk + lane / 16
    static constexpr int TURN = CHUNKS < 16 ? 1 : 0;
    static constexpr int LINE = CHUNKS * 16;                   // bytes of a key
    static constexpr int LOADS = HALVES * 16 * CHUNKS / kWave; // loads of a step's keys
    static constexpr int STAGE = 2 * HALVES * 16 * LINE;       // bytes of LDS for a step's keys and values
    static constexpr int OT = DT / 16;                         // tiles of 16 elements of the output
};

template <int TYPE> __device__ __forceinline__ F4 product(U4 a, U4 b, F4 c) {
    if constexpr (TYPE == COMET_BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(B8, a), __builtin_bit_cast(B8, b), c, 0, 0, 0);
    else if constexpr (TYPE == COMET_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(H8, a), __builtin_bit_cast(H8, b), c, 0, 0, 0);
    else {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0, 0, 0);
        return c;
    }
}

// Tiles of 16 rows that a wavefront's registers hold with two wavefronts a SIMD (one where keys are of more than 128 elements).
constexpr int attend_tiles(int wide) { return wide <= 128 ? 2 : 1; }
constexpr int kWaves = 4;
// Weights are relative to 2^-kRaise of the maximum.  16-bit floats have 15 exponents above 1, which are of no use otherwise: 2^13 is the largest weight
// then (what rounding a maximum beyond 2^24 to 32 bits adds to that is at most 2^2 below 2^26; a row that comes out infinite is done again by itself).
template <int TYPE> constexpr float kRaise = TYPE == COMET_F16 ? 5.f : 0.f;

// What a workgroup works at.
struct Item { int tile, head, chunk, split; int64_t id; };
__device__ __forceinline__ bool item_of(const AttendArgs &a, uint32_t from, Item &i) {
    // neighbouring workgroups go to the eight dies in turn, each of which has a cache of its own: a die gets a stretch of the items
    const uint32_t hc = a.heads * a.chunks, tiles = (uint32_t)a.tiles, splits = a.splits, all = tiles * hc * splits, each = gridDim.x / 8;
    uint32_t x = from + (blockIdx.x & 7) * each + (blockIdx.x >> 3), at;
    if (x >= all) return false;
    if (a.tokens == 1) {             // heads of one token next to each other: their keys are next to each other in memory
        const uint32_t y = x / hc;
        at = x - y * hc, i.tile = (int)(y / splits), i.split = (int)(y - i.tile * splits);
    } else {                         // tokens next to each other: they read the same keys
        const uint32_t y = x / splits;
        i.split = (int)(x - y * splits), at = y / tiles, i.tile = (int)(y - at * tiles);
    }
    i.head = (int)(at / a.chunks), i.chunk = (int)(at - i.head * a.chunks);
    i.id = ((int64_t)i.tile * hc + at) * splits + i.split;
    return true;
}

// The union of the tokens' choices in LDS: entry i is block j[i] of the request, at id[i] in the cache, chosen by the tokens of mask[i] (0 where there is no
// such block: it counts as the cache's first then, and nobody reads it).
struct List { int *j, *id; uint32_t *mask; int n; };
__host__ __device__ inline int behind_list(const AttendArgs &a) { return (3 * a.entries + 3) / 4 * 16; }
constexpr int kMostEntries = 2048;           // tokens times their choices
template <int T> __device__ __forceinline__ List make_list(const AttendArgs &a, const Tile &t, int head, uint32_t *raw, int64_t *buf) {
    uint32_t *bits = raw + behind_list(a) / 4, *before = bits + a.words;          // not needed any more afterwards
    List l{(int *)raw, (int *)raw + a.entries, raw + 2 * a.entries, 0};
    const auto seen = [&](int64_t place) {
        const int64_t c = place < 0 ? 0 : place / a.block + 1;
        return (int)(c < a.q.M ? c : a.q.M);
    };
    const int32_t *table = a.q.table + t.b * a.q.ldt, *sel = a.sel + (t.first * a.heads + head) * a.K;
    const int last = seen(t.place + t.n - 1), all = t.n * a.K;
    const auto id_of = [&](int j) {
        const int id = table[j];
        return id >= 0 && id < a.blocks ? id : -1;
    };
    if (a.blocks == 0 || last == 0) return l;
    constexpr int MOST = kMostEntries / T;
    int j[MOST];                                // the thread's choices, -1 where they are none
#pragma unroll
    for (int k = 0; k < MOST; ++k) {
        j[k] = -1;
        if (k * T >= all) continue;
        const int e = k * T + threadIdx.x;
        if (e >= all) continue;
        const int i = t.n == 1 ? 0 : e / a.K, x = sel[(int64_t)i * a.heads * a.K + (e - i * a.K)];
        j[k] = x >= 0 && x < seen(t.place + i) ? x : -1;
    }
    if (t.n == 1 && all <= T) {
        // one token: its choices as they are, where they ascend, and behind them there is none
        const int e = threadIdx.x;
        int id = -1;
        if (j[0] >= 0) id = id_of(j[0]);
        if (e < all) l.j[e] = j[0];
        __syncthreads();
        const bool mixed = e < all && e > 0 && (j[0] >= 0 ? l.j[e - 1] >= j[0] || l.j[e - 1] < 0 : false);
        const int some = __syncthreads_count(j[0] >= 0);
        if (!__syncthreads_or(mixed)) {
            if (e < some) l.id[e] = id < 0 ? 0 : id, l.mask[e] = id < 0 ? 0 : 1;
            l.n = some;
            __syncthreads();
            return l;
        }
    }
    const int words = (last + 31) / 32;
    for (int w = threadIdx.x; w < words; w += T) bits[w] = 0;
    for (int i = threadIdx.x; i < a.entries; i += T) l.mask[i] = 0;
    int id[MOST];
#pragma unroll
    for (int k = 0; k < MOST; ++k) {
        id[k] = -1;
        if (j[k] >= 0) id[k] = id_of(j[k]);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < MOST; ++k)
        if (j[k] >= 0) atomicOr(&bits[j[k] >> 5], 1u << (j[k] & 31));
    __syncthreads();
    if (words <= kWave) {
        const int lane = threadIdx.x & (kWave - 1);
        const uint32_t mine = lane < words ? bits[lane] : 0;
        const int upto = lanes_scan(__builtin_popcount(mine));
        int at = upto - __builtin_popcount(mine);
        l.n = __builtin_amdgcn_readlane(upto, kWave - 1);
        if (threadIdx.x < words) {
            before[lane] = at;
            for (uint32_t left = mine; left; left &= left - 1) l.j[at++] = lane * 32 + __builtin_ctz(left);
        }
    } else {
        const int each = (words + T - 1) / T, w0 = threadIdx.x * each, w1 = w0 + each < words ? w0 + each : words;
        int64_t mine = 0, total;
        for (int w = w0; w < w1; ++w) mine += __builtin_popcount(bits[w]);
        int at = (int)(block_scan<T>(mine, buf, total) - mine);
        for (int w = w0; w < w1; ++w) {
            before[w] = at;
            for (uint32_t left = bits[w]; left; left &= left - 1) l.j[at++] = w * 32 + __builtin_ctz(left);
        }
        l.n = (int)total;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < MOST; ++k)
        if (j[k] >= 0) {
            const int e = k * T + threadIdx.x, x = (int)before[j[k] >> 5] + __builtin_popcount(bits[j[k] >> 5] & ((1u << (j[k] & 31)) - 1));
            l.id[x] = id[k] < 0 ? 0 : id[k];
            if (id[k] >= 0) atomicOr(&l.mask[x], 1u << (t.n == 1 ? 0 : e / a.K));
        }
    __syncthreads();
    return l;
}

// N elements of a row of the output, at a multiple of N from its start, of which `left` are left: 8 bytes or 16 at a time.
template <int TYPE, int N> __device__ __forceinline__ void put_elements(typename Elem<TYPE>::T *to, const float *f, int left) {
    using E = Elem<TYPE>;
    if constexpr (N < E::kPer) {
        float g[E::kPer] = {};
#pragma unroll
        for (int e = 0; e < N; ++e) g[e] = f[e];
        const uint4 y = E::narrow(g);
        if (left > 0) *(uint2 *)to = make_uint2(y.x, y.y);
    } else {
#pragma unroll
        for (int e = 0; e < N; e += E::kPer)
            if (left > e) *(uint4 *)(to + e) = E::narrow(f + e);
    }
}

__device__ __forceinline__ float xor16(float v) { return __shfl_xor(v, 16); }
__device__ __forceinline__ float xor32(float v) { return __shfl_xor(v, 32); }

// Sixteen places of a block: where they are, who reads them.
struct Places {
    const char *key, *value;                  // the block's first place, of the head
    int start, last;                          // the first place's number in the block, the last one's that any of the tokens reads
    int from;                                 // the first place's number in the request
    uint32_t mask;
};

typedef __attribute__((address_space(1))) const void Global;
typedef __attribute__((address_space(3))) void Lds;

// The wavefront's loads into LDS are there; what it has read from LDS is in registers.
__device__ __forceinline__ void loads_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

template <int TYPE, int DT, int MT>
__global__ void __launch_bounds__(kWaves * kWave, DT <= 128 ? 2 : 1) k_attend(AttendArgs a, uint32_t first) {
    using S = Shape<TYPE, DT>;
    using E = Elem<TYPE>;
    using T = typename E::T;
    constexpr int WAVES = kWaves, THREADS = WAVES * kWave, SIZE = (int)sizeof(T), OT = S::OT, LINE = DT + 4, HALVES = S::HALVES;
    extern __shared__ __align__(16) uint32_t raw[];
    __shared__ int64_t buf[WAVES], where[3];
    __shared__ float2 ml[WAVES][16];
    Item item;
    if (!item_of(a, first, item)) return;
    const Tile t = find_tile<THREADS>(a.q, a.tokens, item.tile, buf, where);
    if (t.n == 0) return;
    const int64_t place0 = t.place, place1 = place0 + t.n - 1;

    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), col = lane & 15, g = lane >> 4;
    const int heads = a.group - item.chunk * a.chunk < a.chunk ? a.group - item.chunk * a.chunk : a.chunk;      // of this chunk
    const int rows = t.n * heads, x0 = item.head * a.group + item.chunk * a.chunk;
    // the lane's row of each tile of 16: its token and what it has to leave out
    int token[MT];
    uint32_t of_tile[MT];                      // tokens that have a row in it
    U4 q[MT][S::NK];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int r = 16 * m + col, i = r / heads;
        token[m] = i < t.n ? i : t.n - 1;
        const int i0 = 16 * m / heads, i1 = (16 * m + 15) / heads, most = i1 < t.n ? i1 : t.n - 1;
        of_tile[m] = i0 > most ? 0 : __builtin_amdgcn_readfirstlane((most == 31 ? ~0u : (2u << most) - 1) & ~((1u << i0) - 1));
        const T *from = (const T *)a.q.q + (t.first + i) * a.q.row + (int64_t)(x0 + r - i * heads) * a.q.head;
#pragma unroll
        for (int kk = 0; kk < S::NK; ++kk) {
            const int d = (4 * kk + g) * S::CH;
            q[m][kk] = U4{0, 0, 0, 0};
            if (r < rows && d < a.size) q[m][kk] = *(const U4 *)(from + d);
        }
    }

    const List list = make_list<THREADS>(a, t, item.head, raw, buf);

    // Sixteens of all blocks, as far as anything is read; the last block of the list is the last of the request.
    const int per = a.block / 16;
    int sixteens = 0;
    if (list.n > 0) {
        const int64_t left = (place1 - (int64_t)list.j[list.n - 1] * a.block) / 16 + 1;
        sixteens = (list.n - 1) * per + (int)(left < per ? left : per);
    }
    const int steps = (sixteens + HALVES - 1) / HALVES;
    const int begin = (int)((int64_t)steps * item.split / a.splits), end = (int)((int64_t)steps * (item.split + 1) / a.splits);

    // Sixteen `r` of entry e.  Those behind the last one are the last one's, and read by nobody.
    const char *const keys = a.keys + item.head * a.key_stride[2], *const values = a.values + item.head * a.value_stride[2];
    const auto places = [&](int e, int r) {
        const bool there = e * per + r < sixteens;
        if (!there) e = list.n - 1, r = 0;
        Places p;
        const int j = __builtin_amdgcn_readfirstlane(list.j[e]), id = __builtin_amdgcn_readfirstlane(list.id[e]);
        const uint32_t mask = __builtin_amdgcn_readfirstlane(list.mask[e]);
        p.start = r * 16;
        p.from = j * a.block + p.start;
        const int last = (int)place1 - j * a.block;
        p.last = last < a.block ? last : a.block - 1;
        p.mask = there ? mask : 0;
        p.key = keys + id * a.key_stride[0];
        p.value = values + id * a.value_stride[0];
        return p;
    };
    // The places of a step, from where it begins; then where the wavefront's next step begins.
    int entry = HALVES * (begin + wave) / per, sixteen = HALVES * (begin + wave) - entry * per;
    const int skip = HALVES * WAVES / per, more = HALVES * WAVES - skip * per;
    const auto step = [&](Places (&x)[HALVES]) {
        x[0] = places(entry, sixteen);
        if constexpr (HALVES == 2) {
            if (sixteen + 1 < per && entry * per + sixteen + 1 < sixteens) {
                x[1] = x[0];
                x[1].start += 16, x[1].from += 16;
            } else {
                x[1] = sixteen + 1 < per ? places(entry, sixteen + 1) : places(entry + 1, 0);
            }
        }
        entry += skip, sixteen += more;
        if (sixteen >= per) sixteen -= per, ++entry;
    };
    // Keys and values go to LDS straight from memory, a row of 16-byte pieces after the other, and from there to the lanes that want them.  Read by
    // those lanes themselves, a load asks for 64 pieces of 16 rows (4093 tokens: 783 us with values by way of registers, 346 so).  Piece c of row i is at c ^ i, so
    // that what is read together, of 16 rows, lies in different banks.  Places behind the last one that is read are taken from there:
    // nothing comes from memory that no token reads.
    char *const stage = (char *)raw + behind_list(a) + wave * S::STAGE, *const stage_v = stage + S::STAGE / 2;
    const bool ragged = a.size % (4 * S::CH) != 0;
    const int key_line = (int)a.key_stride[1], value_line = (int)a.value_stride[1];
    int key_at[S::LOADS], value_at[S::LOADS];
#pragma unroll
    for (int n = 0; n < S::LOADS; ++n) {
        const int k = n * kWave / S::CHUNKS % 16 + lane / S::CHUNKS, at = (n * kWave + lane) % S::CHUNKS, c = at ^ (k >> S::TURN & 15 & (S::CHUNKS - 1));
        const int d = c * S::CH < a.size ? c * 16 : 0;
        key_at[n] = k * key_line + d, value_at[n] = k * value_line + d;
    }
    const auto load = [&](const Places (&x)[HALVES]) {
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            const Places &p = x[h];
            constexpr int EACH = S::LOADS / HALVES;
            if (p.start + 15 <= p.last) {
                const char *key = p.key + (uint32_t)(p.start * key_line), *value = p.value + (uint32_t)(p.start * value_line);
#pragma unroll
                for (int n = h * EACH; n < (h + 1) * EACH; ++n) {
                    if (MT == 1 && a.once) {
                        __builtin_amdgcn_global_load_lds((Global *)(key + (uint32_t)key_at[n]), (Lds *)(stage + n * 1024), 16, 0, 2);
                        __builtin_amdgcn_global_load_lds((Global *)(value + (uint32_t)value_at[n]), (Lds *)(stage_v + n * 1024), 16, 0, 2);
                    } else {
                        __builtin_amdgcn_global_load_lds((Global *)(key + (uint32_t)key_at[n]), (Lds *)(stage + n * 1024), 16, 0, 0);
                        __builtin_amdgcn_global_load_lds((Global *)(value + (uint32_t)value_at[n]), (Lds *)(stage_v + n * 1024), 16, 0, 0);
                    }
                }
            } else {
#pragma unroll
                for (int n = h * EACH; n < (h + 1) * EACH; ++n) {
                    const int k = n * kWave / S::CHUNKS % 16 + lane / S::CHUNKS, i = p.start + k < p.last ? p.start + k : p.last;
                    __builtin_amdgcn_global_load_lds((Global *)(p.key + (uint32_t)(key_at[n] + (i - k) * key_line)), (Lds *)(stage + n * 1024), 16, 0, 0);
                    __builtin_amdgcn_global_load_lds((Global *)(p.value + (uint32_t)(value_at[n] + (i - k) * value_line)), (Lds *)(stage_v + n * 1024), 16, 0, 0);
                }
            }
        }
    };

    F4 o[MT][OT];
    float top[MT], sum[MT];                   // the row's maximum as it was last raised; the lane's part of its sum
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        top[m] = kNegInf, sum[m] = 0.f;
#pragma unroll
        for (int c = 0; c < OT; ++c) o[m][c] = F4{0, 0, 0, 0};
    }

    // The next step's keys and values are on their way while these are computed with.
    if (begin + wave < end) {
        Places now[HALVES];
        step(now);
        load(now);
        for (int i = begin + wave; i < end; i += WAVES) {
            U4 key[HALVES][S::NK], value[TYPE == COMET_F32 ? 4 * OT / 4 : OT];
            loads_done();
#pragma unroll
            for (int h = 0; h < HALVES; ++h)
#pragma unroll
                for (int kk = 0; kk < S::NK; ++kk)
                    key[h][kk] = *(const U4 *)(stage + (16 * h + col) * S::LINE + ((4 * kk + g) ^ (col >> S::TURN & (S::CHUNKS - 1))) * 16);
            if constexpr (TYPE == COMET_F32) {
                // a lane: places 4 g + r, elements 64 dd + 4 col + ..: each of the four belongs to an output tile of its own
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int dd = 0; dd < OT / 4; ++dd)
                        value[r * (OT / 4) + dd] = *(const U4 *)(stage_v + (4 * g + r) * S::LINE + ((16 * dd + col) ^ ((4 * g + r) >> S::TURN & 15)) * 16);
            } else {
                // Sixteen lanes read four places' 16 elements, and get an element's four places each: V^T as the matrix instruction wants it.
                const int row = 4 * g + col / 4, turn = row >> S::TURN & (S::CHUNKS - 1);
#pragma unroll
                for (int c = 0; c < OT; ++c) {
                    const char *at = stage_v + row * S::LINE + ((2 * c + (col >> 1 & 1)) ^ turn) * 16 + (col & 1) * 8;
                    const S4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) S4 *)at);
                    const S4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) S4 *)(at + 16 * S::LINE));
                    const uint2 x = __builtin_bit_cast(uint2, lo), y = __builtin_bit_cast(uint2, hi);
                    value[c] = U4{x.x, x.y, y.x, y.y};
                }
            }
            reads_done();
            Places then[HALVES];
            step(then);
            if (i + WAVES < end) load(then);
            if (ragged) {
#pragma unroll
                for (int h = 0; h < HALVES; ++h)
#pragma unroll
                    for (int kk = 0; kk < S::NK; ++kk)
                        if ((4 * kk + g) * S::CH >= a.size) key[h][kk] = U4{0, 0, 0, 0};
            }
            uint32_t some = 0, all = ~0u;                      // tokens that read something of it, and those that read all
#pragma unroll
            for (int h = 0; h < HALVES; ++h) some |= now[h].mask, all &= now[h].from + 15 <= (int)place0 ? now[h].mask : 0;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                if (!(some & of_tile[m])) continue;
                float z[4 * HALVES];
#pragma unroll
                for (int h = 0; h < HALVES; ++h) {
                    F4 s = F4{0, 0, 0, 0};
#pragma unroll
                    for (int kk = 0; kk < S::NK; ++kk) s = product<TYPE>(key[h][kk], q[m][kk], s);
#pragma unroll
                    for (int r = 0; r < 4; ++r) z[4 * h + r] = s[r];
                }
                if (of_tile[m] & ~all) {
#pragma unroll
                    for (int h = 0; h < HALVES; ++h) {
                        const int last = now[h].mask >> token[m] & 1 ? (int)place0 + token[m] - now[h].from : -1;
#pragma unroll
                        for (int r = 0; r < 4; ++r) z[4 * h + r] = 4 * g + r <= last ? z[4 * h + r] : kNegInf;
                    }
                }
                float most = z[0];
#pragma unroll
                for (int r = 1; r < 4 * HALVES; ++r) most = fmaxf(most, z[r]);
                most *= a.c;
                // The maximum follows when a score is 256 times over it, and not before: weights are 256 at most (above 2^kRaise), which costs nothing in
                // floating point, and the output is seldom scaled anew.
                if (__ballot(most > top[m] + (8.f + kRaise<TYPE>))) {
                    most = fmaxf(most, xor16(most));
                    most = fmaxf(most, xor32(most));
                    const float high = fmaxf(top[m], most - kRaise<TYPE>), back = high == kNegInf ? 1.f : exp2_fast(top[m] - high);
                    top[m] = high;
                    sum[m] *= back;
#pragma unroll
                    for (int c = 0; c < OT; ++c) o[m][c] *= back;
                }
                const float shift = top[m] == kNegInf ? 0.f : top[m];
                float add = 0.f;
#pragma unroll
                for (int r = 0; r < 4 * HALVES; ++r) {
                    z[r] = exp2_fast(__builtin_fmaf(z[r], a.c, -shift));
                    add += z[r];
                }
                sum[m] += add;
                if constexpr (TYPE == COMET_F32) {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
#pragma unroll
                        for (int c = 0; c < OT; ++c)
                            o[m][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(value[r * (OT / 4) + c / 4][c & 3]), z[r], o[m][c], 0, 0, 0);
                } else {
                    // Weights are rounded to the type, and what that takes off goes by a second product: 2^-16 of a weight is lost (bfloat16), 2^-22 and 2^-30 of the
                    // row's largest (16-bit float).  With the first one alone results are off by 0.0022 of their size for 0.0017, all of which is their own
                    // rounding; 4093 tokens take 307 us for 318, 64 single ones 92 for 92.  A product in 32 bits would take 16 times as long.
                    const uint4 y = E::narrow(z);
                    const U4 p = U4{y.x, y.y, y.z, y.w};
                    float rest[8];
                    E::widen(y, rest);
#pragma unroll
                    for (int r = 0; r < 8; ++r) rest[r] = z[r] - rest[r];
                    const uint4 y2 = E::narrow(rest);
                    const U4 p2 = U4{y2.x, y2.y, y2.z, y2.w};
#pragma unroll
                    for (int c = 0; c < OT; ++c) o[m][c] = product<TYPE>(value[c], p, o[m][c]);
#pragma unroll
                    for (int c = 0; c < OT; ++c) o[m][c] = product<TYPE>(value[c], p2, o[m][c]);
                    if constexpr (TYPE == COMET_F16) {
                        // Both together do not hold a weight below 2^-14 to half a step, and none below 2^-25.  What is missing of these goes by a third product, 2^24 times
                        // as large: half a step is lost down to 2^-43 of the row's largest weight, and 2^-54 of that below.  4093 tokens, some of whose
                        // weights are such: 325 us for 318.
                        constexpr uint32_t kLeast = (127u - 49) << 23, kNormal = (127u - 14) << 23;      // bits of 2^-49, 2^-14
                        uint32_t least = ~0u;
#pragma unroll
                        for (int r = 0; r < 8; ++r) {
                            const uint32_t bits = __float_as_uint(z[r]) - kLeast;        // what is below is large
                            least = bits < least ? bits : least;
                        }
                        if (__ballot(least < kNormal - kLeast)) {
#pragma unroll
                            for (int r = 0; r < 8; ++r) z[r] = z[r] < 0x1p-14f ? (z[r] - (float)(_Float16)z[r]) * 0x1p24f : 0.f;
                            const uint4 y = E::narrow(z);
                            const U4 p = U4{y.x, y.y, y.z, y.w};
#pragma unroll
                            for (int c = 0; c < OT; ++c) o[m][c] = product<TYPE>(value[c], p, o[m][c] * 0x1p24f) * 0x1p-24f;
                        }
                    }
                }
            }
#pragma unroll
            for (int h = 0; h < HALVES; ++h) now[h] = then[h];
        }
    }

    // ---- the wavefronts' parts together, one tile of rows after the other
    uint32_t bad[MT];                          // rows with a NaN
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        float any = sum[m];
#pragma unroll
        for (int c = 0; c < OT; ++c) any += (o[m][c][0] + o[m][c][1] + o[m][c][2] + o[m][c][3]) * 0.f;
        const uint64_t b = __ballot(any != any);
        bad[m] = (uint32_t)(b | b >> 16 | b >> 32 | b >> 48) & 0xffff;
        sum[m] += xor16(sum[m]);
        sum[m] += xor32(sum[m]);
    }
    float *const lines = (float *)raw + behind_list(a) / 4, *const line = lines + wave * 16 * LINE;      // where the keys were
    // A row that came out as NaN once more, by itself: what it does not read weighs 0 in the products above, but 0 times a NaN or an infinity of
    // another row's is a NaN.  One place after the other, its own ones only.
    const auto alone = [&](int m, int n) {
        const int r = 16 * m + n;
        if (r >= rows) return;
        const int i = r / heads;
        const T *from = (const T *)a.q.q + (t.first + i) * a.q.row + (int64_t)(x0 + r - i * heads) * a.q.head;
        float high = kNegInf, total = 0.f, out[DT / kWave] = {};
        for (int step = begin + wave; step < end; step += WAVES)
            for (int h = 0; h < HALVES; ++h) {
                const int s = HALVES * step + h;
                if (s >= sixteens) break;
                const int e = s / per, id = list.id[e];
                if (!(list.mask[e] >> i & 1)) continue;
                for (int k = 0; k < 16; ++k) {
                    const int in = (s - e * per) * 16 + k;
                    if ((int64_t)list.j[e] * a.block + in > place0 + i) break;
                    const T *key = (const T *)(a.keys + id * a.key_stride[0] + in * a.key_stride[1] + item.head * a.key_stride[2]);
                    const T *value = (const T *)(a.values + id * a.value_stride[0] + in * a.value_stride[1] + item.head * a.value_stride[2]);
                    float z = 0.f;
                    for (int d = lane; d < a.size; d += kWave) z = __builtin_fmaf(E::one(from[d]), E::one(key[d]), z);
#pragma unroll
                    for (int d = 1; d < kWave; d *= 2) z += __shfl_xor(z, d);
                    z *= a.c;
                    if (z > high || z != z) {
                        const float back = high == kNegInf ? 0.f : exp2_fast(high - z);
                        total *= back;
#pragma unroll
                        for (int u = 0; u < DT / kWave; ++u) out[u] = back == 0.f ? 0.f : out[u] * back;
                        high = z;
                    }
                    if (z == kNegInf && high == kNegInf) continue;
                    const float weight = exp2_fast(z - high);
                    total += weight;
#pragma unroll
                    for (int u = 0; u < DT / kWave; ++u) {
                        const int d = u * kWave + lane;
                        if (d < a.size) out[u] = __builtin_fmaf(weight, E::one(value[d]), out[u]);
                    }
                }
            }
        if (lane == 0) ml[wave][n] = make_float2(high, total);
#pragma unroll
        for (int u = 0; u < DT / kWave; ++u) line[n * LINE + u * kWave + lane] = out[u];
    };
    __syncthreads();
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        if (16 * m >= rows) break;
#pragma unroll
        for (int c = 0; c < OT; ++c) {
            float *to = line + col * LINE;
            if constexpr (TYPE == COMET_F32) {
                if (c % 4 == 0)
#pragma unroll
                    for (int r = 0; r < 4; ++r) *(F4 *)(to + 16 * c + 4 * (4 * g + r)) = F4{o[m][c][r], o[m][c + 1][r], o[m][c + 2][r], o[m][c + 3][r]};
            } else {
                *(F4 *)(to + 16 * c + 4 * g) = o[m][c];
            }
        }
        if (g == 0) ml[wave][col] = make_float2(top[m], sum[m]);
        if (bad[m]) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            for (uint32_t left = bad[m]; left; left &= left - 1) alone(m, __builtin_ctz(left));
        }
        __syncthreads();
        // some threads a row, a few elements each
        constexpr int EACH = 16 * DT / THREADS, OVER = DT / EACH;
        const int n = threadIdx.x / OVER, d0 = threadIdx.x % OVER * EACH, r = 16 * m + n;
        if (r < rows) {
            float high = kNegInf, total = 0.f, part[WAVES], out[EACH] = {};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) high = fmaxf(high, ml[w][n].x);
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float2 y = ml[w][n];
                part[w] = y.x == high || y.x != y.x ? 1.f : y.x == kNegInf ? 0.f : exp2_fast(y.x - high);
                total += y.y * part[w];
            }
#pragma unroll
            for (int w = 0; w < WAVES; ++w)
                if (part[w] != 0.f)
#pragma unroll
                    for (int e = 0; e < EACH; ++e) out[e] = __builtin_fmaf(lines[(w * 16 + n) * LINE + d0 + e], part[w], out[e]);
            if (a.splits > 1) {
                float *to = a.part + (item.id * (16 * MT) + r) * (DT + 4);
                if (d0 == 0) to[DT] = high, to[DT + 1] = total;
#pragma unroll
                for (int e = 0; e < EACH; e += 4) *(F4 *)(to + d0 + e) = F4{out[e], out[e + 1], out[e + 2], out[e + 3]};
            } else {
                const int i = r / heads;
                const int64_t row = (t.first + i) * a.q.Q + x0 + r - i * heads;
                const float by = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
                for (int e = 0; e < EACH; ++e) out[e] = total == 0.f ? 0.f : out[e] * by;
                put_elements<TYPE, EACH>((T *)a.out + row * a.size + d0, out, a.size - d0);
                if (d0 == 0 && a.lse) a.lse[row] = total == 0.f ? kNegInf : (high + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
            }
        }
        __syncthreads();
    }
}

// The parts of a tile that several workgroups share: one workgroup a tile and head, a thread four elements of a row.  Bound by two waits, for the
// requests and for the parts.
constexpr int kSplits = 16;
template <int TYPE, int DT, int MT>
__global__ void __launch_bounds__(256) k_attend_join(AttendArgs a) {
    using E = Elem<TYPE>;
    using T = typename E::T;
    constexpr int THREADS = 256, EACH = DT / 4;
    __shared__ int64_t buf[THREADS / kWave], where[2];
    const uint32_t hc = a.heads * a.chunks, tile = blockIdx.x / hc, at = blockIdx.x - tile * hc;
    const int head = (int)(at / a.chunks), chunk = (int)(at - head * a.chunks);
    const Tile t = find_tile<THREADS>(a.q, a.tokens, (int)tile, buf, where);
    const int heads = a.group - chunk * a.chunk < a.chunk ? a.group - chunk * a.chunk : a.chunk, x0 = head * a.group + chunk * a.chunk;
    const float *from = a.part + (int64_t)blockIdx.x * a.splits * (16 * MT) * (DT + 4);
    for (int x = threadIdx.x; x < t.n * heads * EACH; x += THREADS) {
        const int r = x / EACH, d0 = x % EACH * 4;
        float high[kSplits], sum[kSplits], top = kNegInf, total = 0.f;
        F4 part[kSplits], out = F4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < kSplits; ++s) {
            high[s] = kNegInf, sum[s] = 0.f, part[s] = F4{0, 0, 0, 0};
            if (s >= a.splits) continue;
            const float *p = from + (s * 16 * MT + r) * (DT + 4);
            high[s] = p[DT], sum[s] = p[DT + 1], part[s] = *(const F4 *)(p + d0);
        }
#pragma unroll
        for (int s = 0; s < kSplits; ++s) top = fmaxf(top, high[s]);
#pragma unroll
        for (int s = 0; s < kSplits; ++s) {
            const float weight = high[s] == top || high[s] != high[s] ? 1.f : high[s] == kNegInf ? 0.f : exp2_fast(high[s] - top);
            total += sum[s] * weight;
            if (weight != 0.f) out += part[s] * weight;
        }
        const int i = r / heads;
        const int64_t row = (t.first + i) * a.q.Q + x0 + r - i * heads;
        const float by = total == 0.f ? 0.f : 1.f / total;
        float f[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = total == 0.f ? 0.f : out[e] * by;
        put_elements<TYPE, 4>((T *)a.out + row * a.size + d0, f, a.size - d0);
        if (d0 == 0 && a.lse) a.lse[row] = total == 0.f ? kNegInf : (top + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
    }
}

template <int TYPE, int DT, int MT> hipError_t attend_run(const AttendArgs &a, hipStream_t st) {
    constexpr int WAVES = kWaves;
    const int64_t items = a.tiles * a.heads * a.chunks * a.splits;
    size_t lds = (size_t)WAVES * Shape<TYPE, DT>::STAGE;
    for (const size_t other : {(size_t)WAVES * 16 * (DT + 4) * 4, (size_t)a.words * 8}) lds = other > lds ? other : lds;
    lds += behind_list(a);
    hipError_t e = hipSuccess;
    if (lds > 65536) e = hipFuncSetAttribute((const void *)k_attend<TYPE, DT, MT>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
    e = in_launches((items + 7) / 8 * 8, WAVES * kWave, [&](uint32_t first, unsigned n) {
        hipLaunchKernelGGL((k_attend<TYPE, DT, MT>), dim3(n), dim3(WAVES * kWave), lds, st, a, first);
    });
    if (e != hipSuccess || a.splits == 1) return e;
    hipLaunchKernelGGL((k_attend_join<TYPE, DT, MT>), dim3((unsigned)(a.tiles * a.heads * a.chunks)), dim3(256), 0, st, a);
    return hipGetLastError();
}

template <int TYPE, int DT> hipError_t attend_wide(const AttendArgs &a, int mt, hipStream_t st) {
    if constexpr (attend_tiles(DT) >= 2) if (mt == 2) return attend_run<TYPE, DT, 2>(a, st);
    return attend_run<TYPE, DT, 1>(a, st);
}
template <int TYPE> hipError_t attend_type(const AttendArgs &a, int wide, int mt, hipStream_t st) {
    return wide == 64 ? attend_wide<TYPE, 64>(a, mt, st) : wide == 128 ? attend_wide<TYPE, 128>(a, mt, st) : attend_wide<TYPE, 256>(a, mt, st);
}
hipError_t attend_f32(const AttendArgs &a, int wide, int mt, hipStream_t st);
hipError_t attend_bf16(const AttendArgs &a, int wide, int mt, hipStream_t st);
hipError_t attend_f16(const AttendArgs &a, int wide, int mt, hipStream_t st);

}  // namespace comet
