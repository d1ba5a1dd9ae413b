// Attention over the blocks that are chosen for each query: the kernels.
//
// out = softmax(scale q K^T) V, with a running maximum and sum, over the places of the chosen blocks.  The rows of a matrix instruction are the
// heads of a few tokens that share a head of the cache: G query heads of one token, or of up to 32 neighbouring tokens, which mostly choose
// the same blocks.  A workgroup takes the union of its tokens' blocks, each block with a mask of the tokens that chose it, and reads keys
// and values once for all of them.  Its wavefronts take different places, each with a maximum, a sum and an output of its own, and are
// joined at the end: nothing is handed from wavefront to wavefront on the way, and no barrier waits.
//
// Both products are turned around, S^T = K Q^T and O^T = V^T P^T: then a lane of the first one's result holds four places of one row, which is
// how the second one wants P, and no element has to move.  V^T's fragments come from rows of V in registers: a lane reads the same 4 or 8
// elements of its 8 places, and pairs of places are put together 16 bits by 16 bits.
#pragma once

#include <type_traits>

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
    float *part;                              // splits > 1: [item x splits x rows x (DT + 2)]
};

constexpr int kAttend = 256, kWaves = kAttend / kWave;

typedef float F4 __attribute__((ext_vector_type(4)));
typedef __bf16 B8 __attribute__((ext_vector_type(8)));
typedef _Float16 H8 __attribute__((ext_vector_type(8)));
typedef uint32_t U4 __attribute__((ext_vector_type(4)));

// What the types do differently.  CH: elements of 16 bytes.
template <int TYPE, int DT> struct Shape {
    static constexpr int CH = Elem<TYPE>::kPer;
    static constexpr int NK = DT / (4 * CH);                   // vectors of a key in a lane: d = 4 CH kk + CH (lane / 16) + ..
    static constexpr int U = TYPE == COMET_F32 || DT == 64 ? 4 : 8;      // elements of a value that lie together in a lane: d = 16 U dd + U (lane % 16) + ..
    static constexpr int NV = DT / (16 * U);
    static constexpr int VW = U * (TYPE == COMET_F32 ? 4 : 2) / 4;       // ... in 32-bit words
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

// Which tokens a workgroup has.
struct Tile { int64_t b, first; int n; };

// Tile `tile` of those that cut every request's tokens into pieces of `tokens`; n = 0 where there are not as many.
template <int T> __device__ __forceinline__ Tile find_tile(const Queries &q, int tokens, int64_t tile, int64_t *buf, int64_t *where) {
    if (threadIdx.x == 0) where[0] = -1;
    const int64_t each = (q.B + T - 1) / T, b0 = threadIdx.x * each, b1 = b0 + each < q.B ? b0 + each : q.B;
    int64_t mine = 0, total;
    for (int64_t b = b0; b < b1; ++b) {
        const int n = q.pos[b + 1] - q.pos[b];
        mine += n > 0 ? (n + tokens - 1) / tokens : 0;
    }
    const int64_t upto = block_scan<T>(mine, buf, total);
    if (tile >= upto - mine && tile < upto) {
        int64_t left = tile - (upto - mine);
        for (int64_t b = b0; b < b1; ++b) {
            const int n = q.pos[b + 1] - q.pos[b], pieces = n > 0 ? (n + tokens - 1) / tokens : 0;
            if (left < pieces) {
                where[0] = b, where[1] = q.pos[b] + left * tokens, where[2] = n - left * tokens < tokens ? n - left * tokens : tokens;
                break;
            }
            left -= pieces;
        }
    }
    __syncthreads();
    Tile t{where[0], where[0] < 0 ? 0 : where[1], where[0] < 0 ? 0 : (int)where[2]};
    if (t.first + t.n > q.N) t.n = t.first < q.N ? (int)(q.N - t.first) : 0;
    __syncthreads();
    return t;
}

// What a workgroup works at.
struct Item { int64_t tile; int head, chunk, split; int64_t id; };
__device__ __forceinline__ bool item_of(const AttendArgs &a, Item &i) {
    // neighbouring workgroups go to the eight dies in turn, each of which has a cache of its own: a die gets a stretch of the items
    const int64_t all = a.tiles * a.heads * a.chunks * a.splits, each = gridDim.x / 8;
    int64_t x = (blockIdx.x & 7) * each + (blockIdx.x >> 3);
    if (x >= all) return false;
    const int hc = a.heads * a.chunks;
    int at;
    if (a.tokens == 1) {             // heads of one token next to each other: their keys are next to each other in memory
        at = (int)(x % hc), x /= hc;
        i.split = (int)(x % a.splits), i.tile = x / a.splits;
    } else {                         // tokens next to each other: they read the same keys
        i.split = (int)(x % a.splits), x /= a.splits;
        i.tile = x % a.tiles, at = (int)(x / a.tiles);
    }
    i.head = at / a.chunks, i.chunk = at % a.chunks;
    i.id = (i.tile * hc + at) * a.splits + i.split;
    return true;
}

// The union of the tokens' choices in LDS: entry i is block j[i] of the request, at id[i] in the cache (below 0: it is none), chosen by the tokens of mask[i].
struct List { int *j, *id; uint32_t *mask; int n; };
template <int T> __device__ __forceinline__ List make_list(const AttendArgs &a, const Tile &t, int head, int64_t place0, uint32_t *raw, int64_t *buf) {
    uint32_t *bits = raw, *before = raw + a.words;
    List l{(int *)(raw + 2 * a.words), (int *)(raw + 2 * a.words) + a.entries, raw + 2 * a.words + 2 * a.entries, 0};
    const auto seen = [&](int64_t place) {
        const int64_t c = place < 0 ? 0 : place / a.block + 1;
        return (int)(c < a.q.M ? c : a.q.M);
    };
    const int words = (seen(place0 + t.n - 1) + 31) / 32;
    for (int w = threadIdx.x; w < words; w += T) bits[w] = 0;
    __syncthreads();
    for (int e = threadIdx.x; e < t.n * a.K; e += T) {
        const int i = e / a.K, j = a.sel[((t.first + i) * a.heads + head) * a.K + (e - i * a.K)];
        if (j >= 0 && j < seen(place0 + i)) atomicOr(&bits[j >> 5], 1u << (j & 31));
    }
    __syncthreads();
    const int each = (words + T - 1) / T, w0 = threadIdx.x * each, w1 = w0 + each < words ? w0 + each : words;
    int64_t mine = 0, total;
    for (int w = w0; w < w1; ++w) mine += __builtin_popcount(bits[w]);
    int at = (int)(block_scan<T>(mine, buf, total) - mine);
    for (int w = w0; w < w1; ++w) {
        before[w] = at;
        for (uint32_t left = bits[w]; left; left &= left - 1) l.j[at++] = w * 32 + __builtin_ctz(left);
    }
    l.n = (int)total;
    __syncthreads();
    const int32_t *table = a.q.table + t.b * a.q.ldt;
    for (int i = threadIdx.x; i < l.n; i += T) {
        const int id = table[l.j[i]];
        l.id[i] = id >= 0 && id < a.blocks ? id : -1;
        l.mask[i] = 0;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < t.n * a.K; e += T) {
        const int i = e / a.K, j = a.sel[((t.first + i) * a.heads + head) * a.K + (e - i * a.K)];
        if (j >= 0 && j < seen(place0 + i)) {
            const int x = (int)before[j >> 5] + __builtin_popcount(bits[j >> 5] & ((1u << (j & 31)) - 1));
            if (l.id[x] >= 0) atomicOr(&l.mask[x], 1u << i);
        }
    }
    __syncthreads();
    return l;
}

__device__ __forceinline__ float xor16(float v) { return __shfl_xor(v, 16); }
__device__ __forceinline__ float xor32(float v) { return __shfl_xor(v, 32); }

// Sixteen places of a block: where they are, who reads them.
struct Places {
    const char *key, *value;                  // the block's first place, of the head
    int start, last;                          // the first place's number in the block, the last one's that any of the tokens reads
    int from;                                 // ... and in the request
    uint32_t mask;
};

template <int TYPE, int DT> struct Data {
    using S = Shape<TYPE, DT>;
    U4 k[2][S::NK];
    uint32_t v[8][S::NV * S::VW];
};

template <int TYPE, int DT, int MT>
__global__ void __launch_bounds__(kAttend, MT >= 4 || DT > 128 ? 1 : 2) k_attend(AttendArgs a) {
    using S = Shape<TYPE, DT>;
    using E = Elem<TYPE>;
    using T = typename E::T;
    constexpr int SIZE = (int)sizeof(T), OT = DT / 16, LINE = DT + 4;
    extern __shared__ __align__(16) uint32_t raw[];
    __shared__ int64_t buf[kWaves], where[3];
    __shared__ float2 ml[kWaves][16];
    Item item;
    if (!item_of(a, item)) return;
    const Tile t = find_tile<kAttend>(a.q, a.tokens, item.tile, buf, where);
    if (t.n == 0) return;
    const int64_t place0 = a.q.length[t.b] - ((int64_t)a.q.pos[t.b + 1] - t.first), place1 = place0 + t.n - 1;
    const List list = make_list<kAttend>(a, t, item.head, place0, raw, buf);

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
        const int i0 = 16 * m / heads, i1 = (16 * m + 15) / heads;
        of_tile[m] = 0;
        for (int k = i0; k <= i1 && k < t.n; ++k) of_tile[m] |= 1u << k;
        of_tile[m] = __builtin_amdgcn_readfirstlane(of_tile[m]);
        const T *from = (const T *)a.q.q + (t.first + i) * a.q.row + (int64_t)(x0 + r - i * heads) * a.q.head;
#pragma unroll
        for (int kk = 0; kk < S::NK; ++kk) {
            const int d = (4 * kk + g) * S::CH;
            q[m][kk] = U4{0, 0, 0, 0};
            if (r < rows && d < a.size) q[m][kk] = *(const U4 *)(from + d);
        }
    }
    const uint32_t everyone = t.n == 32 ? ~0u : (1u << t.n) - 1;

    const int per = a.block / 16;             // sixteens of a block
    const int sixteens = list.n * per, pairs = (sixteens + 1) / 2;
    const int begin = (int)((int64_t)pairs * item.split / a.splits), end = (int)((int64_t)pairs * (item.split + 1) / a.splits);

    const auto places = [&](int s) {
        Places p{nullptr, nullptr, 0, 0, 0, 0};
        if (s >= sixteens) return p;
        const int e = s / per, j = __builtin_amdgcn_readfirstlane(list.j[e]), id = __builtin_amdgcn_readfirstlane(list.id[e]);
        p.start = (s - e * per) * 16;
        p.from = j * a.block + p.start;
        const int64_t last = place1 - (int64_t)j * a.block;
        p.last = (int)(last < a.block ? last : a.block - 1);
        p.mask = p.start <= p.last ? __builtin_amdgcn_readfirstlane(list.mask[e]) : 0;
        if (id < 0) p.mask = 0;
        p.key = a.keys + id * a.key_stride[0] + item.head * a.key_stride[2];
        p.value = a.values + id * a.value_stride[0] + item.head * a.value_stride[2];
        return p;
    };
    const bool ragged = a.size % (4 * S::CH) != 0;
    // Places behind the last one that is read are taken from there: nothing comes from memory that no token reads.
    const auto load = [&](const Places &p0, const Places &p1, Data<TYPE, DT> &x) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const Places &p = h ? p1 : p0;
            if (p.mask) {
                const int i = p.start + col < p.last ? p.start + col : p.last;
                const char *from = p.key + (int64_t)i * a.key_stride[1];
#pragma unroll
                for (int kk = 0; kk < S::NK; ++kk) {
                    const int d = (4 * kk + g) * S::CH;
                    x.k[h][kk] = *(const U4 *)(from + (d < a.size ? d * SIZE : 0));
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int iv = p.start + 4 * g + r < p.last ? p.start + 4 * g + r : p.last;
                    const char *v = p.value + (int64_t)iv * a.value_stride[1];
#pragma unroll
                    for (int dd = 0; dd < S::NV; ++dd) {
                        const int d = 16 * S::U * dd + S::U * col;
                        const uint32_t *w = (const uint32_t *)(v + (d < a.size ? d * SIZE : 0));
                        if constexpr (S::VW == 2) {
                            const uint2 y = *(const uint2 *)w;
                            x.v[4 * h + r][2 * dd] = y.x, x.v[4 * h + r][2 * dd + 1] = y.y;
                        } else {
                            const U4 y = *(const U4 *)w;
#pragma unroll
                            for (int e = 0; e < 4; ++e) x.v[4 * h + r][4 * dd + e] = y[e];
                        }
                    }
                }
            } else {
#pragma unroll
                for (int kk = 0; kk < S::NK; ++kk) x.k[h][kk] = U4{0, 0, 0, 0};
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int e = 0; e < S::NV * S::VW; ++e) x.v[4 * h + r][e] = 0;
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

    const auto compute = [&](const Places &p0, const Places &p1, Data<TYPE, DT> &x) {
        if (ragged) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int kk = 0; kk < S::NK; ++kk)
                    if ((4 * kk + g) * S::CH >= a.size) x.k[h][kk] = U4{0, 0, 0, 0};
        }
        const bool whole = p0.mask == everyone && p1.mask == everyone && p0.from + 15 <= place0 && p1.from + 15 <= place0;
        float w[MT][8];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            if (!((p0.mask | p1.mask) & of_tile[m])) continue;
            F4 s[2] = {F4{0, 0, 0, 0}, F4{0, 0, 0, 0}};
#pragma unroll
            for (int kk = 0; kk < S::NK; ++kk) {
                if (4 * kk * S::CH >= a.size) continue;
                s[0] = product<TYPE>(x.k[0][kk], q[m][kk], s[0]);
                s[1] = product<TYPE>(x.k[1][kk], q[m][kk], s[1]);
            }
            float *z = w[m];
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = s[i / 4][i & 3] * a.c;
            if (!whole) {
                const int64_t mine = place0 + token[m];
                const int l0 = p0.mask >> token[m] & 1 ? (int)(mine - p0.from) : -1, l1 = p1.mask >> token[m] & 1 ? (int)(mine - p1.from) : -1;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    z[i] = 4 * g + i <= l0 ? z[i] : kNegInf;
                    z[4 + i] = 4 * g + i <= l1 ? z[4 + i] : kNegInf;
                }
            }
            float most = fmaxf(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])), fmaxf(fmaxf(z[4], z[5]), fmaxf(z[6], z[7])));
            // The maximum follows when a score is 256 times over it, and not before: weights are 256 at most, which costs nothing in floating
            // point, and the output is seldom scaled anew.
            if (__ballot(most > top[m] + 8.f)) {
                most = fmaxf(most, xor16(most));
                most = fmaxf(most, xor32(most));
                const float now = fmaxf(top[m], most), back = now == kNegInf ? 1.f : exp2_fast(top[m] - now);
                top[m] = now;
                sum[m] *= back;
#pragma unroll
                for (int c = 0; c < OT; ++c) o[m][c] *= back;
            }
            const float shift = top[m] == kNegInf ? 0.f : top[m];
            float add[2] = {0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                z[i] = exp2_fast(z[i] - shift);
                add[i & 1] += z[i];
            }
            sum[m] += add[0] + add[1];
        }
        if constexpr (TYPE == COMET_F32) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int c = 0; c < OT; ++c)
#pragma unroll
                    for (int m = 0; m < MT; ++m)
                        if ((p0.mask | p1.mask) & of_tile[m])
                            o[m][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x.v[i][c]), w[m][i], o[m][c], 0, 0, 0);
        } else {
            // Weights are rounded to the type: half a step each, of as many that their errors cancel; a product in 32 bits would take 16 times as long.
            U4 p[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const uint4 y = E::narrow(w[m]);
                p[m] = U4{y.x, y.y, y.z, y.w};
            }
#pragma unroll
            for (int c = 0; c < OT; ++c) {
                const int at = c / 2;
                U4 v;
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = __builtin_amdgcn_perm(x.v[2 * i + 1][at], x.v[2 * i][at], c & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
                for (int m = 0; m < MT; ++m)
                    if ((p0.mask | p1.mask) & of_tile[m]) o[m][c] = product<TYPE>(v, p[m], o[m][c]);
            }
        }
    };

    for (int i = begin + wave; i < end; i += kWaves) {
        const Places p0 = places(2 * i), p1 = places(2 * i + 1);
        if (!(p0.mask | p1.mask)) continue;
        Data<TYPE, DT> x;
        load(p0, p1, x);
        compute(p0, p1, x);
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
    float *line = (float *)raw + wave * 16 * LINE;
    // A row that came out as NaN once more, by itself: what it does not read weighs 0 in the products above, but 0 times a NaN or an infinity of
    // another row's is a NaN.  One place after the other, its own ones only.
    const auto alone = [&](int m, int n) {
        const int r = 16 * m + n;
        if (r >= rows) return;
        const int i = r / heads;
        const T *from = (const T *)a.q.q + (t.first + i) * a.q.row + (int64_t)(x0 + r - i * heads) * a.q.head;
        float high = kNegInf, total = 0.f, out[DT / kWave] = {};
        for (int pair = begin + wave; pair < end; pair += kWaves)
            for (int h = 0; h < 2; ++h) {
                const int s = 2 * pair + h;
                if (s >= sixteens) break;
                const int e = s / per, id = list.id[e];
                if (id < 0 || !(list.mask[e] >> i & 1)) continue;
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
    __syncthreads();                           // the list is not needed any more, unless a row is done again
    const bool again = __syncthreads_or(
        [&] { uint32_t b = 0;
#pragma unroll
              for (int m = 0; m < MT; ++m) b |= bad[m];
              return b != 0; }());
    if (again) line += 2 * a.words + 3 * a.entries;
    float *lines = (float *)raw + (again ? 2 * a.words + 3 * a.entries : 0);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        if (16 * m >= rows) break;
#pragma unroll
        for (int dd = 0; dd < S::NV; ++dd)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float *to = line + col * LINE + 16 * S::U * dd + S::U * (4 * g + r);
#pragma unroll
                for (int e = 0; e < S::U; e += 4)
                    *(F4 *)(to + e) = F4{o[m][dd * S::U + e][r], o[m][dd * S::U + e + 1][r], o[m][dd * S::U + e + 2][r], o[m][dd * S::U + e + 3][r]};
            }
        if (g == 0) ml[wave][col] = make_float2(top[m], sum[m]);
        if (bad[m]) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            for (uint32_t left = bad[m]; left; left &= left - 1) alone(m, __builtin_ctz(left));
        }
        __syncthreads();
        // sixteen threads a row, OT elements each
        const int n = threadIdx.x / 16, d0 = (threadIdx.x & 15) * OT, r = 16 * m + n;
        if (r < rows) {
            float high = kNegInf, total = 0.f, part[kWaves], out[OT] = {};
#pragma unroll
            for (int w = 0; w < kWaves; ++w) high = fmaxf(high, ml[w][n].x);
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float2 y = ml[w][n];
                part[w] = y.x == high || y.x != y.x ? 1.f : y.x == kNegInf ? 0.f : exp2_fast(y.x - high);
                total += y.y * part[w];
            }
#pragma unroll
            for (int w = 0; w < kWaves; ++w)
                if (part[w] != 0.f)
#pragma unroll
                    for (int e = 0; e < OT; ++e) out[e] = __builtin_fmaf(lines[(w * 16 + n) * LINE + d0 + e], part[w], out[e]);
            if (a.splits > 1) {
                float *to = a.part + (item.id * (16 * MT) + r) * (DT + 4);
                if (d0 == 0) to[DT] = high, to[DT + 1] = total;
#pragma unroll
                for (int e = 0; e < OT; e += 4) *(F4 *)(to + d0 + e) = F4{out[e], out[e + 1], out[e + 2], out[e + 3]};
            } else {
                const int i = r / heads;
                const int64_t row = (t.first + i) * a.q.Q + x0 + r - i * heads;
                const float by = total == 0.f ? 0.f : 1.f / total;
                T *to = (T *)a.out + row * a.size + d0;
#pragma unroll
                for (int e = 0; e < OT; ++e)
                    if (d0 + e < a.size) to[e] = (T)E::bits(total == 0.f ? 0.f : out[e] * by);
                if (d0 == 0 && a.lse) a.lse[row] = total == 0.f ? kNegInf : (high + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
            }
        }
        __syncthreads();
    }
}

// The parts of a tile that several workgroups share: one workgroup a tile and head, a wavefront a row.
template <int TYPE, int DT, int MT>
__global__ void __launch_bounds__(kAttend) k_attend_join(AttendArgs a) {
    using E = Elem<TYPE>;
    __shared__ int64_t buf[kWaves], where[3];
    const int hc = a.heads * a.chunks;
    const int64_t tile = blockIdx.x / hc;
    const int at = (int)(blockIdx.x % hc), head = at / a.chunks, chunk = at % a.chunks;
    const Tile t = find_tile<kAttend>(a.q, a.tokens, tile, buf, where);
    const int heads = a.group - chunk * a.chunk < a.chunk ? a.group - chunk * a.chunk : a.chunk, x0 = head * a.group + chunk * a.chunk;
    const int lane = threadIdx.x & (kWave - 1);
    const float *from = a.part + (int64_t)blockIdx.x * a.splits * (16 * MT) * (DT + 4);
    for (int r = threadIdx.x / kWave; r < t.n * heads; r += kWaves) {
        float high = kNegInf, total = 0.f, out[DT / kWave] = {};
        for (int s = 0; s < a.splits; ++s) {
            const float *p = from + (s * 16 * MT + r) * (DT + 4);
            const float m = p[DT], sum = p[DT + 1], now = fmaxf(high, m);
            const float old = high == now ? 1.f : high == kNegInf ? 0.f : exp2_fast(high - now), add = m == now || m != m ? 1.f : m == kNegInf ? 0.f : exp2_fast(m - now);
            total = total * old + sum * add;
#pragma unroll
            for (int u = 0; u < DT / kWave; ++u) out[u] = out[u] * old + (add == 0.f ? 0.f : p[u * kWave + lane] * add);
            high = now;
        }
        const int i = r / heads;
        const int64_t row = (t.first + i) * a.q.Q + x0 + r - i * heads;
#pragma unroll
        for (int u = 0; u < DT / kWave; ++u) {
            const int d = u * kWave + lane;
            if (d < a.size) ((typename E::T *)a.out)[row * a.size + d] = (typename E::T)E::bits(total == 0.f ? 0.f : out[u] / total);
        }
        if (lane == 0 && a.lse) a.lse[row] = total == 0.f ? kNegInf : (high + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
    }
}

template <int TYPE, int DT, int MT> hipError_t attend_run(const AttendArgs &a, hipStream_t st) {
    const int64_t items = a.tiles * a.heads * a.chunks * a.splits;
    const size_t list = (size_t)(2 * a.words + 3 * a.entries) * 4, lds = list + (size_t)kWaves * 16 * (DT + 4) * 4;
    hipError_t e = hipSuccess;
    if (lds > 65536) e = hipFuncSetAttribute((const void *)k_attend<TYPE, DT, MT>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_attend<TYPE, DT, MT>), dim3((unsigned)((items + 7) / 8 * 8)), dim3(kAttend), lds, st, a);
    e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    hipLaunchKernelGGL((k_attend_join<TYPE, DT, MT>), dim3((unsigned)(a.tiles * a.heads * a.chunks)), dim3(kAttend), 0, st, a);
    return hipGetLastError();
}

template <int TYPE> hipError_t attend_type(const AttendArgs &a, int wide, int mt, hipStream_t st) {
    const auto with = [&](auto d) {
        constexpr int DT = decltype(d)::value;
        return mt == 1 ? attend_run<TYPE, DT, 1>(a, st) : mt == 2 ? attend_run<TYPE, DT, 2>(a, st) : attend_run<TYPE, DT, 4>(a, st);
    };
    if (wide == 64) return with(std::integral_constant<int, 64>());
    if (wide == 128) return with(std::integral_constant<int, 128>());
    return with(std::integral_constant<int, 256>());
}
hipError_t attend_f32(const AttendArgs &a, int wide, int mt, hipStream_t st);
hipError_t attend_bf16(const AttendArgs &a, int wide, int mt, hipStream_t st);
hipError_t attend_f16(const AttendArgs &a, int wide, int mt, hipStream_t st);

}  // namespace comet
