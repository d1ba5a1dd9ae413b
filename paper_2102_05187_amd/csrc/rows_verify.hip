// Drafted tokens against the target's logits.
#include "rows_kernels.hpp"
#include "cache.hpp"

namespace comet {

namespace {

// How the draft's distribution is known: not at all (the token has all of it), by some of its logits, by all of them.
enum { kPoint = 0, kEntries = 1, kDense = 2 };

constexpr int kRow = 256, kWavesRow = kRow / kWave;
constexpr int kParts = 32;                    // parts of a piece whose weights are kept: of a wavefront's vectors that lie next to each other

// A thread has VEC 16-byte vectors of a piece, a piece VEC * kRow.  Long rows, or many, are cut into pieces of 2048 vectors, few short ones into
// pieces of 512, so that there are more workgroups, whose latency is what such calls take (8 rows of 32000 32-bit logits: 18 us, 21 in pieces of 2048).
int vectors_of(int64_t N, int64_t V) { return N * V < int64_t(1) << 20 ? 2 : 8; }
int64_t pieces_of(int type, int64_t N, int64_t V) {
    const int64_t n = kRow * vectors_of(N, V) * (type == COMET_F32 ? 4 : 8);
    return V > n ? (V + n - 1) / n : 1;
}

// exp2 in 64 bits for arguments of at most 0: the nearest whole number taken off, by adding 1.5 2^52, and a polynomial for |f| <= 1/2, which goes
// through 2^f at the ten zeros of a Chebyshev polynomial (off by 2e-14 at most).  Below -1000 it is 2^-1000, or 0 where ZERO.  A NaN is not kept.
template <bool ZERO> __device__ __forceinline__ double exp2_wide(double x) {
    const double low = __builtin_fmax(x, -1000.0), big = low + 0x1.8p52, f = low - (big - 0x1.8p52);
    double r = 0x1.b6557c7da8ca4p-24;
    r = __builtin_fma(r, f, 0x1.63efd536dcb25p-20);
    r = __builtin_fma(r, f, 0x1.ffcb7a04d3b13p-17);
    r = __builtin_fma(r, f, 0x1.43088df6dd4a7p-13);
    r = __builtin_fma(r, f, 0x1.5d87fe8e6c4b1p-10);
    r = __builtin_fma(r, f, 0x1.3b2ab72b2b245p-7);
    r = __builtin_fma(r, f, 0x1.c6b08d7045e60p-5);
    r = __builtin_fma(r, f, 0x1.ebfbdff814945p-3);
    r = __builtin_fma(r, f, 0x1.62e42fefa39e9p-1);
    r = __builtin_fma(r, f, 0x1.000000000003dp+0);
    const double y = __hiloint2double(__double2hiint(r) + (__double2loint(big) << 20), __double2loint(r));
    return ZERO && !(x > -1000.0) ? 0.0 : y;
}

// exp2(z c - R) for the logits of a row, or of a piece of one, R the whole number next to m c, m the largest of them.  With t = 16 z c and n the whole
// number next to it, which is found by one multiply-add with 1.5 2^52 - 16 R, it is 2^(n / 16 - R) 2^((t - n) / 16): a sixteenth root of 2 from LDS with its
// exponent, times a polynomial (through 2^(f / 16) at the six zeros of a Chebyshev polynomial, off by 1e-14 at most).  t - n is one multiply-add,
// and exact: no difference of z and m is rounded, and the 64-bit instructions, which take twice as long as those of 32 bits, are ten (17 with exp2_wide of
// (z - m) c).  They bound the sums and the draw all the same: 42 million powers of 320 rows of 131072 44 us (46 with 17), where reading the rows takes 12.
// Sums in 32 bits would take half of it, but not say which token a number draws: a token of the tail has 1e-8 of the whole.
struct Powers {
    double c, m, c16, magic, unit;            // unit: what makes it exp2((z - m) c)
    float low;                                // the logit whose power is about 2^-1000: logits are raised to it
    // m c is below 2^26.  low, which is rounded to 32 bits, is off by half a step then, 2^-24 of its size: four exponents at most, so that its power is
    // one that 64 bits hold.  At 2^28 it is sixteen, from about 2^29 on the exponent wraps into the sign, and from 2^34 on low can be m itself.
    bool plain;
    const double *root;                       // LDS, [16]
    __device__ __forceinline__ Powers(double m, double c, const double *root) : c(c), m(m), root(root) {
        const double R = __builtin_rint(m * c);
        c16 = 16 * c, magic = 0x1.8p52 - 16 * R;
        low = (float)((R - 1000) / c);
        plain = fabs(m * c) < 0x1p26 && c < 0x1p100 && low > kNegInf;
        unit = plain ? exp2_wide<false>(__builtin_fma(-m, c, R)) : 1;
    }
    // the scaled root, and the polynomial that goes with it
    __device__ __forceinline__ double parts(float z, double &poly) const {
        const double x = z > low ? z : low, big = __builtin_fma(x, c16, magic), f = __builtin_fma(x, c16, magic - big);
        const int n = __double2loint(big);
        const double t = root[n & 15];
        double r = 0x1.5d8b6e76d3913p-30;
        r = __builtin_fma(r, f, 0x1.3b2c9c307f552p-23);
        r = __builtin_fma(r, f, 0x1.c6b08d6b1d71bp-17);
        r = __builtin_fma(r, f, 0x1.ebfbdff5547dcp-11);
        r = __builtin_fma(r, f, 0x1.62e42fefa3a3dp-5);
        poly = __builtin_fma(r, f, 0x1.0000000000015p+0);
        return __hiloint2double(__double2hiint(t) + (n >> 4 << 20), __double2loint(t));
    }
    // N of them, added up; PLAIN as it is above
    template <bool PLAIN, int N> __device__ __forceinline__ double sum(const float *z, double s) const {
        double t[N], poly[N], s2 = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            if (PLAIN) t[e] = parts(z[e], poly[e]);
            else t[e] = exp2_wide<false>(((double)z[e] - m) * c), poly[e] = 1;
        }
#pragma unroll
        for (int e = 0; e < N; e += 2) s = __builtin_fma(t[e], poly[e], s), s2 = __builtin_fma(t[e + 1], poly[e + 1], s2);
        return s + s2;
    }
    template <bool PLAIN> __device__ __forceinline__ double one(float z) const {
        if (!PLAIN) return exp2_wide<true>(((double)z - m) * c);
        double poly;
        const double t = parts(z, poly);
        return z > low ? t * poly : 0;
    }
};
__device__ __forceinline__ void make_roots(double *root) {
    if (threadIdx.x < 16) root[threadIdx.x] = exp2_wide<false>(threadIdx.x / 16.0);
}

// The sum of exp2((z - m) c) over a part of a row, m its largest logit: of nothing, m is -inf; with a NaN or +inf in it, s is a NaN.
struct Sum {
    double s;
    double m;
    __device__ __forceinline__ bool good() const { return s > 0; }
};
// What a part's sum is relative to a larger maximum.
__device__ __forceinline__ double onto(Sum a, double m, double c) { return a.m == m || a.s == 0 || a.s != a.s ? a.s : a.s * exp2_wide<true>((a.m - m) * c); }
// Over groups of `over` lanes, a power of two.
__device__ __forceinline__ Sum group_join(Sum a, int over, double c) {
    double m = a.m;
    for (int d = 1; d < over; d *= 2) {
        const double y = __shfl_xor(m, d);
        m = y > m ? y : m;
    }
    double s = onto(a, m, c);
    for (int d = 1; d < over; d *= 2) s += __shfl_xor(s, d);
    return Sum{s, m};
}
__device__ __forceinline__ Sum two(Sum a, Sum b, double c) {
    const double m = a.m > b.m ? a.m : b.m;
    return Sum{onto(a, m, c) + onto(b, m, c), m};
}

struct VerifyArgs {
    const void *Z;
    int64_t N, V, ldz, B;
    const int32_t *pos, *token;
    const float *u, *v;
    const void *draft;
    int64_t ldd;
    const int32_t *crd;
    const float *vals;
    int64_t K;
    double scale;
    const float *scales;
    int32_t *accepted, *next, *length;
    Sum *target, *drafted;                    // [N x pieces], [N x draft_pieces]
    double *weight;                           // [B x pieces x kParts]: what is drawn from
    int32_t *arrived;                         // [B]
    int32_t pieces, draft_pieces;

    // scale log2 e of a request; NaN where it is no scale, +inf where the largest logit is taken
    __device__ __forceinline__ double of(int64_t b) const {
        const double s = scales ? (double)scales[b] : scale;
        return s > 0 ? s * 1.4426950408889634 : __builtin_nan("");
    }
    // the request of a row, by every wavefront for itself where there are no more than 256
    __device__ __forceinline__ int64_t request(int64_t row, int *count) const {
        if (B > 4 * kWave) return request_of<kRow>(pos, B, row, count);
        int32_t end[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int b = i * kWave + (int)(threadIdx.x & (kWave - 1));
            end[i] = b < B ? pos[b + 1] : 0x7fffffff;
        }
        int n = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) n += __builtin_popcountll(__ballot(end[i] <= row));
        return n < B && row >= pos[n] ? n : -1;
    }
};

// One piece of one row.
template <int TYPE, int VEC>
__device__ __forceinline__ void piece_sum(const void *base, int64_t row, int64_t ld, int64_t V, int64_t piece, double c, Sum *out) {
    using E = Elem<TYPE>;
    __shared__ float top[kWavesRow];
    __shared__ double part[kWavesRow], root[16];
    make_roots(root);
    const Row<TYPE> r(base, row, ld, V);
    const int64_t v0 = piece * (kRow * VEC);
    uint4 x[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        const int64_t i = v0 + j * kRow + threadIdx.x;
        if (r.whole(i)) {
            x[j] = r.raw(i);
        } else {
            float f[E::kPer];
            r.load(i, f);
            x[j] = E::narrow(f);
        }
    }
    const auto larger = [](float a, float b) { return __builtin_elementwise_maximum(a, b); };      // a NaN stays
    float m = kNegInf;
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        float f[E::kPer];
        E::widen(x[j], f);
#pragma unroll
        for (int e = 0; e < E::kPer; ++e) m = larger(m, f[e]);
    }
    m = wave_reduce(m, kNegInf, larger);
    if ((threadIdx.x & (kWave - 1)) == 0) top[threadIdx.x / kWave] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWavesRow; ++w) m = larger(m, top[w]);
    double s = 0;
    if (c == __builtin_huge_val()) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            float f[E::kPer];
            E::widen(x[j], f);
#pragma unroll
            for (int e = 0; e < E::kPer; ++e) s += f[e] == m ? 1.0 : 0.0;
        }
    } else {
        const Powers power(m, c, root);
        if (power.plain)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                float f[E::kPer];
                E::widen(x[j], f);
#pragma unroll
                for (int e = 0; e < E::kPer; e += 4) {
                    s = power.sum<true, 4>(f + e, s);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        else
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                float f[E::kPer];
                E::widen(again(x[j]), f);
                s = power.sum<false, E::kPer>(f, s);
            }
        s *= power.unit;
    }
    s = wave_reduce(s, 0.0, Add());
    if ((threadIdx.x & (kWave - 1)) == 0) part[threadIdx.x / kWave] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kWavesRow; ++w) s += part[w];
        if (m == kNegInf) s = 0;
        if (!(m < -kNegInf) || c != c) s = __builtin_nan("");
        *out = Sum{s, m != m ? kNegInfD : (double)m};
    }
}

// Sums of all pieces of all rows that are judged by or drawn from.
template <int TYPE, int DRAFT, int VEC>
__global__ void __launch_bounds__(kRow) k_verify_sums(VerifyArgs a, uint32_t from) {
    __shared__ int count;
    const uint32_t item = from + blockIdx.x, all = a.pieces + a.draft_pieces;
    const int row = (int)(item / all);
    int piece = (int)(item - row * all);
    for (int64_t b = (int64_t)blockIdx.x * kRow + threadIdx.x; b < a.B; b += (int64_t)gridDim.x * kRow) a.arrived[b] = 0;
    const int64_t b = a.request(row, &count);
    if (b < 0) return;
    const double c = a.of(b);
    if (piece < a.pieces) {
        piece_sum<TYPE, VEC>(a.Z, row, a.ldz, a.V, piece, c, a.target + (int64_t)row * a.pieces + piece);
    } else if (row + 1 < a.pos[b + 1]) {
        piece -= a.pieces;
        piece_sum<DRAFT, VEC>(a.draft, row, a.ldd, a.V, piece, c, a.drafted + (int64_t)row * a.draft_pieces + piece);
    }
}

// What is drawn from at one row, where the target's and the draft's sums are known.
template <int TYPE, int DRAFT, int MODE> struct Left {
    Row<TYPE> z;
    Row<DRAFT> x;
    Sum p, q;
    Powers of_p, of_q;
    double p_part, q_part;                    // what makes a power a probability; the second one 0 where there is none
    bool plain;                               // how the powers are computed: both rows' in one way
    bool rejected, largest;                   // something of the draft is taken off; only the largest logit counts
    int64_t d;
    const uint16_t *at;                       // kEntries: 1 + the entry of a place of the piece, 0: none
    const double *chance;                     //           and the entries' probabilities
    static constexpr int PER = Elem<TYPE>::kPer, DRAFT_PER = Elem<DRAFT>::kPer, MORE = DRAFT_PER < PER ? 2 : 1;
    // the logits of vector i, as they are in memory: the target's, and of the draft as many or, where its vectors are longer, those around them
    struct Logits { uint4 z, x[MODE == kDense ? MORE : 1]; };
    template <int K> static __device__ __forceinline__ uint4 vector(const Row<K> &row, int64_t i) {
        if (row.whole(i)) return row.raw(i);
        float f[Elem<K>::kPer];
        row.load(i, f);
        return Elem<K>::narrow(f);
    }
    __device__ __forceinline__ Logits logits(int64_t i) const {
        Logits v;
        v.z = vector<TYPE>(z, i);
        if constexpr (MODE == kDense) {
#pragma unroll
            for (int k = 0; k < MORE; ++k) {
                v.x[k] = make_uint4(0, 0, 0, 0);
                if (rejected) v.x[k] = vector<DRAFT>(x, DRAFT_PER > PER ? i / 2 : MORE * i + k);
            }
        }
        return v;
    }
    // its weights; `in` its number in the piece
    __device__ __forceinline__ void weights(int64_t i, int in, const Logits &v, double *w) const {
        if (plain) weights_as<true>(i, in, v, w);
        else weights_as<false>(i, in, v, w);
    }
    template <bool PLAIN> __device__ __forceinline__ void weights_as(int64_t i, int in, const Logits &v, double *w) const {
        float f[PER], g[MODE == kDense ? (DRAFT_PER > PER ? DRAFT_PER : PER) : 1];
        Elem<TYPE>::widen(v.z, f);
        if constexpr (MODE == kDense) {
#pragma unroll
            for (int k = 0; k < MORE; ++k) Elem<DRAFT>::widen(v.x[k], g + k * DRAFT_PER);
            if constexpr (DRAFT_PER > PER) {
#pragma unroll
                for (int e = 0; e < PER; ++e) g[e] = i & 1 ? g[PER + e] : g[e];
            }
        }
        if (largest) {
#pragma unroll
            for (int e = 0; e < PER; ++e) w[e] = (double)f[e] == p.m ? 1 : 0;
            return;
        }
#pragma unroll
        for (int e = 0; e < PER; ++e) w[e] = of_p.template one<PLAIN>(f[e]) * p_part;
        if (!rejected) return;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            double off = 0;
            if (MODE == kPoint) off = z.first(i) + e == d ? 1 : 0;
            if constexpr (MODE == kDense) off = of_q.template one<PLAIN>(g[e]) * q_part;
            if (MODE == kEntries) {
                const int k = at[in * PER + e];
                off = k ? chance[k - 1] : 0;
            }
            w[e] = w[e] > off ? w[e] - off : 0;
        }
    }
};

// One piece of the row that a request's next token is drawn from.  Each workgroup finds for itself how far the drafted tokens are taken; the one that
// is done last has all parts' weights, and draws.  Bound by 64-bit instructions where rows are long (64 requests, 131072 logits and the draft's: 39 us, of which the
// weights 20), else by the latency of its steps: requests, tokens, sums, logits, weights, and what the last one has to read again, each a read
// from memory that the one before it names (2 requests, 32000 logits: 16 us, of which 4 until it is known how far they are taken, and 6 for choosing a part).
template <int TYPE, int DRAFT, int MODE, int VEC>
__global__ void __launch_bounds__(kRow) k_verify_draw(VerifyArgs a, uint32_t from) {
    constexpr int PER = Elem<TYPE>::kPer, kPiece = kRow * VEC;
    constexpr int kMine = VEC * kWavesRow;       // a part for each wavefront's vectors next to each other
    static_assert(kMine <= kParts && kMine <= kWave, "one wavefront writes them");
    __shared__ int first, final_one, chosen_part, behind;
    __shared__ double part[kWavesRow], sums[kParts], chance[MODE == kEntries ? COMET_MAX_TOP : 1], before_part, goal_;
    __shared__ double root[16];
    __shared__ uint16_t at[MODE == kEntries ? kPiece * PER : 1];
    make_roots(root);
    __shared__ Sum known[2][kRow / 8];
    const uint32_t item = from + blockIdx.x;
    const int b = (int)(item / (unsigned)a.pieces), piece = (int)(item - (uint32_t)b * a.pieces);
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t r0 = a.pos[b], n = (a.pos[b + 1] < a.N ? a.pos[b + 1] : a.N) - r0;
    if (n <= 0 || r0 < 0) {
        if (piece == 0 && threadIdx.x == 0) a.accepted[b] = 0, a.next[b] = -1;
        return;
    }
    const double c = a.of(b);
    const bool largest = c == __builtin_huge_val();
    const auto usable = [&](const Sum &p) { return largest ? p.m > kNegInfD && p.m < -kNegInfD && p.s == p.s : p.good(); };
    // rows in groups of lanes: 8 lanes a row, or a wavefront where there are entries or many pieces
    const int over = MODE == kEntries || a.pieces > 64 || a.draft_pieces > 64 ? kWave : 8, at_once = kRow / over, group = threadIdx.x / over, l = threadIdx.x % over;
    const auto row_sum = [&](const Sum *s, int pieces) {
        Sum x{0, kNegInfD};
        for (int i = l; i < pieces; i += over) x = two(x, s[i], c);
        return group_join(x, over, c);
    };
    if (threadIdx.x == 0) first = (int)(n - 1);
    __syncthreads();
    int took = 0, slot = 0;
    for (int64_t i0 = 0; i0 < n; i0 += at_once) {
        const int64_t i = i0 + group, row = r0 + (i < n ? i : n - 1);
        const bool judged = i < n - 1;
        const int64_t d = judged ? a.token[row + 1] : -1;
        const bool real = d >= 0 && d < a.V;
        float z = 0, x = 0, u = 0;
        if (judged) u = a.u[row];
        if (real) z = Elem<TYPE>::one(((const typename Elem<TYPE>::T *)a.Z)[row * a.ldz + d]);
        if (MODE == kDense && real) x = Elem<DRAFT>::one(((const typename Elem<DRAFT>::T *)a.draft)[row * a.ldd + d]);
        const Sum p = row_sum(a.target + row * a.pieces, a.pieces);
        Sum s{0, kNegInfD};
        double q = 1;
        if (MODE == kDense && judged) {
            s = row_sum(a.drafted + row * a.draft_pieces, a.draft_pieces);
            q = s.good() ? exp2_wide<true>(((double)x - s.m) * c) / s.s : 0;
        }
        if (MODE == kEntries) {
            double mine = 0;
            for (int64_t k = l; k < a.K && judged; k += over) {
                const int64_t col = a.crd[row * a.K + k];
                const double t = a.vals[row * a.K + k];
                if (col < 0 || col >= a.V || t == kNegInfD) continue;
                const Sum one{t - t == 0 ? 1.0 : __builtin_nan(""), t == t ? t : kNegInfD};
                s = k < over ? one : two(s, one, c);
            }
            s = group_join(s, over, c);
            for (int64_t k = l; k < a.K && judged; k += over)
                if (a.crd[row * a.K + k] == d) mine += exp2_wide<true>(((double)a.vals[row * a.K + k] - s.m) * c);
            for (int e = 1; e < over; e *= 2) mine += __shfl_xor(mine, e);
            q = s.good() ? mine / s.s : 0;
        }
        bool take = false;
        if (real && usable(p)) take = largest ? p.m == (double)z : (double)u * q < exp2_wide<true>(((double)z - p.m) * c) / p.s;
        if (l == 0) {
            known[0][group] = p, known[1][group] = s;
            if (judged && !take) atomicMin(&first, (int)i);
        }
        __syncthreads();
        took = first;
        slot = (int)(took - i0);
        if (took < i0 + at_once) break;
        __syncthreads();
    }
    const int64_t row = r0 + took;
    if (piece == 0 && threadIdx.x == 0) {
        a.accepted[b] = took;
        if (a.length) a.length[b] -= (int32_t)(n - 1 - took);
    }
    Left<TYPE, DRAFT, MODE> left{Row<TYPE>(a.Z, row, a.ldz, a.V), Row<DRAFT>(a.draft, MODE == kDense ? row : 0, a.ldd, a.V), known[0][slot], known[1][slot], Powers(known[0][slot].m, c, root),
                                 Powers(MODE == kDense && known[1][slot].good() ? known[1][slot].m : 0, c, root), 0, 0, false,
                                 took < n - 1 && !largest, largest, took < n - 1 ? a.token[row + 1] : -1, at, chance};
    if (!usable(left.p)) {
        if (piece == 0 && threadIdx.x == 0) a.next[b] = -1;
        return;
    }
    left.plain = left.of_p.plain && (MODE != kDense || left.of_q.plain);
    left.p_part = (left.plain ? left.of_p.unit : 1) / left.p.s;
    left.q_part = left.q.good() ? (MODE == kDense && left.plain ? left.of_q.unit : 1) / left.q.s : 0;
    // a draft row without probabilities takes nothing off, whatever its logits: 0 times the power of +inf would be a NaN
    if (MODE != kPoint && !left.q.good()) left.rejected = false;
    // the entries that lie in a piece, by place
    const auto lay_out = [&](int64_t of) {
        if (MODE != kEntries || !left.rejected) return;
        __syncthreads();
        for (int i = threadIdx.x; i < kPiece * PER; i += kRow) at[i] = 0;
        __syncthreads();
        if (left.q_part > 0)
            for (int64_t k = threadIdx.x; k < a.K; k += kRow) {
                const int64_t col = a.crd[row * a.K + k], to = col - of * kPiece * PER;
                chance[k] = exp2_wide<true>(((double)a.vals[row * a.K + k] - left.q.m) * c) * left.q_part;
                if (col >= 0 && col < a.V && to >= 0 && to < kPiece * PER) at[to] = (uint16_t)(k + 1);
            }
        __syncthreads();
    };
    // the weights of a piece's parts: part j * 4 + w are the vectors of wavefront w at j, in the order of the row
    const auto piece_parts = [&](int64_t of, auto put) {
        // all are asked for before the first is waited for: eight vectors and the draft's take 44 thousand clocks, 52 with the next one under way only
        typename Left<TYPE, DRAFT, MODE>::Logits v[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[j] = left.logits(of * kPiece + j * kRow + threadIdx.x);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            double w[PER], s = 0;
            left.weights(of * kPiece + j * kRow + threadIdx.x, j * kRow + threadIdx.x, v[j], w);
#pragma unroll
            for (int e = 0; e < PER; ++e) s += w[e];
            s = wave_reduce(s, 0.0, Add());
            if (lane == 0) put(j * kWavesRow + wave, s);
        }
    };
    lay_out(piece);
    double *weight = a.weight + (int64_t)b * a.pieces * kParts;
    piece_parts(piece, [&](int i, double s) { sums[i] = s; });
    __syncthreads();
    if (threadIdx.x < kMine) __hip_atomic_store(weight + piece * kParts + threadIdx.x, sums[threadIdx.x], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();                             // thread 0 makes known what all of them have stored
    if (threadIdx.x == 0) final_one = __hip_atomic_fetch_add(a.arrived + b, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == a.pieces - 1;
    __syncthreads();
    if (!final_one) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");

    // Of `count` weights in order the first at which their running sum, from `upto` on, is beyond the goal: chosen_part, and the sum before it.  Where there is
    // none, the last one that has a weight.  The goal is v times the sum of all where v is given (0 and above).
    const auto choose = [&](int count, auto get, double v, double goal) {
        if (threadIdx.x == 0) chosen_part = 0x7fffffff, behind = -1;
        const int each = (count + kRow - 1) / kRow, i0 = threadIdx.x * each, i1 = i0 + each < count ? i0 + each : count;
        double mine = 0, kept[4];
        if (each <= 4) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                kept[k] = 0;
                if (i0 + k < i1) kept[k] = get(i0 + k);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) mine += kept[k];
        } else {
            for (int i = i0; i < i1; ++i) mine += get(i);
        }
        double run = mine;
#pragma unroll
        for (int step = 1; step < kWave; step *= 2) {
            const double y = __shfl_up(run, step);
            if (lane >= step) run += y;
        }
        if (lane == kWave - 1) part[wave] = run;
        __syncthreads();
        double upto = run - mine, all = 0;
        for (int w = 0; w < kWavesRow; ++w) {
            if (w < wave) upto += part[w];
            all += part[w];
        }
        if (v >= 0) goal = v * all;
        int last = -1, hit = -1;
        double x = upto, before = 0;
        const auto take = [&](int i, double w) {
            if (w > 0) last = i;
            if (hit < 0 && w > 0 && x + w > goal) hit = i, before = x;          // a running sum of another rounding may be beyond it already
            x += w;
        };
        if (each <= 4) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i0 + k < i1) take(i0 + k, kept[k]);
        } else {
            for (int i = i0; i < i1; ++i) take(i, get(i));
        }
        if (hit >= 0) atomicMin(&chosen_part, hit);
        if (last >= 0) atomicMax(&behind, last);
        __syncthreads();
        if (hit >= 0 && hit == chosen_part) before_part = before;
        if (threadIdx.x == 0) {
            goal_ = goal;
            if (chosen_part == 0x7fffffff) chosen_part = behind, goal_ = __builtin_huge_val(), before_part = 0;         // v rounds to all of the sum
        }
        __syncthreads();
        return all;
    };
    const double v = largest || !(a.v[b] > 0) ? 0 : (double)a.v[b];
    const double sum = choose(a.pieces * kMine, [&](int i) {
        return __hip_atomic_load(weight + i / kMine * kParts + i % kMine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }, v, 0);
    int64_t of = chosen_part / kMine;
    int in = chosen_part % kMine;
    if (!(sum > 0)) {
        // p <= q throughout: p itself is drawn from, first a piece of it, then a part of that
        left.rejected = false;
        __syncthreads();
        // pieces whose powers may all be taken as 0, being below 2^-996 of the largest, are left out
        choose(a.pieces, [&](int i) {
            const double w = onto(a.target[row * a.pieces + i], left.p.m, c) / left.p.s;
            return w > 0x1p-900 ? w : 0;
        }, v, 0);
        of = chosen_part < 0 ? piece : chosen_part;
        const double goal = goal_ - before_part;
        piece_parts(of, [&](int i, double s) { sums[i] = s; });
        __syncthreads();
        choose(kMine, [&](int i) { return sums[i]; }, -1, goal);
        in = chosen_part;
    }
    if (in < 0) {                                // nothing has a weight: no place is read
        if (threadIdx.x == 0) a.next[b] = -1;
        return;
    }
    if (of != piece) lay_out(of);
    if (wave != 0) return;
    // the part's vectors, one a lane
    const int vec = (in / kWavesRow) * kRow + (in % kWavesRow) * kWave + lane;
    double w[PER], s = 0;
    left.weights(of * kPiece + vec, vec, left.logits(of * kPiece + vec), w);
#pragma unroll
    for (int e = 0; e < PER; ++e) s += w[e];
    double run = s;
#pragma unroll
    for (int step = 1; step < kWave; step *= 2) {
        const double y = __shfl_up(run, step);
        if (lane >= step) run += y;
    }
    int place = -1, last = -1;
    double x = before_part + (run - s);
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        x += w[e];
        if (w[e] > 0) {
            last = e;
            if (place < 0 && x > goal_) place = e;
        }
    }
    const uint64_t over_it = __ballot(place >= 0), some = __ballot(last >= 0);
    const int who = over_it ? __builtin_ctzll(over_it) : some ? 63 - __builtin_clzll(some) : 0;
    const int e = __builtin_amdgcn_readlane(over_it ? place : last, who);
    if (lane == 0) a.next[b] = e < 0 ? -1 : (int32_t)((of * kPiece + vec + who) * PER + e);
}

template <int TYPE, int DRAFT, int MODE, int VEC> hipError_t launch(const VerifyArgs &a, hipStream_t st) {
    const hipError_t e = in_launches(a.N * (a.pieces + a.draft_pieces), kRow, [&](uint32_t from, unsigned n) {
        hipLaunchKernelGGL((k_verify_sums<TYPE, DRAFT, VEC>), dim3(n), dim3(kRow), 0, st, a, from);
    });
    if (e != hipSuccess) return e;
    return in_launches(a.B * a.pieces, kRow, [&](uint32_t from, unsigned n) {
        hipLaunchKernelGGL((k_verify_draw<TYPE, DRAFT, MODE, VEC>), dim3(n), dim3(kRow), 0, st, a, from);
    });
}
template <int TYPE, int VEC> hipError_t launch(const VerifyArgs &a, int draft_type, hipStream_t st) {
    if (a.draft) {
        if (draft_type == COMET_F32) return launch<TYPE, COMET_F32, kDense, VEC>(a, st);
        if (draft_type == COMET_BF16) return launch<TYPE, COMET_BF16, kDense, VEC>(a, st);
        return launch<TYPE, COMET_F16, kDense, VEC>(a, st);
    }
    return a.K > 0 ? launch<TYPE, TYPE, kEntries, VEC>(a, st) : launch<TYPE, TYPE, kPoint, VEC>(a, st);
}
template <int TYPE> hipError_t launch(const VerifyArgs &a, int draft_type, hipStream_t st) {
    return vectors_of(a.N, a.V) == 2 ? launch<TYPE, 2>(a, draft_type, st) : launch<TYPE, 8>(a, draft_type, st);
}

struct Layout { int64_t target, drafted, weight, arrived, bytes; };
Layout layout(int type, int64_t N, int64_t V, int64_t B, int draft_type, bool with_draft) {
    Layout l{};
    l.target = 0;
    l.drafted = l.target + N * pieces_of(type, N, V) * (int64_t)sizeof(Sum);
    l.weight = l.drafted + (with_draft ? N * pieces_of(draft_type, N, V) * (int64_t)sizeof(Sum) : 0);
    l.arrived = l.weight + B * pieces_of(type, N, V) * kParts * 8;
    l.bytes = l.arrived + B * 4;
    return l;
}

}  // namespace

int64_t draft_verify_work(int type, int64_t N, int64_t V, int64_t B, bool with_draft) { return layout(type, N, V, B, COMET_F32, with_draft).bytes; }

hipError_t draft_verify(const void *Z, int type, int64_t N, int64_t V, int64_t ldz, int64_t B, const int32_t *pos, const int32_t *token, const float *u,
                        const float *v, const void *draft, int draft_type, int64_t ldd, const int32_t *crd, const float *vals, int64_t K, double scale,
                        const float *scales, int32_t *accepted, int32_t *next, int32_t *length, void *work, hipStream_t st) {
    const Layout l = layout(type, N, V, B, draft_type, draft != nullptr);
    char *w = (char *)work;
    const VerifyArgs a{Z, N, V, ldz, B, pos, token, u, v, draft, ldd, crd, vals, K, scale, scales, accepted, next, length, (Sum *)(w + l.target),
                       (Sum *)(w + l.drafted), (double *)(w + l.weight), (int32_t *)(w + l.arrived), (int32_t)pieces_of(type, N, V),
                       draft ? (int32_t)pieces_of(draft_type, N, V) : 0};
    if (type == COMET_F32) return launch<COMET_F32>(a, draft_type, st);
    if (type == COMET_BF16) return launch<COMET_BF16>(a, draft_type, st);
    return launch<COMET_F16>(a, draft_type, st);
}

}  // namespace comet
