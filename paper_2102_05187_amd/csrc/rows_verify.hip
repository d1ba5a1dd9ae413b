// Drafted tokens against the target's logits.
#include "rows_kernels.hpp"
#include "cache.hpp"

namespace comet {

namespace {

// How the draft's distribution is known: not at all (the token has all of it), by some of its logits, by all of them.
enum { kPoint = 0, kEntries = 1, kDense = 2 };

constexpr int kRow = 256;
constexpr int kVectors = 8;                   // 16-byte vectors of a thread: a piece of a row is 2048 vectors

int64_t pieces_of(int type, int64_t V) {
    const int64_t n = kRow * kVectors * (type == COMET_F32 ? 4 : 8);
    return V > n ? (V + n - 1) / n : 1;
}

// exp2 in 64 bits for arguments of at most 0, to about 2^-49: the nearest whole number taken off, a Taylor polynomial of exp(f ln 2) for |f| <= 1/2
// (the first term that is left out is 4e-18 of the sum at most, the roundings of its steps are more).
__device__ __forceinline__ double exp2_wide(double x) {
    if (!(x > -1000.0)) return x != x ? x : 0.0;
    const double n = __builtin_rint(x), f = (x - n) * 0.6931471805599453094;
    double r = 1.0 / 6227020800.0;
    r = __builtin_fma(r, f, 1.0 / 479001600.0);
    r = __builtin_fma(r, f, 1.0 / 39916800.0);
    r = __builtin_fma(r, f, 1.0 / 3628800.0);
    r = __builtin_fma(r, f, 1.0 / 362880.0);
    r = __builtin_fma(r, f, 1.0 / 40320.0);
    r = __builtin_fma(r, f, 1.0 / 5040.0);
    r = __builtin_fma(r, f, 1.0 / 720.0);
    r = __builtin_fma(r, f, 1.0 / 120.0);
    r = __builtin_fma(r, f, 1.0 / 24.0);
    r = __builtin_fma(r, f, 1.0 / 6.0);
    r = __builtin_fma(r, f, 0.5);
    r = __builtin_fma(r, f, 1.0);
    r = __builtin_fma(r, f, 1.0);
    return __builtin_amdgcn_ldexp(r, (int)n);
}

// The sum of exp2((z - m) c) over a part of a row, m its largest logit: of nothing, m is -inf; with a NaN or +inf in it, s is a NaN.
struct Sum {
    double s;
    double m;
    __device__ __forceinline__ bool good() const { return s > 0; }
};
__device__ __forceinline__ Sum join(Sum a, Sum b, double c) {
    Sum r;
    r.m = a.m > b.m ? a.m : b.m;
    r.s = (a.m == r.m ? a.s : a.s == 0 ? 0 : a.s * exp2_wide((a.m - r.m) * c)) + (b.m == r.m ? b.s : b.s == 0 ? 0 : b.s * exp2_wide((b.m - r.m) * c));
    return r;
}
__device__ __forceinline__ Sum wave_join(Sum a, double c) {
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const Sum b{__shfl_xor(a.s, d), __shfl_xor(a.m, d)};
        a = join(a, b, c);
    }
    return a;
}
// Of a whole row, from its pieces' sums; by a wavefront, the same in all lanes.
__device__ __forceinline__ Sum row_sum(const Sum *piece, int64_t pieces, double c) {
    Sum a{0, kNegInfD};
    for (int64_t i = threadIdx.x & (kWave - 1); i < pieces; i += kWave) a = join(a, piece[i], c);
    return wave_join(a, c);
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
    double *weight;                           // [B x pieces]: what is drawn from, piece by piece
    int32_t *arrived;                         // [B]
    int64_t pieces, draft_pieces;

    // scale log2 e of a request; NaN where it is no scale, +inf where the largest logit is taken
    __device__ __forceinline__ double of(int64_t b) const {
        const double s = scales ? (double)scales[b] : scale;
        return s > 0 ? s * 1.4426950408889634 : __builtin_nan("");
    }
};

// One piece of one row.
template <int TYPE>
__device__ void piece_sum(const void *base, int64_t row, int64_t ld, int64_t V, int64_t piece, double c, Sum *out) {
    using E = Elem<TYPE>;
    __shared__ float top[kRow / kWave];
    __shared__ double part[kRow / kWave];
    const Row<TYPE> r(base, row, ld, V);
    const int64_t v0 = piece * (kRow * kVectors);
    uint4 x[kVectors];
#pragma unroll
    for (int j = 0; j < kVectors; ++j) {
        const int64_t i = v0 + j * kRow + threadIdx.x;
        if (r.whole(i)) {
            x[j] = r.raw(i);
        } else {
            float f[E::kPer];
            r.load(i, f);
            x[j] = E::narrow(f);
        }
    }
    float m = kNegInf;
#pragma unroll
    for (int j = 0; j < kVectors; ++j) {
        float f[E::kPer];
        E::widen(x[j], f);
#pragma unroll
        for (int e = 0; e < E::kPer; ++e) m = fmaxf(m, f[e]);
    }
    m = wave_reduce(m, kNegInf, Larger());
    if ((threadIdx.x & (kWave - 1)) == 0) top[threadIdx.x / kWave] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kRow / kWave; ++w) m = fmaxf(m, top[w]);
    double s = 0;
    const double big = m == kNegInf ? 0 : m;                    // exp2 of -inf is 0
    const bool largest = c == __builtin_huge_val();
    for (int j = 0; j < kVectors; ++j) {
        float f[E::kPer];
        E::widen(x[j], f);
#pragma unroll
        for (int e = 0; e < E::kPer; ++e) s += largest ? (f[e] != f[e] ? f[e] : f[e] == m ? 1.0 : 0.0) : exp2_wide(((double)f[e] - big) * c);
    }
    s = wave_reduce(s, 0.0, Add());
    if ((threadIdx.x & (kWave - 1)) == 0) part[threadIdx.x / kWave] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kRow / kWave; ++w) s += part[w];
        *out = Sum{s, m};
    }
}

// Sums of all pieces of all rows that are judged by or drawn from.
template <int TYPE, int DRAFT>
__global__ void __launch_bounds__(kRow) k_verify_sums(VerifyArgs a) {
    __shared__ int count;
    const int64_t all = a.pieces + a.draft_pieces, row = blockIdx.x / all;
    int64_t piece = blockIdx.x - row * all;
    for (int64_t b = (int64_t)blockIdx.x * kRow + threadIdx.x; b < a.B; b += (int64_t)gridDim.x * kRow) a.arrived[b] = 0;
    const int64_t b = request_of<kRow>(a.pos, a.B, row, &count);
    if (b < 0) return;
    const double c = a.of(b);
    if (piece < a.pieces) {
        piece_sum<TYPE>(a.Z, row, a.ldz, a.V, piece, c, a.target + row * a.pieces + piece);
    } else if (row + 1 < a.pos[b + 1]) {
        piece -= a.pieces;
        piece_sum<DRAFT>(a.draft, row, a.ldd, a.V, piece, c, a.drafted + row * a.draft_pieces + piece);
    }
}

// What is drawn from at one row, where the target's and the draft's sums are known.
template <int TYPE, int DRAFT, int MODE> struct Left {
    Row<TYPE> z;
    Row<DRAFT> x;
    Sum p, q;
    double c, p_part, q_part;                 // 1 / p.s, and 1 / q.s or 0
    bool rejected, largest;                   // something of the draft is taken off; only the largest logit counts
    int64_t d;
    const uint16_t *at;                       // kEntries: 1 + the entry of a place of the piece, 0: none
    const double *chance;                     //           and the entries' probabilities
    // weights of vector i, `in` its number in the piece
    __device__ __forceinline__ void weights(int64_t i, int in, double *w) const {
        constexpr int PER = Elem<TYPE>::kPer;
        float f[PER], g[PER];
        z.load(i, f);
        if (MODE == kDense && rejected) {
            if constexpr (Elem<DRAFT>::kPer == PER) {
                x.load(i, g);
            } else if constexpr (Elem<DRAFT>::kPer < PER) {
                x.load(2 * i, g), x.load(2 * i + 1, g + Elem<DRAFT>::kPer);
            } else {
                float both[Elem<DRAFT>::kPer];
                x.load(i / 2, both);
#pragma unroll
                for (int e = 0; e < PER; ++e) g[e] = both[(i & 1) * PER + e];
            }
        }
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            if (largest) { w[e] = (double)f[e] == p.m ? 1 : 0; continue; }
            w[e] = exp2_wide(((double)f[e] - p.m) * c) * p_part;
            if (!rejected) continue;
            double off = 0;
            if (MODE == kPoint) off = z.first(i) + e == d ? 1 : 0;
            if (MODE == kDense) off = q_part > 0 ? exp2_wide(((double)g[e] - q.m) * c) * q_part : 0;
            if (MODE == kEntries) {
                const int k = at[in * PER + e];
                off = k ? chance[k - 1] : 0;
            }
            w[e] = w[e] > off ? w[e] - off : 0;
        }
    }
};

// One piece of the row that a request's next token is drawn from.  Each workgroup finds for itself how far the drafted tokens are taken; the one that
// is done last has all pieces' weights, and draws.
template <int TYPE, int DRAFT, int MODE>
__global__ void __launch_bounds__(kRow) k_verify_draw(VerifyArgs a) {
    constexpr int PER = Elem<TYPE>::kPer, kPiece = kRow * kVectors;
    __shared__ int first, hit, final_one;
    __shared__ double part[kRow / kWave], chance[MODE == kEntries ? COMET_MAX_TOP : 1];
    __shared__ uint16_t at[MODE == kEntries ? kPiece * PER : 1];
    const int64_t b = blockIdx.x / a.pieces, piece = blockIdx.x - b * a.pieces;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t r0 = a.pos[b], n = (a.pos[b + 1] < a.N ? a.pos[b + 1] : a.N) - r0;
    if (n <= 0) {
        if (piece == 0 && threadIdx.x == 0) a.accepted[b] = 0, a.next[b] = -1;
        return;
    }
    const double c = a.of(b);
    const bool largest = c == __builtin_huge_val();
    // the sum of a row's entries; by a wavefront
    const auto entries = [&](int64_t row) {
        Sum s{0, kNegInfD};
        for (int64_t k = lane; k < a.K; k += kWave) {
            const int64_t col = a.crd[row * a.K + k];
            if (col < 0 || col >= a.V) continue;
            const double t = a.vals[row * a.K + k];
            s = join(s, Sum{t == kNegInfD ? 0.0 : t - t == 0 ? 1.0 : __builtin_nan(""), t == t ? t : kNegInfD}, c);
        }
        return wave_join(s, c);
    };
    if (threadIdx.x == 0) first = (int)(n - 1);
    __syncthreads();
    for (int64_t i = wave; i < n - 1; i += kRow / kWave) {
        if (i > first) break;
        const int64_t row = r0 + i, d = a.token[row + 1];
        bool take = false;
        if (d >= 0 && d < a.V) {
            const Sum p = row_sum(a.target + row * a.pieces, a.pieces, c);
            const double z = Elem<TYPE>::one(((const typename Elem<TYPE>::T *)a.Z)[row * a.ldz + d]);
            if (largest) {
                take = p.m == z && p.m > kNegInfD && p.m < -kNegInfD && p.s == p.s;
            } else if (p.good()) {
                double q = 1;
                if (MODE == kDense) {
                    const Sum s = row_sum(a.drafted + row * a.draft_pieces, a.draft_pieces, c);
                    q = s.good() ? exp2_wide(((double)Elem<DRAFT>::one(((const typename Elem<DRAFT>::T *)a.draft)[row * a.ldd + d]) - s.m) * c) / s.s : 0;
                }
                if (MODE == kEntries) {
                    const Sum s = entries(row);
                    q = 0;
                    if (s.good())
                        for (int64_t k = lane; k < a.K; k += kWave)
                            if (a.crd[row * a.K + k] == d) q = exp2_wide(((double)a.vals[row * a.K + k] - s.m) * c) / s.s;
                    q = wave_reduce(q, 0.0, Add());
                }
                take = (double)a.u[row] * q < exp2_wide((z - p.m) * c) / p.s;
            }
        }
        if (!take && lane == 0) atomicMin(&first, (int)i);
    }
    __syncthreads();
    const int64_t took = first, row = r0 + took;
    if (piece == 0 && threadIdx.x == 0) {
        a.accepted[b] = (int32_t)took;
        if (a.length) a.length[b] -= (int32_t)(n - 1 - took);
    }
    Left<TYPE, DRAFT, MODE> left{Row<TYPE>(a.Z, row, a.ldz, a.V), Row<DRAFT>(a.draft, MODE == kDense ? row : 0, a.ldd, a.V), row_sum(a.target + row * a.pieces, a.pieces, c),
                                 Sum{0, 0}, c, 0, 0, took < n - 1 && !largest, largest, took < n - 1 ? a.token[row + 1] : -1, at, chance};
    const bool any = largest ? left.p.m > kNegInfD && left.p.m < -kNegInfD && left.p.s == left.p.s : left.p.good();
    if (!any) {
        if (piece == 0 && threadIdx.x == 0) a.next[b] = -1;
        return;
    }
    if (left.rejected) {
        if (MODE == kDense) left.q = row_sum(a.drafted + row * a.draft_pieces, a.draft_pieces, c);
        if (MODE == kEntries) left.q = entries(row);
        left.q_part = left.q.good() ? 1 / left.q.s : 0;
    }
    left.p_part = 1 / left.p.s;
    // the entries that lie in a piece, by place
    const auto lay_out = [&](int64_t of) {
        if (MODE != kEntries || !left.rejected) return;
        __syncthreads();
        for (int i = threadIdx.x; i < kPiece * PER; i += kRow) at[i] = 0;
        __syncthreads();
        if (left.q_part > 0)
            for (int64_t k = threadIdx.x; k < a.K; k += kRow) {
                const int64_t col = a.crd[row * a.K + k], to = col - of * kPiece * PER;
                chance[k] = exp2_wide(((double)a.vals[row * a.K + k] - left.q.m) * c) * left.q_part;
                if (col >= 0 && col < a.V && to >= 0 && to < kPiece * PER) at[to] = (uint16_t)(k + 1);
            }
        __syncthreads();
    };
    const auto total = [&](double s) {
        s = wave_reduce(s, 0.0, Add());
        if (lane == 0) part[wave] = s;
        __syncthreads();
        s = 0;
        for (int w = 0; w < kRow / kWave; ++w) s += part[w];
        __syncthreads();
        return s;
    };
    const auto piece_weight = [&](int64_t of) {
        double s = 0;
        for (int j = 0; j < kVectors; ++j) {
            double w[PER];
            left.weights(of * kPiece + j * kRow + threadIdx.x, j * kRow + threadIdx.x, w);
#pragma unroll
            for (int e = 0; e < PER; ++e) s += w[e];
        }
        return total(s);
    };
    lay_out(piece);
    const double mine = piece_weight(piece);
    double *weight = a.weight + b * a.pieces;
    if (a.pieces > 1) {
        if (threadIdx.x == 0) {
            __hip_atomic_store(weight + piece, mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            final_one = __hip_atomic_fetch_add(a.arrived + b, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (int)a.pieces - 1;
        }
        __syncthreads();
        if (!final_one) return;
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    }
    const auto of_piece = [&](int64_t i) { return a.pieces > 1 ? __hip_atomic_load(weight + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : mine; };
    double sum = 0;
    for (int64_t i = 0; i < a.pieces; ++i) sum += of_piece(i);
    const bool nothing = !(sum > 0);                             // p <= q throughout: p itself, of which the pieces are known
    if (nothing) left.rejected = false;
    const auto now = [&](int64_t i) {
        if (!nothing) return of_piece(i);
        const Sum s = a.target[row * a.pieces + i];
        return s.s > 0 ? s.s * exp2_wide((s.m - left.p.m) * c) / left.p.s : 0.0;
    };
    if (nothing) {
        sum = 0;
        for (int64_t i = 0; i < a.pieces; ++i) sum += now(i);
    }
    const double v = largest || !(a.v[b] > 0) ? 0 : (double)a.v[b];
    double goal = v * sum, upto = 0;
    int64_t chosen = -1, last = 0;
    for (int64_t i = 0; i < a.pieces && chosen < 0; ++i) {
        const double w = now(i);
        if (w > 0) last = i;
        if (upto + w > goal) chosen = i;
        else upto += w;
    }
    if (chosen < 0) chosen = last, goal = -kNegInfD;              // v rounds to all of the sum: the last place that has a weight
    if (chosen != piece && left.rejected) lay_out(chosen);
    if (threadIdx.x == 0) hit = -1;
    __syncthreads();
    int behind = -1;                                             // the last place with a weight so far
    for (int j = 0; j < kVectors; ++j) {
        const int in = j * kRow + threadIdx.x;
        double w[PER], s = 0;
        left.weights(chosen * kPiece + in, in, w);
        int at_last = -1;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            s += w[e];
            if (w[e] > 0) at_last = in * PER + e;
        }
        double run = s;
#pragma unroll
        for (int step = 1; step < kWave; step *= 2) {
            const double y = __shfl_up(run, step);
            if (lane >= step) run += y;
        }
        if (lane == kWave - 1) part[wave] = run;
        __syncthreads();
        double before = upto;
        for (int w2 = 0; w2 < wave; ++w2) before += part[w2];
        const double end = before + run;
        if (at_last >= 0) behind = at_last;
        const uint64_t over = __ballot(end > goal && s > 0);
        if (over && lane == __builtin_ctzll(over)) {
            double x = end - s;
            int place = at_last;
            for (int e = PER - 1; e >= 0; --e) {
                double y = x;
                for (int g = 0; g <= e; ++g) y += w[g];
                if (w[e] > 0 && y > goal) place = in * PER + e;
            }
            atomicMin((unsigned *)&hit, (unsigned)place);
        }
        for (int w2 = 0; w2 < kRow / kWave; ++w2) upto += part[w2];
        __syncthreads();
        if (hit >= 0) break;
        __syncthreads();
    }
    if (hit < 0) {
        if (threadIdx.x == 0) first = -1;
        __syncthreads();
        if (behind >= 0) atomicMax(&first, behind);
        __syncthreads();
        if (threadIdx.x == 0) hit = first;
        __syncthreads();
    }
    if (threadIdx.x == 0) a.next[b] = hit < 0 ? -1 : (int32_t)(chosen * kPiece * PER + hit);
}

template <int TYPE, int DRAFT, int MODE> hipError_t launch(const VerifyArgs &a, hipStream_t st) {
    if (a.N > 0) {
        hipLaunchKernelGGL((k_verify_sums<TYPE, DRAFT>), dim3((unsigned)(a.N * (a.pieces + a.draft_pieces))), dim3(kRow), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((k_verify_draw<TYPE, DRAFT, MODE>), dim3((unsigned)(a.B * a.pieces)), dim3(kRow), 0, st, a);
    return hipGetLastError();
}
template <int TYPE> hipError_t launch(const VerifyArgs &a, int draft_type, hipStream_t st) {
    if (a.draft) {
        if (draft_type == COMET_F32) return launch<TYPE, COMET_F32, kDense>(a, st);
        if (draft_type == COMET_BF16) return launch<TYPE, COMET_BF16, kDense>(a, st);
        return launch<TYPE, COMET_F16, kDense>(a, st);
    }
    return a.K > 0 ? launch<TYPE, TYPE, kEntries>(a, st) : launch<TYPE, TYPE, kPoint>(a, st);
}

struct Layout { int64_t target, drafted, weight, arrived, bytes; };
Layout layout(int type, int64_t N, int64_t V, int64_t B, int draft_type, bool with_draft) {
    Layout l{};
    l.target = 0;
    l.drafted = l.target + N * pieces_of(type, V) * (int64_t)sizeof(Sum);
    l.weight = l.drafted + (with_draft ? N * pieces_of(draft_type, V) * (int64_t)sizeof(Sum) : 0);
    l.arrived = l.weight + B * pieces_of(type, V) * 8;
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
                       (Sum *)(w + l.drafted), (double *)(w + l.weight), (int32_t *)(w + l.arrived), pieces_of(type, V), draft ? pieces_of(draft_type, V) : 0};
    if (type == COMET_F32) return launch<COMET_F32>(a, draft_type, st);
    if (type == COMET_BF16) return launch<COMET_BF16>(a, draft_type, st);
    return launch<COMET_F16>(a, draft_type, st);
}

}  // namespace comet
