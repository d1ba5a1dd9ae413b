// C ABI of the operators on dense rows: argument checks, then the launchers of rows_kernels.hpp.
#include <cmath>

#include "rows_kernels.hpp"

namespace {

constexpr int64_t kLim = int64_t(1) << 31;
constexpr int64_t kRows = int64_t(1) << 23;      // a grid holds a workgroup or more for each row

constexpr int64_t kTop = int64_t(1) << 29;       // V * K: one workgroup joins the lists of a row's pieces, 2^29 / 65536 + 1024 keys at most, or 16 * 1024

int element_size(int type) { return type == COMET_F32 ? 4 : 2; }
bool known(comet_type_t type) { return type == COMET_F32 || type == COMET_BF16 || type == COMET_F16; }
bool aligned(const void *p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
bool good_scale(double s) { return std::isfinite(s) && s > 0 && std::isfinite((float)(s * 1.4426950408889634)) && (float)s > 0; }

comet_status done(hipError_t e) {
    if (e == hipSuccess) return COMET_OK;
    (void)hipGetLastError();
    return COMET_ERR_DEVICE;
}

comet_status check_rows(const void *Z, comet_type_t type, int64_t N, int64_t V, int64_t ldz) {
    if (!known(type) || N < 0 || V < 0) return COMET_ERR_INVALID_ARG;
    if (N > kRows || V >= kLim) return COMET_ERR_UNSUPPORTED;
    if (ldz < V) return COMET_ERR_SHAPE;
    if (ldz > (int64_t(1) << 40)) return COMET_ERR_UNSUPPORTED;
    if (N > 0 && V > 0 && !Z) return COMET_ERR_INVALID_ARG;
    if (!aligned(Z, element_size(type))) return COMET_ERR_INVALID_ARG;
    return COMET_OK;
}

comet_status check_work(const void *work, int64_t have, int64_t need) {
    if (need > 0 && (!work || have < need || !aligned(work, 16))) return COMET_ERR_INVALID_ARG;
    return COMET_OK;
}

comet_status check_distill(const comet::DistillArgs &a) {
    comet_status s = check_rows(a.Z, (comet_type_t)a.type, a.N, a.V, a.ldz);
    if (s != COMET_OK) return s;
    if (!good_scale(a.scale)) return COMET_ERR_INVALID_ARG;
    if (!a.pos && a.K < 0) return COMET_ERR_INVALID_ARG;
    if (!a.pos && a.K >= kLim) return COMET_ERR_UNSUPPORTED;
    if (!aligned(a.pos, 4) || !aligned(a.crd, 4) || !aligned(a.tvals, 4) || !aligned(a.tlse, 4) || !aligned(a.weight, 4))
        return COMET_ERR_INVALID_ARG;
    if (!a.pos && a.K > 0 && a.N > 0 && (!a.crd || !a.tvals)) return COMET_ERR_INVALID_ARG;
    return COMET_OK;
}

comet_status check_gradient(const comet::DistillArgs &a, const void *dZ, int64_t lddz) {
    if (lddz < a.V) return COMET_ERR_SHAPE;
    if (lddz > (int64_t(1) << 40)) return COMET_ERR_UNSUPPORTED;
    if (a.N > 0 && a.V > 0 && !dZ) return COMET_ERR_INVALID_ARG;
    if (!aligned(dZ, element_size(a.type)) || (dZ && dZ == a.Z && lddz != a.ldz)) return COMET_ERR_INVALID_ARG;
    return COMET_OK;
}

comet_status check_select(comet_type_t type, int64_t B, int64_t W, int64_t V, int64_t n) {
    if (!known(type) || B < 0 || W < 1 || V < 0 || n < 1) return COMET_ERR_INVALID_ARG;
    if (B > kRows || W > COMET_MAX_BEAMS || n > COMET_MAX_TOP || W * n > 8192 || V >= (1 << 24) || V * n > kTop || B * W > kRows) return COMET_ERR_UNSUPPORTED;
    return COMET_OK;
}

// Whether `count` pieces at `stride` bytes from each other, each of `extent` bytes, keep apart; the extent grows to all of them.
struct Nested {
    int64_t extent;
    bool add(int64_t count, int64_t stride) {
        if (count <= 1) return true;
        if (stride < extent || stride > (int64_t(1) << 44)) return false;
        extent += (count - 1) * stride;
        return true;
    }
};

}  // namespace

extern "C" {

comet_status comet_rows_topk_work(comet_type_t type, int64_t N, int64_t V, int64_t K, int64_t *bytes) {
    if (!bytes || !known(type) || N < 0 || V < 0 || K < 1) return COMET_ERR_INVALID_ARG;
    if (N > kRows || V >= kLim || K > COMET_MAX_TOP || V * K > kTop) return COMET_ERR_UNSUPPORTED;
    *bytes = comet::rows_topk_work(type, N, V, K);
    return COMET_OK;
}

comet_status comet_rows_topk(const void *Z, comet_type_t type, int64_t N, int64_t V, int64_t ldz, double scale, int64_t K, unsigned flags,
                             int32_t *crd, float *vals, float *lse, void *work, int64_t work_bytes, void *stream) {
    comet_status s = check_rows(Z, type, N, V, ldz);
    if (s != COMET_OK) return s;
    if (!good_scale(scale) || K < 1 || (flags & ~COMET_BY_COORDINATE)) return COMET_ERR_INVALID_ARG;
    if (K > COMET_MAX_TOP || V * K > kTop) return COMET_ERR_UNSUPPORTED;
    if (N == 0) return COMET_OK;
    if (!crd || !vals || !aligned(crd, 4) || !aligned(vals, 4) || !aligned(lse, 4)) return COMET_ERR_INVALID_ARG;
    s = check_work(work, work_bytes, comet::rows_topk_work(type, N, V, K));
    if (s != COMET_OK) return s;
    return done(comet::rows_topk(Z, type, N, V, ldz, scale, K, (flags & COMET_BY_COORDINATE) != 0, crd, vals, lse, work, (hipStream_t)stream));
}

comet_status comet_distill_work(comet_type_t type, int64_t N, int64_t V, int64_t *bytes) {
    if (!bytes || !known(type) || N < 0 || V < 0) return COMET_ERR_INVALID_ARG;
    if (N > kRows || V >= kLim) return COMET_ERR_UNSUPPORTED;
    *bytes = comet::distill_work(type, N, V);
    return COMET_OK;
}

comet_status comet_distill_forward(const void *Z, comet_type_t type, int64_t N, int64_t V, int64_t ldz, const int32_t *pos, int64_t K,
                                   const int32_t *crd, const float *tvals, const float *tlse, double scale, const float *weight,
                                   float *loss, double *stat, void *work, int64_t work_bytes, void *stream) {
    const comet::DistillArgs a{Z, type, N, V, ldz, pos, K, crd, tvals, tlse, scale, weight};
    comet_status s = check_distill(a);
    if (s != COMET_OK || N == 0) return s;
    if (!loss || !stat || !aligned(loss, 4) || !aligned(stat, 8)) return COMET_ERR_INVALID_ARG;
    s = check_work(work, work_bytes, comet::distill_work(type, N, V));
    if (s != COMET_OK) return s;
    return done(comet::distill_forward(a, loss, stat, work, (hipStream_t)stream));
}

comet_status comet_distill_backward(const void *Z, comet_type_t type, int64_t N, int64_t V, int64_t ldz, const int32_t *pos, int64_t K,
                                    const int32_t *crd, const float *tvals, const float *tlse, double scale, const float *weight,
                                    const double *stat, const float *dloss, void *dZ, int64_t lddz, void *stream) {
    const comet::DistillArgs a{Z, type, N, V, ldz, pos, K, crd, tvals, tlse, scale, weight};
    comet_status s = check_distill(a);
    if (s == COMET_OK) s = check_gradient(a, dZ, lddz);
    if (s != COMET_OK || N == 0 || V == 0) return s;
    if (!stat || !aligned(stat, 8) || !aligned(dloss, 4)) return COMET_ERR_INVALID_ARG;
    return done(comet::distill_backward(a, stat, dloss, dZ, lddz, (hipStream_t)stream));
}

comet_status comet_distill_step(const void *Z, comet_type_t type, int64_t N, int64_t V, int64_t ldz, const int32_t *pos, int64_t K,
                                const int32_t *crd, const float *tvals, const float *tlse, double scale, const float *weight, float *loss,
                                void *dZ, int64_t lddz, void *work, int64_t work_bytes, void *stream) {
    const comet::DistillArgs a{Z, type, N, V, ldz, pos, K, crd, tvals, tlse, scale, weight};
    comet_status s = check_distill(a);
    if (s == COMET_OK) s = check_gradient(a, dZ, lddz);
    if (s != COMET_OK || N == 0) return s;
    if (!loss || !aligned(loss, 4)) return COMET_ERR_INVALID_ARG;
    s = check_work(work, work_bytes, comet::distill_work(type, N, V));
    if (s != COMET_OK) return s;
    return done(comet::distill_step(a, loss, dZ, lddz, work, (hipStream_t)stream));
}

comet_status comet_beam_select_work(comet_type_t type, int64_t B, int64_t W, int64_t V, int64_t n, int64_t *bytes) {
    if (!bytes) return COMET_ERR_INVALID_ARG;
    const comet_status s = check_select(type, B, W, V, n);
    if (s == COMET_OK) *bytes = comet::beam_select_work(type, B, W, V, n);
    return s;
}

comet_status comet_beam_select(const void *Z, comet_type_t type, int64_t B, int64_t W, int64_t V, int64_t ldz, const float *score,
                               const uint8_t *finished, int32_t eos, int64_t n, float *out_score, int32_t *out_parent, int32_t *out_token,
                               void *work, int64_t work_bytes, void *stream) {
    comet_status s = check_select(type, B, W, V, n);
    if (s == COMET_OK) s = check_rows(Z, type, B * W, V, ldz);
    if (s != COMET_OK || B == 0) return s;
    if (!score || !out_score || !out_parent || !out_token) return COMET_ERR_INVALID_ARG;
    if (!aligned(score, 4) || !aligned(out_score, 4) || !aligned(out_parent, 4) || !aligned(out_token, 4)) return COMET_ERR_INVALID_ARG;
    if (finished && (eos < 0 || eos >= V)) return COMET_ERR_INVALID_ARG;
    s = check_work(work, work_bytes, comet::beam_select_work(type, B, W, V, n));
    if (s != COMET_OK) return s;
    return done(comet::beam_select(Z, type, B, W, V, ldz, score, finished, eos, n, out_score, out_parent, out_token, work, (hipStream_t)stream));
}

comet_status comet_beam_reorder(void *const *states, int64_t nstates, int64_t B, int64_t W, int64_t batch_stride, int64_t beam_stride,
                                int64_t outer, int64_t outer_stride, int64_t inner, const int32_t *parent, void *stream) {
    if (nstates < 0 || B < 0 || W < 1 || outer < 0 || inner < 0) return COMET_ERR_INVALID_ARG;
    if (W > COMET_MAX_BEAMS || B >= kLim || nstates >= kLim || inner > (int64_t(1) << 44) || outer > (int64_t(1) << 44)) return COMET_ERR_UNSUPPORTED;
    if (nstates == 0 || B == 0 || outer == 0 || inner == 0) return COMET_OK;
    if (!states || !parent || !aligned(parent, 4)) return COMET_ERR_INVALID_ARG;
    for (int64_t i = 0; i < nstates; ++i)
        if (!states[i]) return COMET_ERR_INVALID_ARG;
    // pieces nested in the order of their strides must not reach into each other
    int64_t count[3] = {B, W, outer}, stride[3] = {batch_stride, beam_stride, outer_stride};
    for (int i = 0; i < 3; ++i)
        for (int j = 0; j < 2 - i; ++j)
            if (stride[j] > stride[j + 1]) {
                const int64_t c = count[j], t = stride[j];
                count[j] = count[j + 1], stride[j] = stride[j + 1];
                count[j + 1] = c, stride[j + 1] = t;
            }
    Nested all{inner};
    for (int i = 0; i < 3; ++i) {
        if (count[i] > 1 && count[i] > (int64_t(1) << 47) / (stride[i] > 0 ? stride[i] : 1)) return COMET_ERR_INVALID_ARG;
        if (!all.add(count[i], stride[i])) return COMET_ERR_INVALID_ARG;
    }
    const comet::StateLayout l{B, W, batch_stride, beam_stride, outer, outer_stride, inner};
    return done(comet::beam_reorder(states, nstates, l, parent, (hipStream_t)stream));
}

}  // extern "C"
