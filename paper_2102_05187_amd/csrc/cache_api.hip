// C ABI of the operators over a cache in blocks: argument checks, then the launchers of cache.hpp and rows_kernels.hpp.
#include <cmath>
#include <initializer_list>

#include "cache.hpp"
#include "rows_kernels.hpp"

namespace {

constexpr int64_t kLim = int64_t(1) << 31, kRows = int64_t(1) << 23, kStride = int64_t(1) << 40;

bool known(int type) { return type == COMET_F32 || type == COMET_BF16 || type == COMET_F16; }
int element_size(int type) { return type == COMET_F32 ? 4 : 2; }
bool aligned(const void *p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

comet_status done(hipError_t e) {
    if (e == hipSuccess) return COMET_OK;
    (void)hipGetLastError();
    return COMET_ERR_DEVICE;
}

comet_status check_strides(const int64_t *stride, int n, int type) {
    if (!stride) return COMET_ERR_INVALID_ARG;
    for (int i = 0; i < n; ++i) {
        if (stride[i] < 0 || stride[i] % (16 / element_size(type)) != 0) return COMET_ERR_INVALID_ARG;
        if (stride[i] > kStride) return COMET_ERR_UNSUPPORTED;
    }
    return COMET_OK;
}

// Sizes, strides and pointers; which of the arrays the call needs.
comet_status check_cache(const comet_cache *c, bool data, bool mean) {
    if (!c || !known(c->type) || c->blocks < 0 || c->block < 1 || c->heads < 1 || c->size < 1) return COMET_ERR_INVALID_ARG;
    if (c->blocks >= kLim || c->block > COMET_MAX_BLOCK || c->block % 16 || c->heads > 65536 || c->size > 256 || c->size % 8) return COMET_ERR_UNSUPPORTED;
    comet_status s = COMET_OK;
    if (data) {
        s = check_strides(c->key_stride, 3, c->type);
        if (s == COMET_OK) s = check_strides(c->value_stride, 3, c->type);
        if (s != COMET_OK) return s;
        if (c->blocks > 0 && (!c->keys || !c->values)) return COMET_ERR_INVALID_ARG;
        if (!aligned(c->keys, 16) || !aligned(c->values, 16)) return COMET_ERR_INVALID_ARG;
        // a place's distance from its block's first is computed in 32 bits
        for (const int64_t line : {c->key_stride[1], c->value_stride[1]})
            if (line * element_size(c->type) * c->block >= kLim - 1024) return COMET_ERR_UNSUPPORTED;
    }
    if (mean || c->mean) {
        s = check_strides(c->mean_stride, 2, c->type);
        if (s != COMET_OK) return s;
        if ((mean && c->blocks > 0 && !c->mean) || !aligned(c->mean, 16)) return COMET_ERR_INVALID_ARG;
    }
    return COMET_OK;
}

// Whether what is written lies apart: neighbours in each dimension of more than one element at least.
bool apart(const int64_t *stride, std::initializer_list<int64_t> sizes, int64_t length) {
    for (const int64_t n : sizes) {
        if (n > 1 && *stride < length) return false;
        ++stride;
    }
    return true;
}

comet_status check_sizes(const comet_cache *c, int64_t N, int64_t Q, int64_t B, int64_t M, int64_t K, int64_t most) {
    if (N < 0 || Q < 1 || B < 0 || M < 0 || K < 1) return COMET_ERR_INVALID_ARG;
    if (Q % c->heads) return COMET_ERR_SHAPE;
    if (N > kRows || Q > 65536 || N * Q >= kLim || B > kRows || M > most || K > COMET_MAX_CHOSEN || N * c->heads * K >= int64_t(1) << 40) return COMET_ERR_UNSUPPORTED;
    return COMET_OK;
}

comet_status check_queries(const comet_cache *c, const comet::Queries &q) {
    if (q.ldt < q.M) return COMET_ERR_SHAPE;
    if (q.ldt > kStride) return COMET_ERR_UNSUPPORTED;
    if (!aligned(q.q, 16) || !aligned(q.pos, 4) || !aligned(q.length, 4) || !aligned(q.table, 4)) return COMET_ERR_INVALID_ARG;
    if (q.N > 0 && (!q.q || !q.pos || (q.B > 0 && !q.length) || (q.B > 0 && q.M > 0 && !q.table))) return COMET_ERR_INVALID_ARG;
    return COMET_OK;
}

comet_status check_work(const void *work, int64_t have, int64_t need) {
    if (need > 0 && (!work || have < need || !aligned(work, 16))) return COMET_ERR_INVALID_ARG;
    return COMET_OK;
}

comet_status check_map(int64_t B, int64_t M, int64_t N) {
    if (B < 0 || M < 0 || N < 0) return COMET_ERR_INVALID_ARG;
    if (B > (int64_t(1) << 20) || M >= kLim || B * M >= (int64_t(1) << 40) || N >= kLim) return COMET_ERR_UNSUPPORTED;
    return COMET_OK;
}

comet_status check_verify(int type, int64_t N, int64_t V, int64_t B, int64_t K) {
    if (!known(type) || N < 0 || V < 0 || B < 0 || K < 0) return COMET_ERR_INVALID_ARG;
    if (N > kRows || V >= kLim || B > kRows || K > COMET_MAX_TOP) return COMET_ERR_UNSUPPORTED;
    // a workgroup for each piece of a row, of 2048 vectors of 4 elements or more, of the target and of the draft
    if ((N > B ? N : B) * 2 * (V / 8192 + 1) >= kLim) return COMET_ERR_UNSUPPORTED;
    return COMET_OK;
}

}  // namespace

extern "C" {

comet_status comet_cache_map_work(int64_t B, int64_t M, int64_t N, int64_t *bytes) {
    if (!bytes) return COMET_ERR_INVALID_ARG;
    const comet_status s = check_map(B, M, N);
    if (s == COMET_OK) *bytes = comet::cache_map_work(B, M, N);
    return s;
}

comet_status comet_cache_map(int64_t B, int64_t M, int64_t block, const int32_t *add, const uint8_t *ended, int32_t *length, int32_t *held, int32_t *table,
                             int64_t ldt, int32_t *spare, int64_t S, int32_t *count, int64_t N, int32_t *pos, int64_t *slot, int32_t *place, void *work,
                             int64_t work_bytes, void *stream) {
    comet_status s = check_map(B, M, N);
    if (s != COMET_OK) return s;
    if (block < 1 || S < 0) return COMET_ERR_INVALID_ARG;
    if (block > COMET_MAX_BLOCK || M * block >= kLim || S >= kLim || ldt > kStride) return COMET_ERR_UNSUPPORTED;
    if (ldt < M) return COMET_ERR_SHAPE;
    if (!pos || !count || (B > 0 && (!add || !length || !held)) || (B > 0 && M > 0 && !table) || (S > 0 && !spare) || (N > 0 && (!slot || !place)))
        return COMET_ERR_INVALID_ARG;
    if (!aligned(add, 4) || !aligned(length, 4) || !aligned(held, 4) || !aligned(table, 4) || !aligned(spare, 4) || !aligned(count, 4) || !aligned(pos, 4) ||
        !aligned(slot, 8) || !aligned(place, 4))
        return COMET_ERR_INVALID_ARG;
    s = check_work(work, work_bytes, comet::cache_map_work(B, M, N));
    if (s != COMET_OK) return s;
    return done(comet::cache_map({B, M, block, add, ended, length, held, table, ldt, spare, S, count, N, pos, slot, place}, work, (hipStream_t)stream));
}

comet_status comet_cache_write(const comet_cache *cache, int64_t N, const void *k, const int64_t k_stride[2], const void *v, const int64_t v_stride[2],
                               const int64_t *slot, void *stream) {
    comet_status s = check_cache(cache, true, false);
    if (s == COMET_OK) s = check_strides(k_stride, 2, cache->type);
    if (s == COMET_OK) s = check_strides(v_stride, 2, cache->type);
    if (s != COMET_OK) return s;
    if (N < 0) return COMET_ERR_INVALID_ARG;
    if (!apart(cache->key_stride, {cache->blocks, cache->block, cache->heads}, cache->size) ||
        !apart(cache->value_stride, {cache->blocks, cache->block, cache->heads}, cache->size) ||
        (cache->mean && !apart(cache->mean_stride, {cache->blocks, cache->heads}, cache->size)))
        return COMET_ERR_INVALID_ARG;
    if (N >= kLim) return COMET_ERR_UNSUPPORTED;
    if (N == 0) return COMET_OK;
    if (!k || !v || !slot || !aligned(k, 16) || !aligned(v, 16) || !aligned(slot, 8)) return COMET_ERR_INVALID_ARG;
    return done(comet::cache_write(*cache, N, k, k_stride, v, v_stride, slot, (hipStream_t)stream));
}

comet_status comet_block_select_work(const comet_cache *cache, int64_t N, int64_t Q, int64_t B, int64_t M, int64_t K, int64_t *bytes) {
    if (!bytes) return COMET_ERR_INVALID_ARG;
    comet_status s = check_cache(cache, false, false);
    if (s == COMET_OK) s = check_sizes(cache, N, Q, B, M, K, COMET_MAX_CANDIDATES);
    if (s == COMET_OK) *bytes = comet::block_select_work(*cache, N, Q, B, M, K);
    return s;
}

comet_status comet_block_select(const comet_cache *cache, int64_t N, int64_t Q, const void *q, const int64_t q_stride[2], int64_t B, const int32_t *pos,
                                const int32_t *length, const int32_t *table, int64_t M, int64_t ldt, int64_t K, int64_t first, int64_t last, int32_t *sel,
                                void *work, int64_t work_bytes, void *stream) {
    comet_status s = check_cache(cache, false, true);
    if (s == COMET_OK) s = check_sizes(cache, N, Q, B, M, K, COMET_MAX_CANDIDATES);
    if (s == COMET_OK) s = check_strides(q_stride, 2, cache->type);
    if (s != COMET_OK) return s;
    if (first < 0 || last < 1 || first > K || last > K || first + last > K) return COMET_ERR_INVALID_ARG;
    const comet::Queries queries{q, N, Q, q_stride[0], q_stride[1], B, pos, length, table, M, ldt};
    s = check_queries(cache, queries);
    if (s != COMET_OK) return s;
    if (N == 0 || B == 0) return COMET_OK;
    if (!sel || !aligned(sel, 4)) return COMET_ERR_INVALID_ARG;
    s = check_work(work, work_bytes, comet::block_select_work(*cache, N, Q, B, M, K));
    if (s != COMET_OK) return s;
    return done(comet::block_select(*cache, queries, K, first, last, sel, work, (hipStream_t)stream));
}

comet_status comet_block_attend_work(const comet_cache *cache, int64_t N, int64_t Q, int64_t B, int64_t M, int64_t K, int64_t *bytes) {
    if (!bytes) return COMET_ERR_INVALID_ARG;
    comet_status s = check_cache(cache, false, false);
    if (s == COMET_OK) s = check_sizes(cache, N, Q, B, M, K, COMET_MAX_TABLE);
    if (s == COMET_OK) *bytes = comet::block_attend_work(*cache, N, Q, B, M, K);
    return s;
}

comet_status comet_block_attend(const comet_cache *cache, int64_t N, int64_t Q, const void *q, const int64_t q_stride[2], int64_t B, const int32_t *pos,
                                const int32_t *length, const int32_t *table, int64_t M, int64_t ldt, const int32_t *sel, int64_t K, double scale, void *out,
                                float *lse, void *work, int64_t work_bytes, void *stream) {
    comet_status s = check_cache(cache, true, false);
    if (s == COMET_OK) s = check_sizes(cache, N, Q, B, M, K, COMET_MAX_TABLE);
    if (s == COMET_OK) s = check_strides(q_stride, 2, cache->type);
    if (s != COMET_OK) return s;
    if (!std::isfinite(scale) || !(scale > 0) || !std::isfinite((float)(scale * 1.4426950408889634)) || !((float)scale > 0)) return COMET_ERR_INVALID_ARG;
    const comet::Queries queries{q, N, Q, q_stride[0], q_stride[1], B, pos, length, table, M, ldt};
    s = check_queries(cache, queries);
    if (s != COMET_OK) return s;
    if (N == 0 || B == 0) return COMET_OK;
    if (!sel || !out || !aligned(sel, 4) || !aligned(out, 16) || !aligned(lse, 4)) return COMET_ERR_INVALID_ARG;
    s = check_work(work, work_bytes, comet::block_attend_work(*cache, N, Q, B, M, K));
    if (s != COMET_OK) return s;
    return done(comet::block_attend(*cache, queries, sel, K, scale, out, lse, work, (hipStream_t)stream));
}

comet_status comet_draft_verify_work(comet_type_t type, int64_t N, int64_t V, int64_t B, int64_t K, int with_draft, int64_t *bytes) {
    if (!bytes) return COMET_ERR_INVALID_ARG;
    const comet_status s = check_verify(type, N, V, B, K);
    if (s == COMET_OK) *bytes = comet::draft_verify_work(type, N, V, B, with_draft != 0);
    return s;
}

comet_status comet_draft_verify(const void *Z, comet_type_t type, int64_t N, int64_t V, int64_t ldz, int64_t B, const int32_t *pos, const int32_t *token,
                                const float *u, const float *v, const void *draft, comet_type_t draft_type, int64_t ldd, const int32_t *crd, const float *vals,
                                int64_t K, double scale, const float *scales, int32_t *accepted, int32_t *next, int32_t *length, void *work, int64_t work_bytes,
                                void *stream) {
    comet_status s = check_verify(type, N, V, B, K);
    if (s != COMET_OK) return s;
    if (draft && (!known(draft_type) || K > 0)) return COMET_ERR_INVALID_ARG;
    if (ldz < V || (draft && ldd < V)) return COMET_ERR_SHAPE;
    if (ldz > kStride || (draft && ldd > kStride)) return COMET_ERR_UNSUPPORTED;
    if (!scales && !(scale > 0)) return COMET_ERR_INVALID_ARG;
    if (B == 0) return COMET_OK;
    if (!pos || !accepted || !next || !v || (N > 0 && (!token || !u || (V > 0 && !Z) || (K > 0 && (!crd || !vals))))) return COMET_ERR_INVALID_ARG;
    if (!aligned(Z, element_size(type)) || (draft && !aligned(draft, element_size(draft_type))) || !aligned(pos, 4) || !aligned(token, 4) || !aligned(u, 4) ||
        !aligned(v, 4) || !aligned(crd, 4) || !aligned(vals, 4) || !aligned(scales, 4) || !aligned(accepted, 4) || !aligned(next, 4) || !aligned(length, 4))
        return COMET_ERR_INVALID_ARG;
    s = check_work(work, work_bytes, comet::draft_verify_work(type, N, V, B, draft != nullptr));
    if (s != COMET_OK) return s;
    return done(comet::draft_verify(Z, type, N, V, ldz, B, pos, token, u, v, draft, draft_type, ldd, crd, vals, K, scale, scales, accepted, next, length, work,
                                    (hipStream_t)stream));
}

}  // extern "C"
