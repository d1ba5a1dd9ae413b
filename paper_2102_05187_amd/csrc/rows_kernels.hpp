// Launchers of the operators on dense rows (rows_topk.hip, rows_distill.hip, rows_beam.hip, rows_verify.hip).  Arguments are checked by the
// entry points (rows_api.hip); every launcher only enqueues work on `st`.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

#include "../../include/comet.h"

namespace comet {

int64_t rows_topk_work(int type, int64_t N, int64_t V, int64_t K);
hipError_t rows_topk(const void *Z, int type, int64_t N, int64_t V, int64_t ldz, double scale, int64_t K, bool by_coordinate,
                     int32_t *crd, float *vals, float *lse, void *work, hipStream_t st);
// The K largest keys of every row as `lists` lists of K each (largest first, 0 where there are fewer), with as many running maxima and sums (float2):
// the sums begin at byte `at` of the work space, the keys `sums` bytes behind them; it takes `bytes`.  A workgroup can join `together` rows'
// lists afterwards: a row's lists are made one where those would be more than 16384 keys.  `finished` as in comet_beam_select.
struct TopLists { int64_t lists, at = 0, sums, bytes; bool joined; };
TopLists rows_top_lists(int type, int64_t N, int64_t V, int64_t K, int64_t together);
hipError_t rows_top_keys(const void *Z, int type, int64_t N, int64_t V, int64_t ldz, int64_t K, int64_t together, const TopLists &l, const uint8_t *finished, int32_t eos,
                         void *work, hipStream_t st);

struct DistillArgs {
    const void *Z;
    int type;
    int64_t N, V, ldz;
    const int32_t *pos;
    int64_t K;
    const int32_t *crd;
    const float *tvals, *tlse;
    double scale;
    const float *weight;
    bool once = false, shift = false;     // how rows are read: set by the launchers (once: the forward pass alone)
};
int64_t distill_work(int type, int64_t N, int64_t V);
hipError_t distill_forward(const DistillArgs &a, float *loss, double *stat, void *work, hipStream_t st);
hipError_t distill_backward(const DistillArgs &a, const double *stat, const float *dloss, void *dZ, int64_t lddz, hipStream_t st);
hipError_t distill_step(const DistillArgs &a, float *loss, void *dZ, int64_t lddz, void *work, hipStream_t st);

int64_t beam_select_work(int type, int64_t B, int64_t W, int64_t V, int64_t n);
hipError_t beam_select(const void *Z, int type, int64_t B, int64_t W, int64_t V, int64_t ldz, const float *score, const uint8_t *finished,
                       int32_t eos, int64_t n, float *out_score, int32_t *out_parent, int32_t *out_token, void *work, hipStream_t st);

int64_t draft_verify_work(int type, int64_t N, int64_t V, int64_t B, bool with_draft);
hipError_t draft_verify(const void *Z, int type, int64_t N, int64_t V, int64_t ldz, int64_t B, const int32_t *pos, const int32_t *token, const float *u,
                        const float *v, const void *draft, int draft_type, int64_t ldd, const int32_t *crd, const float *vals, int64_t K, double scale,
                        const float *scales, int32_t *accepted, int32_t *next, int32_t *length, void *work, hipStream_t st);

struct StateLayout {
    int64_t B, W, batch_stride, beam_stride, outer, outer_stride, inner;      // strides and inner in bytes
};
hipError_t beam_reorder(void *const *states, int64_t nstates, const StateLayout &l, const int32_t *parent, hipStream_t st);

}  // namespace comet
