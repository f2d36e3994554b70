// The kernels around the tensor-core passes of a distillation step (distill.cu).
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace ais {

// Opening of a distillation step: a teacher's entries of every row brought into the order that the tensor-core epilogues walk, ids ascending,
// the logits along; the rows of every 128-row tile counted; `clear` (16-byte words) zeroed.
struct TeacherJob {
    const int32_t* ids;
    const void* logits;
    int dtype;
    int64_t ldk;
    int32_t K, V;
    int64_t T;
    const uint8_t* mask;
    int32_t* sorted_ids;       // [T][K]; negative and out-of-range ids keep their place in the order
    float* sorted_logits;      // [T][K]; -inf for entries that do not count
    uint8_t* tile_rows;        // rows with mask 1 of every tile
    void* clear;
    int64_t clear_bytes;
    uint32_t* status;
};
cudaError_t launch_teacher(const TeacherJob& job, cudaStream_t stream);

// The rows of one forward launch: its partial sums merged, KL per row, gradient factors, and what the scratch holds at the listed
// columns.
struct DistillJob {
    int64_t row0, rows;        // of the batch
    int32_t K, V;
    double inv_tau;
    const uint8_t* mask;
    const float *part_m, *part_s;   // [nparts][part_ld], indexed by the row of the batch
    int32_t nparts;
    int64_t part_ld;
    const int32_t* ids;        // sorted, [T][K]
    const float* logits;
    float* pick;               // [T][K]: scaled student logits in, scratch values out
    const float* teacher_lse;
    const float* weights;
    const uint8_t* tile_rows;  // [ceil(T / 128)] rows with mask 1
    int32_t tiles;
    float *kl, *lse;           // lse may be NULL
    float* row_lse;            // [T] workspace: lse of every row, for the recompute pass
    float* coef;               // [T] workspace: w M / tau
    float* scale;              // [T] factor of the row in the dH pass: 0 where there is no gradient (the row's scratch may meet a NaN in W)
    __nv_bfloat16* U;          // scratch of this launch's rows in exponent form; NULL: codes, or no scratch
    int64_t ldU;
    bool redo;                 // row tiles with a row outside the form of the scratch are marked
    uint8_t* redo_flags;       // per row tile of the batch, zeroed before
    uint32_t* redo_count;
    double* partials;          // [ceil(T / kDistillRows)]
    int32_t n_partials;        // of the whole batch
    uint32_t* ticket;          // zeroed before; the block that completes the batch adds up the loss
    float* loss;
    uint32_t* status;
};
constexpr int kDistillRows = 8;         // rows of a block (a warp each)
cudaError_t launch_distill_rows(const DistillJob& job, cudaStream_t stream);

// Scratch rows of codes (kCodeSteps in lmhead.cuh) to coef e^(x - lse), and what pick holds at the listed columns; zeros for rows with coef 0.
// All per-row arrays begin at the first row of the scratch.
struct ExpandJob {
    __nv_bfloat16* U;
    int64_t ldU, rows;
    int32_t V, K;
    const float *coef, *lse;
    const int32_t* ids;
    const float* pick;
};
cudaError_t launch_expand(const ExpandJob& job, cudaStream_t stream);

// dst = src for the rows with coef != 0, zeros for the others; both with row stride ld.
cudaError_t launch_live_rows(const __nv_bfloat16* src, int64_t ld, int64_t rows, int32_t d, const float* coef, __nv_bfloat16* dst, cudaStream_t stream);

}  // namespace ais
