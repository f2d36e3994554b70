// Distillation from a teacher's top logits: the kernels before and after the tensor-core passes.
//
// The student's logits at the K listed columns of a row are needed in fp32, at the precision that its log-sum-exp has.  Dot products
// of their own would read K rows of W per row of H (4.8 GB for 9,217 rows, K = 64, d = 4096; a [d, V] head has no such rows); the
// epilogue of the forward pass has every logit in a register, so it writes out the listed ones as it comes by.  For that the
// columns of a row have to be ascending: teacher_kernel sorts them.  Sorted entries also put an id that is given twice side by side.
//
// distill_rows_kernel then has one warp per row.  With r the teacher's probabilities over its entries and M their mass,
//     kl = M sum r (log r + log M - x + lse),   d kl / d x_v = M (p_v - sum_{k: id_k = v} r_k).
// The gradient off the listed columns is M p_v = M e^-lse e^x_v: the scratch keeps the e^x that the forward pass leaves (exp_form
// in lmhead.cuh), the listed columns become (p_v - r_v) e^lse, the difference formed in fp64 before its one rounding to bf16, and
// the dH pass scales the row by w M e^-lse / tau.  With dW the scratch is plain, coef (p - r), from 16-bit codes of the logits (code_form).  Rows
// whose lse is out of their form's range are recomputed in plain form.
#include <cuda_fp16.h>
#include <float.h>

#include "../../include/ais.h"
#include "distill.cuh"
#include "launch.cuh"
#include "lmhead.cuh"

namespace ais {

namespace {

constexpr int kTeacherWarps = 4;

__device__ __forceinline__ float load_logit(const void* p, int dtype, int64_t i) {
    return dtype == AIS_F32 ? static_cast<const float*>(p)[i]
           : dtype == AIS_F16 ? __half2float(static_cast<const __half*>(p)[i])
                              : __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}

// A warp sorts the (id, position) pairs of a row; n2 is K rounded up to a power of two.
__global__ void __launch_bounds__(kTeacherWarps * 32) teacher_kernel(const TeacherJob a, int n2) {
    extern __shared__ unsigned long long keys_all[];
    pdl_enter();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < a.clear_bytes / 16; i += static_cast<int64_t>(gridDim.x) * blockDim.x)
        static_cast<uint4*>(a.clear)[i] = make_uint4(0, 0, 0, 0);
    if (warp == 0 && static_cast<int64_t>(blockIdx.x) * kBM < a.T) {
        int rows = 0;
        for (int j = 0; j < kBM; j += 32) {
            const int64_t t = static_cast<int64_t>(blockIdx.x) * kBM + j + lane;
            rows += __popc(__ballot_sync(0xffffffffu, t < a.T && a.mask[t] != 0));
        }
        if (lane == 0) a.tile_rows[blockIdx.x] = static_cast<uint8_t>(rows);      // (128 at most)
    }
    const int64_t t = static_cast<int64_t>(blockIdx.x) * kTeacherWarps + warp;
    if (t < a.T && a.mask[t] != 0) {
        unsigned long long* keys = keys_all + warp * n2;
        bool beyond = false;
        for (int k = lane; k < n2; k += 32) {
            int id = 0;
            if (k < a.K) id = a.ids[t * a.ldk + k];
            beyond |= k < a.K && id >= a.V;
            keys[k] = k < a.K ? (static_cast<unsigned long long>(static_cast<uint32_t>(id) ^ 0x80000000u) << 32) | static_cast<uint32_t>(k) : ~0ull;
        }
        __syncwarp();
        for (int size = 2; size <= n2; size <<= 1)
            for (int stride = size >> 1; stride > 0; stride >>= 1) {
                for (int p = lane; p < n2 / 2; p += 32) {
                    const int i = 2 * p - (p & (stride - 1)), j = i + stride;
                    const unsigned long long x = keys[i], y = keys[j];
                    if ((x > y) == ((i & size) == 0)) {
                        keys[i] = y;
                        keys[j] = x;
                    }
                }
                __syncwarp();
            }
        for (int k = lane; k < a.K; k += 32) {
            const unsigned long long key = keys[k];
            const int id = static_cast<int>(static_cast<uint32_t>(key >> 32) ^ 0x80000000u);
            a.sorted_ids[t * a.K + k] = id;
            a.sorted_logits[t * a.K + k] = id >= 0 && id < a.V ? load_logit(a.logits, a.dtype, t * a.ldk + static_cast<uint32_t>(key)) : -INFINITY;
        }
        if (__any_sync(0xffffffffu, beyond) && lane == 0 && a.status) atomicOr(a.status, AIS_FLAG_TOKEN_RANGE);
    }
}

__device__ __forceinline__ double warp_add(double v) {
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ float warp_max(float v) {
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

__global__ void __launch_bounds__(kDistillRows * 32) distill_rows_kernel(const __grid_constant__ DistillJob a) {
    __shared__ double row_loss[kDistillRows];
    __shared__ int warp_rows[kDistillRows];
    __shared__ bool last;
    pdl_enter();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int n_valid = 0;                                              // rows of the batch with mask 1
    for (int i = threadIdx.x; i < a.tiles; i += kDistillRows * 32) n_valid += a.tile_rows[i];
    n_valid = __reduce_add_sync(0xffffffffu, n_valid);
    if (lane == 0) warp_rows[warp] = n_valid;
    __syncthreads();
    n_valid = 0;
    for (int i = 0; i < kDistillRows; ++i) n_valid += warp_rows[i];
    const int64_t lrow = static_cast<int64_t>(blockIdx.x) * kDistillRows + warp, t = a.row0 + lrow;
    double contribution = 0.0;
    if (lrow < a.rows) {
        float kl = 0.f, lse_out = 0.f, coef = 0.f, scale = 0.f;
        if (a.mask[t] != 0) {
            // the student's log-sum-exp from the partial sums of its vocabulary ranges
            float m = -INFINITY;
            bool nan = false;
            for (int i = lane; i < a.nparts; i += 32) {
                const float pm = a.part_m[i * a.part_ld + t];
                nan |= isnan(pm);
                m = fmaxf(m, pm);
            }
            m = warp_max(m);
            double s = 0.0;
            for (int i = lane; i < a.nparts; i += 32)
                s += static_cast<double>(a.part_s[i * a.part_ld + t]) * exp(static_cast<double>(a.part_m[i * a.part_ld + t]) - static_cast<double>(m));
            const double lse = static_cast<double>(m) + log(warp_add(s));
            // the teacher's over its entries
            const int64_t at = t * a.K;
            float top = -INFINITY;
            for (int k = lane; k < a.K; k += 32) {
                const float v = a.logits[at + k];
                nan |= !(v < INFINITY);
                top = fmaxf(top, v);
            }
            top = warp_max(top);
            nan = __any_sync(0xffffffffu, nan);
            const bool empty = !nan && top == -INFINITY;
            double z = 0.0;
            if (!empty)
                for (int k = lane; k < a.K; k += 32) z += exp((static_cast<double>(a.logits[at + k]) - static_cast<double>(top)) * a.inv_tau);
            const double lse_k = static_cast<double>(top) * a.inv_tau + log(warp_add(z));
            const double log_mass = a.teacher_lse && !empty ? lse_k - static_cast<double>(a.teacher_lse[t]) : 0.0;
            const double mass = exp(log_mass);
            double sum = 0.0;
            if (!empty)
                for (int k = lane; k < a.K; k += 32) {
                    const double log_r = static_cast<double>(a.logits[at + k]) * a.inv_tau - lse_k;
                    const double r = exp(log_r);
                    if (r > 0.0) sum += r * (log_r + log_mass - static_cast<double>(a.pick[at + k]) + lse);
                }
            sum = mass * warp_add(sum);
            const double w = a.weights ? static_cast<double>(a.weights[t]) : 1.0 / static_cast<double>(n_valid);
            const bool good = !nan && isfinite(lse) && isfinite(sum) && isfinite(mass) && isfinite(w);
            lse_out = good ? static_cast<float>(lse) : NAN;
            if (!good && lane == 0 && a.status) atomicOr(a.status, AIS_FLAG_NONFINITE);
            if (good && !empty) {
                kl = static_cast<float>(sum);
                contribution = w * sum;
                coef = static_cast<float>(w * mass * a.inv_tau);
                // the row's factor, and what the scratch holds at the listed columns: (p - r) e^lse, or coef (p - r).  A factor that fp32
                // would cut to a few bits (|w| M / tau below 5e-13 at an lse of 59) leaves the row to the plain form, which is factor 1.
                const double factor = w * mass * a.inv_tau * exp(-lse);
                const bool kept = a.U != nullptr && exp_form(lse_out) && fabs(factor) >= static_cast<double>(FLT_MIN);
                scale = kept ? static_cast<float>(factor) : 1.f;
                const double f = kept ? exp(lse) : w * mass * a.inv_tau;
                if (a.redo && !(a.U ? kept : code_form(lse_out)) && coef != 0.f && lane == 0) {
                    a.redo_flags[t / kBM] = 1;
                    atomicAdd(a.redo_count, 1u);
                }
                for (int k = lane; k < a.K; k += 32) {
                    const int id = a.ids[at + k];
                    if (id < 0 || id >= a.V) continue;
                    double r = 0.0;                          // all entries with this id, in their order
                    int j = k;
                    while (j > 0 && a.ids[at + j - 1] == id) --j;
                    for (; j < a.K && a.ids[at + j] == id; ++j) r += exp(static_cast<double>(a.logits[at + j]) * a.inv_tau - lse_k);
                    const float v = static_cast<float>((exp(static_cast<double>(a.pick[at + k]) - lse) - r) * f);
                    a.pick[at + k] = v;
                    if (kept) a.U[lrow * a.ldU + id] = __float2bfloat16(v);
                }
            }
        }
        if (lane == 0) {
            a.kl[t] = kl;
            if (a.lse) a.lse[t] = lse_out;
            a.row_lse[t] = lse_out;
            a.coef[t] = coef;
            a.scale[t] = coef != 0.f ? scale : 0.f;
        }
    }
    // the loss: rows of a block in order, then the blocks in order, by the block that finishes last
    if (lane == 0) row_loss[warp] = contribution;
    __syncthreads();
    if (threadIdx.x == 0) {
        double sum = 0.0;
        for (int i = 0; i < kDistillRows; ++i) sum += row_loss[i];
        a.partials[a.row0 / kDistillRows + blockIdx.x] = sum;
        __threadfence();
        last = atomicAdd(a.ticket, 1u) == static_cast<uint32_t>(a.n_partials - 1);
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double sum = 0.0;
    for (int i = threadIdx.x; i < a.n_partials; i += kDistillRows * 32) sum += __ldcg(a.partials + i);
    sum = warp_add(sum);
    __syncthreads();
    if (lane == 0) row_loss[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double all = 0.0;
        for (int i = 0; i < kDistillRows; ++i) all += row_loss[i];
        if (a.loss) *a.loss = static_cast<float>(all);
        if (n_valid == 0 && a.status) atomicOr(a.status, AIS_FLAG_EMPTY);
    }
}

// A block has 8,192 columns of a row, 16 bytes of codes per thread and load.
constexpr int kExpandCols = 8192;
__global__ void __launch_bounds__(256) expand_kernel(const __grid_constant__ ExpandJob a) {
    pdl_enter();
    const int64_t t = blockIdx.y;
    const int from = blockIdx.x * kExpandCols, to = min(from + kExpandCols, a.V);
    uint4* row = reinterpret_cast<uint4*>(a.U + t * a.ldU);
    const float coef = a.coef[t];
    constexpr float kLog2e = 1.4426950408889634f;
    const float step = kLog2e / kCodeSteps, shift = -(kCodeZero + a.lse[t]) * kLog2e;
    uint4 raw[kExpandCols / 2048];
    if (coef != 0.f) {
#pragma unroll
        for (int j = 0; j < kExpandCols / 2048; ++j) {
            const int c = from + (j * 256 + threadIdx.x) * 8;
            if (c < to) raw[j] = __ldcs(row + c / 8);
        }
    }
#pragma unroll
    for (int j = 0; j < kExpandCols / 2048; ++j) {
        const int c = from + (j * 256 + threadIdx.x) * 8;
        if (c >= to) break;
        uint32_t w[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t lo = w[k] & 0xffffu, hi = w[k] >> 16;
            const float x = lo != 0u && coef != 0.f ? coef * exp2f(fmaf(static_cast<float>(lo), step, shift)) : 0.f;
            const float y = hi != 0u && coef != 0.f ? coef * exp2f(fmaf(static_cast<float>(hi), step, shift)) : 0.f;
            const __nv_bfloat162 p = __floats2bfloat162_rn(x, y);
            w[k] = *reinterpret_cast<const uint32_t*>(&p);
        }
        row[c / 8] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    if (coef == 0.f) return;
    __syncthreads();
    const int32_t* ids = a.ids + t * a.K;
    int lo = 0, hi = a.K;                                         // the first listed column of this block
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (ids[mid] < from) lo = mid + 1;
        else hi = mid;
    }
    for (int k = lo + threadIdx.x; k < a.K && ids[k] < to; k += 256) a.U[t * a.ldU + ids[k]] = __float2bfloat16(a.pick[t * a.K + k]);
}

__global__ void __launch_bounds__(256) live_rows_kernel(const __nv_bfloat16* src, int64_t ld, int d, const float* coef, __nv_bfloat16* dst) {
    pdl_enter();
    const int64_t t = blockIdx.x;
    const bool live = coef[t] != 0.f;
    for (int c = threadIdx.x; c < d / 8; c += 256)
        reinterpret_cast<uint4*>(dst + t * ld)[c] = live ? reinterpret_cast<const uint4*>(src + t * ld)[c] : make_uint4(0, 0, 0, 0);
}

}  // namespace

cudaError_t launch_expand(const ExpandJob& job, cudaStream_t stream) {
    // (65,535 rows per launch at most: the y dimension of a grid)
    for (int64_t r0 = 0; r0 < job.rows; r0 += 65535) {
        ExpandJob part = job;
        part.U += r0 * job.ldU;
        part.rows = job.rows - r0 < 65535 ? job.rows - r0 : 65535;
        part.coef += r0;
        part.lse += r0;
        part.ids += r0 * job.K;
        part.pick += r0 * job.K;
        const cudaError_t e = launch_pdl(expand_kernel, dim3((job.V + kExpandCols - 1) / kExpandCols, static_cast<unsigned>(part.rows)), 256, 0, stream, part);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

cudaError_t launch_live_rows(const __nv_bfloat16* src, int64_t ld, int64_t rows, int32_t d, const float* coef, __nv_bfloat16* dst, cudaStream_t stream) {
    return launch_pdl(live_rows_kernel, static_cast<unsigned>(rows), 256, 0, stream, src, ld, d, coef, dst);
}

cudaError_t launch_teacher(const TeacherJob& job, cudaStream_t stream) {
    int n2 = 2;
    while (n2 < job.K) n2 <<= 1;
    const unsigned blocks = static_cast<unsigned>((job.T + kTeacherWarps - 1) / kTeacherWarps);
    return launch_pdl(teacher_kernel, blocks, kTeacherWarps * 32, sizeof(unsigned long long) * kTeacherWarps * n2, stream, job, n2);
}

cudaError_t launch_distill_rows(const DistillJob& job, cudaStream_t stream) {
    const unsigned blocks = static_cast<unsigned>((job.rows + kDistillRows - 1) / kDistillRows);
    return launch_pdl(distill_rows_kernel, blocks, kDistillRows * 32, 0, stream, job);
}

}  // namespace ais
