// A student's loss against a teacher's largest logits and the labels, and its gradient (rk_distill_loss,
// rk_distill_backward, rk_distill_loss_backward).
#include <cmath>
#include <type_traits>

#include "rk_vec.h"

namespace {

constexpr int DS_THREADS = 512, DS_WAVES = 8;

struct DistillArgs {
    const void *student;
    void *d_student;
    uint64_t st, d_st, n_rows;
    uint32_t vocab, top_k, t_type;
    const void *teacher;
    uint64_t t_st;
    const int32_t *index, *label;
    const float *row_weight, *d_total;
    float *loss, *lse, *total;
    float temperature, kd, ce;
};

__device__ __forceinline__ float block_sum(float v, float *lds, uint32_t lane, uint32_t wave) {
    v = wave_sum(v);
    __syncthreads();
    if (lane == 0) lds[wave] = v;
    __syncthreads();
    return row_sum((lane & 15u) < DS_WAVES ? lds[lane & 15u] : 0.f);
}
__device__ __forceinline__ float block_max(float v, float *lds, uint32_t lane, uint32_t wave) {
    v = wave_max(v);
    __syncthreads();
    if (lane == 0) lds[wave] = v;
    __syncthreads();
    return row_max((lane & 15u) < DS_WAVES ? lds[lane & 15u] : -INFINITY);
}
__device__ __forceinline__ float teacher_at(const DistillArgs &A, uint64_t r, uint32_t k) {
    const uint64_t at = r * A.t_st + k;
    return A.t_type == RK_F32 ? ((const float *)A.teacher)[at] : A.t_type == RK_BF16 ? (float)((const __bf16 *)A.teacher)[at] : (float)((const _Float16 *)A.teacher)[at];
}

// A workgroup a row.  LOSS: the sums of the softmax over the row, then the loss; GRAD: the gradient, from these or from lse.
template <bool CUTS, typename T, int CH, bool LOSS, bool GRAD>
__global__ __launch_bounds__(DS_THREADS) void k_distill(DistillArgs A) {
    __shared__ float q[RK_MAX_TEACHER_LOGITS], sv[RK_MAX_TEACHER_LOGITS], red[16];
    __shared__ int32_t at[RK_MAX_TEACHER_LOGITS];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6, V = A.vocab, K = A.kd > 0.f ? A.top_k : 0u;
    const uint64_t r = blockIdx.x;
    const T *const row = (const T *)A.student + r * A.st;
    T *const out = (T *)A.d_student + r * A.d_st;
    const Row<T> from(A.student, r, A.st, V), to(A.d_student, r, A.d_st, V);
    const float weight = A.row_weight ? A.row_weight[r] : 1.f;
    const float inv_t = 1.f / A.temperature;
    float lse_t = 0.f, lse_1 = 0.f;
    bool there = weight != 0.f;
    if (there && LOSS) {
        float m = -INFINITY, st = 0.f, s1 = 0.f;
        for (uint32_t c0 = tid * CH; c0 < V; c0 += DS_THREADS * CH) {
            const Place at(c0, V, CH);
            const int32_t valid = at.valid;
            float v[CH], top = m;
            load_row<CUTS, T, CH>(from, at, v);
#pragma unroll
            for (int i = 0; i < CH; ++i) if (i < valid) top = fmaxf(top, v[i]);
            const float ref = top == -INFINITY ? 0.f : top;
            if (top > m) { st *= exp_f32((m - ref) * inv_t); s1 *= exp_f32(m - ref); m = top; }
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                if (i >= valid) continue;
                if (A.kd > 0.f) st += exp_f32((v[i] - ref) * inv_t);
                if (A.ce > 0.f) s1 += exp_f32(v[i] - ref);
            }
        }
        const float top = block_max(m, red, lane, wave);
        if (top == -INFINITY) {
            there = false;
            lse_t = A.kd > 0.f ? -INFINITY : 0.f; lse_1 = A.ce > 0.f ? -INFINITY : 0.f;
        } else {
            // a thread that saw nothing above -inf has sums of zero (or NaN), taken about zero
            const float own = m == -INFINITY ? 0.f : (m - top);
            st = block_sum(st * exp_f32(own * inv_t), red, lane, wave);
            s1 = block_sum(s1 * exp_f32(own), red, lane, wave);
            if (A.kd > 0.f) lse_t = top * inv_t + logf(st);
            if (A.ce > 0.f) lse_1 = top + logf(s1);
        }
    }
    if (there && !LOSS) {
        lse_t = A.lse[2 * r]; lse_1 = A.lse[2 * r + 1];
        there = (A.kd > 0.f ? lse_t : lse_1) != -INFINITY;
    }
    const int32_t label = A.ce > 0.f && there ? A.label[r] : -1;
    const bool labelled = label >= 0 && (uint32_t)label < V;
    float ce = labelled ? A.ce : 0.f, big_q = 0.f, log_sum = 0.f, tmax = -INFINITY;
    if (there && K) {
        for (uint32_t k = tid; k < K; k += DS_THREADS) {
            const int32_t i = A.index[r * K + k];
            const float t = teacher_at(A, r, k);
            const bool kept = i >= 0 && (uint32_t)i < V && t != -INFINITY;
            at[k] = kept ? i : -1;
            q[k] = t;
            sv[k] = kept ? (float)row[i] : 0.f;
            if (kept) tmax = fmaxf(tmax, t);
        }
        tmax = block_max(tmax, red, lane, wave);
        float s = 0.f, some = 0.f;
        for (uint32_t k = tid; k < K; k += DS_THREADS) {
            if (at[k] < 0) continue;
            some = 1.f;
            s += exp_f32((q[k] - tmax) * inv_t);
        }
        s = block_sum(s, red, lane, wave);
        big_q = block_max(some, red, lane, wave);
        log_sum = logf(s);
    }
    const float kd = big_q > 0.f ? A.kd : 0.f;
    if (there && K) {
        float part = 0.f;
        for (uint32_t k = tid; k < K; k += DS_THREADS) {
            if (at[k] < 0) continue;
            const float log_q = (q[k] - tmax) * inv_t - log_sum, v = exp_f32(log_q);
            q[k] = v;
            if (v != 0.f) part += v * (log_q - (sv[k] * inv_t - lse_t));
        }
        if (LOSS) part = block_sum(part, red, lane, wave);
        if (LOSS && tid == 0) {
            float l = kd * A.temperature * A.temperature * part;
            if (labelled) l += ce * (lse_1 - (float)row[label]);
            A.loss[r] = l;
        }
    } else if (LOSS && tid == 0) {
        A.loss[r] = there && labelled ? ce * (lse_1 - (float)row[label]) : 0.f;
    }
    if (LOSS && tid == 0) { A.lse[2 * r] = lse_t; A.lse[2 * r + 1] = lse_1; }
    if (!GRAD) return;
    const float scale = there ? weight * (A.d_total ? A.d_total[0] : 1.f) : 0.f;
    const float ft = scale * kd * A.temperature, f1 = scale * ce;
    const float label_v = labelled ? (float)row[label] : 0.f;
    __syncthreads();                            // d_student may be student: what the rest needs of the row is held
    for (uint32_t c0 = tid * CH; c0 < V; c0 += DS_THREADS * CH) {
        const Place place(c0, V, CH);
        float v[CH] = {};
        if (there) {
            load_row<CUTS, T, CH>(from, place, v);
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                float d = 0.f;
                if (kd > 0.f) d += ft * exp_f32(v[i] * inv_t - lse_t);
                if (ce > 0.f) d += f1 * exp_f32(v[i] - lse_1);
                v[i] = d;
            }
        }
        store_row<CUTS, T, CH>(to, place, v);
    }
    if (!there) return;
    __syncthreads();
    // where teacher or label have something: the whole value, once more (equal indices get equal values)
    auto fix = [&](int32_t i, float s) {
        float d = 0.f;
        if (kd > 0.f) {
            float mass = 0.f;
            for (uint32_t k = 0; k < K; ++k) mass += at[k] == i ? q[k] : 0.f;
            d += ft * (exp_f32(s * inv_t - lse_t) - mass);
        }
        if (ce > 0.f) d += f1 * (exp_f32(s - lse_1) - (i == label ? 1.f : 0.f));
        out[i] = (T)d;
    };
    for (uint32_t k = tid; k < K; k += DS_THREADS)
        if (at[k] >= 0) fix(at[k], sv[k]);
    if (tid == 0 && labelled) fix(label, label_v);
}

// the rows' losses added up, in one order
__global__ __launch_bounds__(1024) void k_distill_total(DistillArgs A) {
    __shared__ double lds[1024];
    double s = 0.0;
    for (uint64_t r = threadIdx.x; r < A.n_rows; r += 1024) {
        const float w = A.row_weight ? A.row_weight[r] : 1.f;
        if (w != 0.f) s += (double)w * (double)A.loss[r];
    }
    lds[threadIdx.x] = s;
    for (uint32_t off = 512; off; off >>= 1) {
        __syncthreads();
        if (threadIdx.x < off) lds[threadIdx.x] += lds[threadIdx.x + off];
    }
    if (threadIdx.x == 0) A.total[0] = (float)lds[0];
}

// ---- host
int32_t check_distill(rk_ctx *ctx, const rk_distill *d, uint64_t n_rows, uint32_t vocab, const rk_matrix *student, const rk_teacher *t, DistillArgs &A) {
    if (!d || !t) return rk_fail(ctx, RK_ERR_INVALID_ARG, "distill or teacher is null");
    if (!(d->temperature > 0.f) || !std::isfinite(d->temperature) || !(d->kd_weight >= 0.f) || !(d->ce_weight >= 0.f) ||
        !std::isfinite(d->kd_weight) || !std::isfinite(d->ce_weight) || (d->kd_weight == 0.f && d->ce_weight == 0.f))
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "temperature not positive, or weights negative, not finite or both 0");
    if (vocab < 1) return rk_fail(ctx, RK_ERR_INVALID_ARG, "vocab below 1");
    if (vocab > ROW_MAX || n_rows > 0x7FFFFFFFull) return rk_fail(ctx, RK_ERR_UNSUPPORTED, "vocab beyond 2^28, or n_rows beyond 2^31 - 1");
    if (!rk_matrix_ok(student, n_rows, vocab)) return rk_fail(ctx, RK_ERR_INVALID_ARG, "student null, misaligned or of a stride below vocab");
    if ((t->logits != nullptr) != (d->kd_weight > 0.f)) return rk_fail(ctx, RK_ERR_INVALID_ARG, "the teacher's logits go with kd_weight");
    if ((t->label != nullptr) != (d->ce_weight > 0.f) && n_rows) return rk_fail(ctx, RK_ERR_INVALID_ARG, "labels go with ce_weight");
    if (t->logits) {
        if (t->top_k < 1) return rk_fail(ctx, RK_ERR_INVALID_ARG, "top_k below 1");
        if (t->top_k > RK_MAX_TEACHER_LOGITS) return rk_fail(ctx, RK_ERR_UNSUPPORTED, "%u logits of the teacher, %u at most", t->top_k, RK_MAX_TEACHER_LOGITS);
        if (!rk_matrix_ok(t->logits, n_rows, t->top_k) || (n_rows && !t->index)) return rk_fail(ctx, RK_ERR_INVALID_ARG, "the teacher's logits or indices null, misaligned or of a stride below top_k");
    }
    if ((((uintptr_t)t->index | (uintptr_t)t->label | (uintptr_t)t->row_weight) & 3u)) return rk_fail(ctx, RK_ERR_INVALID_ARG, "misaligned indices, labels or weights");
    A.student = student->data; A.st = student->stride; A.n_rows = n_rows; A.vocab = vocab;
    if (t->logits) { A.teacher = t->logits->data; A.t_st = t->logits->stride; A.t_type = t->logits->type; A.index = t->index; A.top_k = t->top_k; }
    A.label = t->label; A.row_weight = t->row_weight;
    A.temperature = d->temperature; A.kd = d->kd_weight; A.ce = d->ce_weight;
    return RK_OK;
}
template <bool LOSS, bool GRAD> void launch_type(hipStream_t st, uint32_t type, const DistillArgs &A) {
    const uint32_t n = (uint32_t)A.n_rows;
    auto go = [&](auto cuts) {
        constexpr bool CUTS = decltype(cuts)::value;
        if (type == RK_F32) k_distill<CUTS, float, 4, LOSS, GRAD><<<n, DS_THREADS, 0, st>>>(A);
        else if (type == RK_BF16) k_distill<CUTS, __bf16, 8, LOSS, GRAD><<<n, DS_THREADS, 0, st>>>(A);
        else k_distill<CUTS, _Float16, 8, LOSS, GRAD><<<n, DS_THREADS, 0, st>>>(A);
    };
    if (A.vocab % (type == RK_F32 ? 4 : 8)) go(std::true_type()); else go(std::false_type());
}
int32_t run(rk_ctx *ctx, uint32_t type, DistillArgs &A, bool want_loss, bool want_grad) {
    RK_HIP(ctx, hipSetDevice(ctx->device));
    if (A.n_rows) {
        if (want_loss && want_grad) launch_type<true, true>(ctx->stream, type, A);
        else if (want_loss) launch_type<true, false>(ctx->stream, type, A);
        else launch_type<false, true>(ctx->stream, type, A);
        RK_CHECK_LAUNCH(ctx, "k_distill");
    }
    if (want_loss) {
        k_distill_total<<<1, 1024, 0, ctx->stream>>>(A);
        RK_CHECK_LAUNCH(ctx, "k_distill_total");
    }
    return RK_OK;
}
int32_t check_results(rk_ctx *ctx, const DistillArgs &A) {
    if ((A.n_rows && (!A.loss || !A.lse)) || !A.total || (((uintptr_t)A.loss | (uintptr_t)A.lse | (uintptr_t)A.total) & 3u))
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "loss, lse or total null or misaligned");
    return RK_OK;
}
int32_t check_gradient(rk_ctx *ctx, const rk_matrix *d, const rk_matrix *student, const float *d_total, DistillArgs &A) {
    if (!rk_matrix_ok(d, A.n_rows, A.vocab) || d->type != student->type || ((uintptr_t)d_total & 3u))
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "d_student null, misaligned, of a stride below vocab or of another type than the student; or d_total misaligned");
    A.d_student = d->data; A.d_st = d->stride; A.d_total = d_total;
    return RK_OK;
}

}  // namespace

extern "C" int32_t rk_distill_loss(rk_ctx *ctx, const rk_distill *distill, uint64_t n_rows, uint32_t vocab, const rk_matrix *student,
                                   const rk_teacher *teacher, float *loss, float *lse, float *total) {
    if (!ctx) return RK_ERR_INVALID_ARG;
    DistillArgs A{};
    int32_t rc = check_distill(ctx, distill, n_rows, vocab, student, teacher, A);
    if (rc != RK_OK) return rc;
    A.loss = loss; A.lse = lse; A.total = total;
    if ((rc = check_results(ctx, A)) != RK_OK) return rc;
    return run(ctx, student->type, A, true, false);
}

extern "C" int32_t rk_distill_backward(rk_ctx *ctx, const rk_distill *distill, uint64_t n_rows, uint32_t vocab, const rk_matrix *student,
                                       const rk_teacher *teacher, const float *lse, const float *d_total, const rk_matrix *d_student) {
    if (!ctx) return RK_ERR_INVALID_ARG;
    DistillArgs A{};
    int32_t rc = check_distill(ctx, distill, n_rows, vocab, student, teacher, A);
    if (rc != RK_OK) return rc;
    if (n_rows && (!lse || ((uintptr_t)lse & 3u))) return rk_fail(ctx, RK_ERR_INVALID_ARG, "lse null or misaligned");
    A.lse = const_cast<float *>(lse);
    if ((rc = check_gradient(ctx, d_student, student, d_total, A)) != RK_OK) return rc;
    return run(ctx, student->type, A, false, true);
}

extern "C" int32_t rk_distill_loss_backward(rk_ctx *ctx, const rk_distill *distill, uint64_t n_rows, uint32_t vocab, const rk_matrix *student,
                                            const rk_teacher *teacher, const float *d_total, float *loss, float *lse, float *total,
                                            const rk_matrix *d_student) {
    if (!ctx) return RK_ERR_INVALID_ARG;
    DistillArgs A{};
    int32_t rc = check_distill(ctx, distill, n_rows, vocab, student, teacher, A);
    if (rc != RK_OK) return rc;
    A.loss = loss; A.lse = lse; A.total = total;
    if ((rc = check_results(ctx, A)) != RK_OK) return rc;
    if ((rc = check_gradient(ctx, d_student, student, d_total, A)) != RK_OK) return rc;
    return run(ctx, student->type, A, true, true);
}
