// Gated linear recurrence over packed sequences, and its gradient (rk_recur in rubick.h).
//
// The simplest form: a lane has a column and goes through all rows of it, one after the other.
#include "rk_vec.h"

namespace {

constexpr uint32_t RC_THREADS = 64;

struct RecurArgs {
    const void *x, *z, *h, *dh, *bias;
    void *out, *dx, *dz;
    uint64_t x_st, z_st, h_st, dh_st, o_st, dx_st, dz_st;
    const float *state_in, *d_state_out;
    float *state_out, *d_state_in, *d_bias;
    uint64_t si_st, so_st, dso_st, dsi_st;
    const int32_t *offsets;
    uint64_t seq_rows, n_rows;
    uint32_t n_seqs, width, coupled, bias_type;
};

__device__ __forceinline__ float bias_at(const RecurArgs &A, uint32_t c) {
    if (!A.bias) return 0.f;
    if (A.bias_type == RK_F32) return ((const float *)A.bias)[c];
    return A.bias_type == RK_BF16 ? (float)((const __bf16 *)A.bias)[c] : (float)((const _Float16 *)A.bias)[c];
}
// f = sigmoid(v) and 1 - f, neither as a difference from one
struct Gate { float f, not_f; };
__device__ __forceinline__ Gate gate_of(float v) {
    const float e = exp_f32(-fabsf(v)), near = 1.f / (1.f + e), far = e * near;
    return v >= 0.f ? Gate{near, far} : Gate{v != v ? v : far, v != v ? v : near};
}
__device__ __forceinline__ void seq_range(const RecurArgs &A, uint32_t s, uint64_t &first, uint64_t &end) {
    if (A.offsets) {
        const int64_t a = A.offsets[s], b = A.offsets[s + 1];
        first = a < 0 ? 0 : (uint64_t)a;
        end = b < 0 ? 0 : (uint64_t)b < A.n_rows ? (uint64_t)b : A.n_rows;
    } else {
        first = s * A.seq_rows;
        end = first + A.seq_rows < A.n_rows ? first + A.seq_rows : A.n_rows;
    }
}

template <typename T> __global__ __launch_bounds__(RC_THREADS) void k_recur_forward(const RecurArgs A) {
    const uint32_t c = blockIdx.x * RC_THREADS + threadIdx.x;
    if (c >= A.width) return;
    const float bias = bias_at(A, c);
    for (uint32_t s = 0; s < A.n_seqs; ++s) {
        uint64_t first, end;
        seq_range(A, s, first, end);
        float h = A.state_in ? A.state_in[s * A.si_st + c] : 0.f;
        for (uint64_t t = first; t < end; ++t) {
            const Gate g = gate_of((float)((const T *)A.z)[t * A.z_st + c] + bias);
            const float x = (float)((const T *)A.x)[t * A.x_st + c];
            h = g.f * h + (A.coupled ? g.not_f * x : x);
            ((T *)A.out)[t * A.o_st + c] = (T)h;
        }
        if (A.state_out) A.state_out[s * A.so_st + c] = h;
    }
}

template <typename T> __global__ __launch_bounds__(RC_THREADS) void k_recur_backward(const RecurArgs A) {
    const uint32_t c = blockIdx.x * RC_THREADS + threadIdx.x;
    if (c >= A.width) return;
    const float bias = bias_at(A, c);
    float sum = 0.f;
    for (uint32_t s = 0; s < A.n_seqs; ++s) {
        uint64_t first, end;
        seq_range(A, s, first, end);
        const float before = A.state_in ? A.state_in[s * A.si_st + c] : 0.f;
        float carry = A.d_state_out ? A.d_state_out[s * A.dso_st + c] : 0.f;
        for (uint64_t t = end; t-- > first;) {
            const Gate g = gate_of((float)((const T *)A.z)[t * A.z_st + c] + bias);
            const float x = A.coupled ? (float)((const T *)A.x)[t * A.x_st + c] : 0.f;
            const float h = t > first ? (float)((const T *)A.h)[(t - 1) * A.h_st + c] : before;
            const float e = (float)((const T *)A.dh)[t * A.dh_st + c] + carry;
            const float dz = e * (h - x) * (g.f * g.not_f);
            carry = g.f * e;
            sum += dz;
            ((T *)A.dx)[t * A.dx_st + c] = (T)(A.coupled ? g.not_f * e : e);
            ((T *)A.dz)[t * A.dz_st + c] = (T)dz;
        }
        if (A.d_state_in) A.d_state_in[s * A.dsi_st + c] = carry;
    }
    if (A.d_bias) A.d_bias[c] = sum;
}

template <typename F> void with_type(uint32_t type, F f) {
    if (type == RK_F32) f(float()); else if (type == RK_BF16) f(__bf16()); else f(_Float16());
}
// what both directions check alike; how many sequences there are
int32_t check_recur(rk_ctx *ctx, const rk_recur *r, uint64_t n_rows, uint32_t width, const rk_matrix *z, uint64_t &n_seqs) {
    if (!r || r->coupled > 1) return rk_fail(ctx, RK_ERR_INVALID_ARG, "recur is null or coupled is neither 0 nor 1");
    if (r->bias && (r->param_type > RK_F16 || ((uintptr_t)r->bias & (r->param_type == RK_F32 ? 3u : 1u))))
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "bias misaligned or of no known type");
    if (r->offsets && (((uintptr_t)r->offsets & 3u) || r->seq_rows)) return rk_fail(ctx, RK_ERR_INVALID_ARG, "offsets misaligned, or seq_rows beside them");
    if (!r->offsets && r->n_seqs) return rk_fail(ctx, RK_ERR_INVALID_ARG, "n_seqs without offsets");
    if (width < 1) return rk_fail(ctx, RK_ERR_INVALID_ARG, "rows have no elements");
    if (width > RK_RECUR_MAX_WIDTH || n_rows > 0x7FFFFFFFull || r->n_seqs > 0x7FFFFFFEu)
        return rk_fail(ctx, RK_ERR_UNSUPPORTED, "more than 2^31 - 1 rows or sequences, or more than %u columns", RK_RECUR_MAX_WIDTH);
    if (!rk_matrix_ok(z, n_rows, width)) return rk_fail(ctx, RK_ERR_INVALID_ARG, "z null, misaligned or of a stride below the width");
    n_seqs = r->offsets ? r->n_seqs : r->seq_rows ? (n_rows + r->seq_rows - 1) / r->seq_rows : 1;
    return RK_OK;
}
bool alike(const rk_matrix *m, const rk_matrix *z, uint64_t n_rows, uint32_t width) { return rk_matrix_ok(m, n_rows, width) && m->type == z->type; }
bool state_ok(const rk_matrix *m, uint64_t n_seqs, uint32_t width) { return !m || (rk_matrix_ok(m, n_seqs, width) && m->type == RK_F32); }
void fill_recur(RecurArgs &A, const rk_recur *r, uint64_t n_rows, uint32_t width, uint64_t n_seqs, const rk_matrix *z) {
    A.z = z->data; A.z_st = z->stride;
    A.bias = r->bias; A.bias_type = r->param_type;
    A.offsets = r->offsets;
    A.seq_rows = r->seq_rows && r->seq_rows < n_rows ? r->seq_rows : n_rows;
    A.n_rows = n_rows; A.n_seqs = (uint32_t)n_seqs; A.width = width; A.coupled = r->coupled;
}

}  // namespace

extern "C" int32_t rk_recur_forward(rk_ctx *ctx, const rk_recur *recur, uint64_t n_rows, uint32_t width, const rk_matrix *x,
                                    const rk_matrix *z, const rk_matrix *state_in, const rk_matrix *h, const rk_matrix *state_out) {
    if (!ctx) return RK_ERR_INVALID_ARG;
    uint64_t n_seqs = 0;
    int32_t rc = check_recur(ctx, recur, n_rows, width, z, n_seqs);
    if (rc != RK_OK) return rc;
    if (!alike(x, z, n_rows, width) || !alike(h, z, n_rows, width))
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "x or h null, misaligned, of a stride below the width or of another type than z");
    if (!state_ok(state_in, n_seqs, width) || !state_ok(state_out, n_seqs, width))
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "a state is misaligned, of a stride below the width or not in 32 bits");
    if (n_seqs == 0 || (n_rows == 0 && !state_out)) return RK_OK;
    RK_HIP(ctx, hipSetDevice(ctx->device));
    RecurArgs A{};
    fill_recur(A, recur, n_rows, width, n_seqs, z);
    A.x = x->data; A.x_st = x->stride;
    A.out = h->data; A.o_st = h->stride;
    if (state_in) { A.state_in = (const float *)state_in->data; A.si_st = state_in->stride; }
    if (state_out) { A.state_out = (float *)state_out->data; A.so_st = state_out->stride; }
    with_type(z->type, [&](auto t) {
        k_recur_forward<decltype(t)><<<(width + RC_THREADS - 1) / RC_THREADS, RC_THREADS, 0, ctx->stream>>>(A);
    });
    RK_CHECK_LAUNCH(ctx, "k_recur_forward");
    return RK_OK;
}

extern "C" int32_t rk_recur_backward(rk_ctx *ctx, const rk_recur *recur, uint64_t n_rows, uint32_t width, const rk_matrix *x,
                                     const rk_matrix *z, const rk_matrix *h, const rk_matrix *state_in, const rk_matrix *dh,
                                     const rk_matrix *d_state_out, const rk_matrix *dx, const rk_matrix *dz, const rk_matrix *d_state_in,
                                     float *d_bias) {
    if (!ctx) return RK_ERR_INVALID_ARG;
    uint64_t n_seqs = 0;
    int32_t rc = check_recur(ctx, recur, n_rows, width, z, n_seqs);
    if (rc != RK_OK) return rc;
    if ((recur->coupled && !x) || (x && !alike(x, z, n_rows, width)) || !alike(h, z, n_rows, width) || !alike(dh, z, n_rows, width) ||
        !alike(dx, z, n_rows, width) || !alike(dz, z, n_rows, width))
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "a matrix is null, misaligned, of a stride below the width or of another type than z");
    if (!state_ok(state_in, n_seqs, width) || !state_ok(d_state_out, n_seqs, width) || !state_ok(d_state_in, n_seqs, width))
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "a state is misaligned, of a stride below the width or not in 32 bits");
    if (d_bias && (!recur->bias || ((uintptr_t)d_bias & 3u))) return rk_fail(ctx, RK_ERR_INVALID_ARG, "d_bias misaligned, or there is no bias");
    if ((n_seqs == 0 || (n_rows == 0 && !d_state_in)) && !d_bias) return RK_OK;
    RK_HIP(ctx, hipSetDevice(ctx->device));
    RecurArgs A{};
    fill_recur(A, recur, n_rows, width, n_seqs, z);
    if (recur->coupled) { A.x = x->data; A.x_st = x->stride; }
    A.h = h->data; A.h_st = h->stride;
    A.dh = dh->data; A.dh_st = dh->stride;
    A.dx = dx->data; A.dx_st = dx->stride;
    A.dz = dz->data; A.dz_st = dz->stride;
    if (state_in) { A.state_in = (const float *)state_in->data; A.si_st = state_in->stride; }
    if (d_state_out) { A.d_state_out = (const float *)d_state_out->data; A.dso_st = d_state_out->stride; }
    if (d_state_in) { A.d_state_in = (float *)d_state_in->data; A.dsi_st = d_state_in->stride; }
    A.d_bias = d_bias;
    with_type(z->type, [&](auto t) {
        k_recur_backward<decltype(t)><<<(width + RC_THREADS - 1) / RC_THREADS, RC_THREADS, 0, ctx->stream>>>(A);
    });
    RK_CHECK_LAUNCH(ctx, "k_recur_backward");
    return RK_OK;
}
