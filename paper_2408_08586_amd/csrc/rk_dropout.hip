// Dropout whose mask is made from a counter where it is needed (rk_dropout in rubick.h).
//
// A lane takes eight columns of a row, so that one Philox block (ten rounds, twenty 32 x 32 -> 64 bit products) serves it whole: its four words
// are eight 16-bit numbers.  Vectors are numbered through the matrix, row after row, and a workgroup takes a run of them, so that rows of
// any width fill its lanes.  What is dropped is taken out by a selection, not by a product: an infinity or NaN there leaves nothing behind.
//
// 8,192 x 12,288 in bfloat16 with a residual: 87 to 88 us, 6.9 TB/s of 604 MB (a call among others, with other rows in the caches, 100): HBM's rate; the numbers take 0.64 of the vector
// units' cycles beside it.  3,001 x 5,003 from float16 into float32, rows of odd strides: 18 us (90 MB, 5.0 TB/s).
#include "rk_vec.h"

namespace {

constexpr uint32_t DROP_THREADS = 256, DROP_EACH = 2;      // vectors of a lane

struct DropArgs {
    const void *x, *residual;
    void *out;
    uint64_t x_st, r_st, o_st;
    const uint64_t *rng;
    uint64_t n_vectors;
    uint32_t per_row, width;        // vectors of a row
    uint32_t least;                 // 16-bit numbers below it are dropped
    float scale;
};

struct Philox { uint32_t w[4]; };
__device__ __forceinline__ Philox philox(uint32_t c0, uint32_t c1, uint64_t offset, uint64_t seed) {
    uint32_t c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32), k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t p = (uint64_t)c0 * 0xD2511F53u, q = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(q >> 32) ^ c1 ^ k0;
        c2 = (uint32_t)(p >> 32) ^ c3 ^ k1;
        c1 = (uint32_t)q;
        c3 = (uint32_t)p;
        k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
    }
    return Philox{{c0, c1, c2, c3}};
}

// eight elements, `n` of them in the row, of any alignment; what passes once is streamed
template <typename T> __device__ __forceinline__ Words<T, 8> load8(const T *p, uint32_t n) {
    constexpr int PARTS = (int)sizeof(T) / 2;
    Words<T, 8> w = 0u;
    if (n >= 8) {
#pragma unroll
        for (int h = 0; h < PARTS; ++h) {
            const Vec<uint32_t, 4> x = __builtin_nontemporal_load((const Loose<Vec<uint32_t, 4>, T> *)p + h);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[4 * h + i] = x[i];
        }
    } else {
        Vec<T, 8> v = (T)0.f;
#pragma unroll
        for (uint32_t i = 0; i < 7; ++i) if (i < n) v[i] = p[i];
        w = __builtin_bit_cast(Words<T, 8>, v);
    }
    return w;
}
template <typename T> __device__ __forceinline__ void store8(T *p, uint32_t n, const float (&v)[8]) {
    constexpr int PARTS = (int)sizeof(T) / 2;
    const Words<T, 8> w = words_of<T, 8>(v);
    if (n >= 8) {
#pragma unroll
        for (int h = 0; h < PARTS; ++h) {
            Vec<uint32_t, 4> y;
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = w[4 * h + i];
            __builtin_nontemporal_store(y, (Loose<Vec<uint32_t, 4>, T> *)p + h);
        }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 7; ++i) if (i < n) p[i] = (T)v[i];
    }
}

// X: what is dropped from; R: the residual and the result
template <typename X, typename R> __global__ __launch_bounds__(DROP_THREADS) void k_dropout(const DropArgs A) {
    const uint64_t seed = A.rng[0], offset = A.rng[1];
    constexpr uint32_t RUN = DROP_THREADS * DROP_EACH;
    for (uint64_t begin = (uint64_t)blockIdx.x * RUN; begin < A.n_vectors; begin += (uint64_t)gridDim.x * RUN) {
        // the run's first vector by a division that is the same for all lanes, the others from there
        const uint64_t row0 = begin / A.per_row;
        const uint32_t v0 = (uint32_t)(begin - row0 * A.per_row);
        Words<X, 8> x[DROP_EACH];
        Words<R, 8> r[DROP_EACH];
        uint32_t n[DROP_EACH], v[DROP_EACH];
        uint64_t row[DROP_EACH];
#pragma unroll
        for (uint32_t e = 0; e < DROP_EACH; ++e) {
            const uint32_t t = v0 + threadIdx.x + e * DROP_THREADS, q = t / A.per_row;
            row[e] = row0 + q;
            v[e] = t - q * A.per_row;
            n[e] = begin + threadIdx.x + e * DROP_THREADS < A.n_vectors ? A.width - 8 * v[e] : 0;
            x[e] = load8((const X *)A.x + row[e] * A.x_st + 8 * v[e], n[e]);
            r[e] = load8((const R *)A.residual + row[e] * A.r_st + 8 * v[e], A.residual ? n[e] : 0);
        }
#pragma unroll
        for (uint32_t e = 0; e < DROP_EACH; ++e) {
            const Philox p = philox(v[e], (uint32_t)row[e], offset, seed);
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t number = i & 1 ? p.w[i / 2] >> 16 : p.w[i / 2] & 0xFFFFu;
                const float dropped = number >= A.least ? element<X>(x[e], i) * A.scale : 0.f;
                y[i] = A.residual ? element<R>(r[e], i) + dropped : dropped;
            }
            store8((R *)A.out + row[e] * A.o_st + 8 * v[e], n[e], y);
        }
    }
}

template <typename X, typename R> void launch(const DropArgs &A, hipStream_t stream) {
    const uint64_t runs = (A.n_vectors + DROP_THREADS * DROP_EACH - 1) / (DROP_THREADS * DROP_EACH);
    const uint64_t most = RK_LAUNCH_THREADS / DROP_THREADS;
    k_dropout<X, R><<<(uint32_t)(runs < most ? runs : most), DROP_THREADS, 0, stream>>>(A);
}

// in: what is dropped from.  wide: which of the two may be RK_F32 beside a narrow other
int32_t run_dropout(rk_ctx *ctx, const rk_dropout *d, uint64_t n_rows, uint32_t width, const rk_matrix *in, const rk_matrix *residual,
                    const rk_matrix *out, const rk_matrix *wide) {
    if (!ctx) return RK_ERR_INVALID_ARG;
    if (!d || !(d->p >= 0.f) || !(d->p <= 1.f)) return rk_fail(ctx, RK_ERR_INVALID_ARG, "dropout is null or its share is not from 0 to 1");
    if (!d->rng || ((uintptr_t)d->rng & 7u)) return rk_fail(ctx, RK_ERR_INVALID_ARG, "rng is null or misaligned");
    if (width < 1) return rk_fail(ctx, RK_ERR_INVALID_ARG, "rows have no elements");
    if (width > ROW_MAX || n_rows > 0x7FFFFFFFull) return rk_fail(ctx, RK_ERR_UNSUPPORTED, "more than 2^31 - 1 rows or 2^28 columns");
    if (!rk_matrix_ok(in, n_rows, width) || !rk_matrix_ok(out, n_rows, width) || (residual && !rk_matrix_ok(residual, n_rows, width)))
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "a matrix is null, misaligned or of a stride below the width");
    if ((residual && residual->type != out->type) || (in->type != out->type && wide->type != RK_F32))
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "types that do not go together");
    if (n_rows == 0) return RK_OK;
    RK_HIP(ctx, hipSetDevice(ctx->device));
    DropArgs A{};
    A.x = in->data; A.x_st = in->stride;
    if (residual) { A.residual = residual->data; A.r_st = residual->stride; }
    A.out = out->data; A.o_st = out->stride;
    A.rng = d->rng;
    A.width = width; A.per_row = (width + 7) / 8;
    A.n_vectors = n_rows * A.per_row;
    A.least = (uint32_t)floor((double)d->p * 65536.0 + 0.5);
    A.scale = A.least < 65536u ? 65536.f / (float)(65536u - A.least) : 0.f;
    const uint32_t i = in->type, o = out->type;
    if (i == RK_F32) {
        if (o == RK_F32) launch<float, float>(A, ctx->stream);
        else if (o == RK_BF16) launch<float, __bf16>(A, ctx->stream);
        else launch<float, _Float16>(A, ctx->stream);
    } else if (i == RK_BF16) {
        if (o == RK_F32) launch<__bf16, float>(A, ctx->stream); else launch<__bf16, __bf16>(A, ctx->stream);
    } else {
        if (o == RK_F32) launch<_Float16, float>(A, ctx->stream); else launch<_Float16, _Float16>(A, ctx->stream);
    }
    RK_CHECK_LAUNCH(ctx, "k_dropout");
    return RK_OK;
}

}  // namespace

extern "C" int32_t rk_dropout_forward(rk_ctx *ctx, const rk_dropout *dropout, uint64_t n_rows, uint32_t width, const rk_matrix *x,
                                      const rk_matrix *residual, const rk_matrix *out) {
    return run_dropout(ctx, dropout, n_rows, width, x, residual, out, out);
}

extern "C" int32_t rk_dropout_backward(rk_ctx *ctx, const rk_dropout *dropout, uint64_t n_rows, uint32_t width, const rk_matrix *d_out,
                                       const rk_matrix *dx) {
    return run_dropout(ctx, dropout, n_rows, width, d_out, nullptr, dx, d_out);
}
