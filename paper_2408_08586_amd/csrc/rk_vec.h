// What the operators of a training step share: element types, vectors of a row, sums over a wavefront.
#pragma once
#include "rk_internal.h"

// Products and sums of the operators may be fused: each result is compared within a tolerance, none bit for bit.
#pragma clang fp contract(fast)

template <typename T, int N> using Vec = T __attribute__((ext_vector_type(N)));

// N consecutive elements of a row from `p` on, those from `valid` on being zero.  Whole vectors are loaded and stored as
// one whatever their alignment: rows of odd strides stay on the same path, and the memory system takes accesses that are not
// aligned apart by itself.
template <typename T, int N> __device__ __forceinline__ void load_row(const T *__restrict__ p, int32_t valid, float (&v)[N]) {
    typedef Vec<T, N> Any __attribute__((aligned(sizeof(T))));
    if (valid >= N) {
        const Vec<T, N> x = *reinterpret_cast<const Any *>(p);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = (float)x[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = i < valid ? (float)p[i] : 0.f;
    }
}
template <typename T, int N> __device__ __forceinline__ void store_row(T *__restrict__ p, int32_t valid, const float (&v)[N]) {
    typedef Vec<T, N> Any __attribute__((aligned(sizeof(T))));
    if (valid >= N) {
        Vec<T, N> x;
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = (T)v[i];         // to nearest, ties to even
        *reinterpret_cast<Any *>(p) = x;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < valid) p[i] = (T)v[i];
    }
}

// the lanes 32 and 16 apart are reached by swaps of half wavefronts, those of a row by its rotations; every lane ends with the result
__device__ __forceinline__ float swap32(float v, float &other) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    other = __uint_as_float(a[1]);
    return __uint_as_float(a[0]);
}
__device__ __forceinline__ float swap16(float v, float &other) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    other = __uint_as_float(a[1]);
    return __uint_as_float(a[0]);
}
template <int CTRL> __device__ __forceinline__ float dpp_of(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xF, 0xF, false));
}
// row_ror:8, 4, 2, 1
__device__ __forceinline__ float row_sum(float v) {
    v += dpp_of<0x128>(v); v += dpp_of<0x124>(v); v += dpp_of<0x122>(v); v += dpp_of<0x121>(v);
    return v;
}
__device__ __forceinline__ float row_max(float v) {
    v = fmaxf(v, dpp_of<0x128>(v)); v = fmaxf(v, dpp_of<0x124>(v)); v = fmaxf(v, dpp_of<0x122>(v)); v = fmaxf(v, dpp_of<0x121>(v));
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
    float o;
    v = row_sum(v);
    v = swap16(v, o) + o;
    v = swap32(v, o);
    return v + o;
}
__device__ __forceinline__ float wave_max(float v) {
    float o;
    v = row_max(v);
    v = swap16(v, o); v = fmaxf(v, o);
    v = swap32(v, o);
    return fmaxf(v, o);
}

// e^x to about one unit in the last place: the product with log2(e) is carried in two parts, the lower of which enters as its
// first-order factor.  Below 2^-126 zero, also for -inf; NaN stays.
__device__ __forceinline__ float exp_f32(float x) {
    constexpr float L = 1.4426950408889634f, LOW = 1.9259629911e-8f, LN2 = 0.6931471805599453f;
    const float t = x * L;
    const float low = __builtin_fmaf(x, LOW, __builtin_fmaf(x, L, -t));
    const float e = __builtin_amdgcn_exp2f(t);
    return x < -87.4f ? 0.f : __builtin_fmaf(e, low * LN2, e);
}

// host side: a matrix of the operators
static inline bool rk_matrix_ok(const rk_matrix *m, uint64_t n_rows, uint64_t width) {
    if (!m || m->type > RK_F16) return false;
    if (n_rows == 0) return true;
    const uint64_t align = m->type == RK_F32 ? 4 : 2;
    return m->data && ((uintptr_t)m->data & (align - 1)) == 0 && (m->stride >= width || n_rows == 1) && m->stride < (1ull << 40);
}
