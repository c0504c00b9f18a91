// What the operators of a training step share: element types, vectors of a row, sums over a wavefront.
#pragma once
#include "rk_internal.h"

// Products and sums of the operators may be fused: each result is compared within a tolerance, none bit for bit.
#pragma clang fp contract(fast)

template <typename T, int N> using Vec = T __attribute__((ext_vector_type(N)));
// N elements of a row as they lie in memory: whole 32-bit words, two narrow elements each (vectors of narrow elements themselves are
// taken apart where paths meet, a register an element)
template <typename T, int N> using Words = Vec<uint32_t, N * (int)sizeof(T) / 4>;

// V where it begins at any element of T.  (As a class's member: an alias template would drop the attribute, which depends on T, and say nothing.)
template <typename V, typename T> struct LooseAs { typedef V type __attribute__((aligned(sizeof(T)))); };
template <typename V, typename T> using Loose = typename LooseAs<V, T>::type;
static_assert(alignof(Loose<Vec<uint32_t, 4>, __bf16>) == 2 && alignof(Loose<Vec<uint32_t, 2>, float>) == 4, "what begins at any element is declared so");

// A row as a buffer that ends with it: what is loaded from behind its end is zero and what is stored there is dropped, by the memory
// system, so that rows of any width take the same instructions; a matrix that is not there is one whose rows have no elements; and a
// lane's place in a row is one register, whatever the matrix.
template <typename T> struct Row {
    __amdgpu_buffer_rsrc_t buf;
    __device__ __forceinline__ Row(const void *base, uint64_t row, uint64_t stride, uint32_t width)
        : buf(__builtin_amdgcn_make_buffer_rsrc(const_cast<T *>((const T *)base + row * stride), 0, (int)(base ? width * (uint32_t)sizeof(T) : 0u), 0x00027000)) {}
};
// A lane's N elements of a row, from element `first` on.  Those that are all inside go as whole vectors, whatever their alignment;
// the one that the row's end cuts goes in the pieces that its length has in base 2 (CUTS: the width is no multiple of N, there is such
// a vector, and it has width % N elements: the same for all rows, so that the pieces' places are known to the scalar unit).
constexpr uint32_t ROW_NOWHERE = 1u << 29, ROW_MAX = 1u << 28;      // elements: behind every row; the widest row
struct Place {
    uint32_t whole, cut;            // where the vector begins, or ROW_NOWHERE
    int32_t valid;
    uint32_t tail;                  // width % n
    bool cut_here;                  // some lane of the wavefront has one that is cut: only these take the long way
    __device__ __forceinline__ Place() {}
    __device__ __forceinline__ Place(uint32_t first, uint32_t width, int n) {
        valid = (int32_t)width - (int32_t)first;
        tail = width % (uint32_t)n;
        whole = valid >= n ? first : ROW_NOWHERE;
        cut = valid > 0 && valid < n ? first : ROW_NOWHERE;
        cut_here = __builtin_amdgcn_ballot_w64(cut != ROW_NOWHERE) != 0;
    }
};
// How long the caches are to keep what passes: STREAM is for what is read or written once (the instructions' non-temporal bit).
enum { KEEP = 0, STREAM = 2 };
template <typename T, int N, int HINT = KEEP> __device__ __forceinline__ Words<T, N> fetch_at(const Row<T> &row, uint32_t first) {
    Words<T, N> w;
    constexpr int PARTS = N * (int)sizeof(T) / 16;
    const uint32_t at = first * (uint32_t)sizeof(T);
#pragma unroll
    for (int h = 0; h < PARTS; ++h) {
        const Vec<uint32_t, 4> x = __builtin_amdgcn_raw_buffer_load_b128(row.buf, at + 16u * h, 0, HINT);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[4 * h + i] = x[i];
    }
    return w;
}
// A vector under way: what is whole, and the pieces of one that is cut, four, two and one element of it.  They become one vector where
// they are wanted (`whole_of`), so that a wavefront with a cut vector does not wait for each as it asks for it.
template <bool CUTS, typename T, int N> struct Held { Words<T, N> w; };
template <typename T, int N> struct Held<true, T, N> {
    Words<T, N> w;
    Vec<uint32_t, 4> four;              // (of narrow elements two words)
    Vec<uint32_t, 2> two;               // (of narrow elements one word)
    uint32_t one;
};
// the pieces beside a vector `w` that has been asked for
template <typename T, int N> __device__ __forceinline__ Held<true, T, N> with_pieces(const Row<T> &row, const Place &p, const Words<T, N> &w) {
    Held<true, T, N> h;
    h.w = w;
    h.four = 0u; h.two = 0u; h.one = 0u;
    if (!p.cut_here) return h;
    const uint32_t from = p.cut * (uint32_t)sizeof(T);
    if constexpr (sizeof(T) == 4) {
        static_assert(N == 4 || N == 8, "");
        if (N == 8 && (p.tail & 4u)) h.four = __builtin_amdgcn_raw_buffer_load_b128(row.buf, from, 0, 0);
        if (p.tail & 2u) h.two = __builtin_amdgcn_raw_buffer_load_b64(row.buf, from + 4u * (N == 8 ? p.tail & 4u : 0u), 0, 0);
        if (p.tail & 1u) h.one = __builtin_amdgcn_raw_buffer_load_b32(row.buf, from + 4u * (p.tail & 6u), 0, 0);
    } else {
        static_assert(N == 8, "");
        if (p.tail & 4u) {
            const Vec<uint32_t, 2> x = __builtin_amdgcn_raw_buffer_load_b64(row.buf, from, 0, 0);
            h.four[0] = x[0]; h.four[1] = x[1];
        }
        if (p.tail & 2u) h.two[0] = __builtin_amdgcn_raw_buffer_load_b32(row.buf, from + 2u * (p.tail & 4u), 0, 0);
        if (p.tail & 1u) h.one = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(row.buf, from + 2u * (p.tail & 6u), 0, 0);
    }
    return h;
}
template <typename T, int N, int HINT = KEEP> __device__ __forceinline__ Held<true, T, N> hold_row(const Row<T> &row, const Place &p) {
    return with_pieces<T, N>(row, p, fetch_at<T, N, HINT>(row, p.whole));
}
template <typename T, int N> __device__ __forceinline__ Words<T, N> whole_of(const Held<false, T, N> &h, const Place &) { return h.w; }
template <typename T, int N> __device__ __forceinline__ Words<T, N> whole_of(const Held<true, T, N> &h, const Place &p) {
    Words<T, N> w = h.w;
    if (!p.cut_here) return w;
    if constexpr (sizeof(T) == 4) {
        const bool behind = N == 8 && (p.tail & 4u);
        if constexpr (N == 8)
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] |= h.four[i];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (N == 8) w[(4 + i) % N] |= behind ? h.two[i] : 0u;
            w[i] |= behind ? 0u : h.two[i];
        }
#pragma unroll
        for (uint32_t i = 0; i < N; i += 2) w[i] |= (p.tail & 6u) == i ? h.one : 0u;
    } else {
        w[0] |= h.four[0]; w[1] |= h.four[1];
        w[0] |= p.tail & 4u ? 0u : h.two[0]; w[2] |= p.tail & 4u ? h.two[0] : 0u;
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) w[i] |= (p.tail & 6u) == 2u * i ? h.one : 0u;
    }
    return w;
}
template <bool CUTS, typename T, int N, int HINT = KEEP> __device__ __forceinline__ Words<T, N> fetch_row(const Row<T> &row, const Place &p) {
    if constexpr (CUTS) return whole_of<T, N>(hold_row<T, N, HINT>(row, p), p);
    else return fetch_at<T, N, HINT>(row, p.whole);
}
// HOLD: the pieces are asked for along with the vector; otherwise where it is wanted (with_pieces)
template <bool HOLD, typename T, int N, int HINT = KEEP> __device__ __forceinline__ Held<HOLD, T, N> held(const Row<T> &row, const Place &p) {
    if constexpr (HOLD) return hold_row<T, N, HINT>(row, p);
    else return Held<false, T, N>{fetch_at<T, N, HINT>(row, p.whole)};
}
template <typename T, int W> __device__ __forceinline__ float element(const Vec<uint32_t, W> &w, int i) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else if constexpr (__is_same(T, __bf16)) return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    else return (float)__builtin_bit_cast(_Float16, (uint16_t)(i & 1 ? w[i / 2] >> 16 : w[i / 2]));
}
template <bool CUTS, typename T, int N, int HINT = KEEP> __device__ __forceinline__ void load_row(const Row<T> &row, const Place &p, float (&v)[N]) {
    const Words<T, N> w = fetch_row<CUTS, T, N, HINT>(row, p);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = element<T>(w, i);
}
template <typename T, int N> __device__ __forceinline__ Words<T, N> words_of(const float (&v)[N]) {
    Vec<T, N> x;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (T)v[i];             // to nearest, ties to even
    return __builtin_bit_cast(Words<T, N>, x);
}
template <typename T, int N, int HINT = KEEP> __device__ __forceinline__ void store_at(const Row<T> &row, uint32_t first, const Words<T, N> &w) {
    constexpr int PARTS = N * (int)sizeof(T) / 16;
    const uint32_t at = first * (uint32_t)sizeof(T);
#pragma unroll
    for (int h = 0; h < PARTS; ++h) {
        Vec<uint32_t, 4> y;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = w[4 * h + i];
        __builtin_amdgcn_raw_buffer_store_b128(y, row.buf, at + 16u * h, 0, HINT);
    }
}
template <bool CUTS, typename T, int N, int HINT = KEEP> __device__ __forceinline__ void store_row(const Row<T> &row, const Place &p, const float (&v)[N]) {
    const Words<T, N> w = words_of<T, N>(v);
    store_at<T, N, HINT>(row, p.whole, w);
    if (CUTS && p.cut_here) {
        const uint32_t from = p.cut * (uint32_t)sizeof(T);
        if constexpr (sizeof(T) == 4) {
            constexpr uint32_t HALF = N / 2;
            uint32_t at = 0;
            if (N == 8 && (p.tail & 4u)) {
                Vec<uint32_t, 4> x;
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = w[i];
                __builtin_amdgcn_raw_buffer_store_b128(x, row.buf, from, 0, 0);
                at = HALF;
            }
            if (p.tail & 2u) {
                Vec<uint32_t, 2> x;
#pragma unroll
                for (uint32_t i = 0; i < 2; ++i) x[i] = at ? w[(HALF + i) % N] : w[i];
                __builtin_amdgcn_raw_buffer_store_b64(x, row.buf, from + 4u * at, 0, 0);
            }
            if (p.tail & 1u) {
                uint32_t x = w[0];
#pragma unroll
                for (uint32_t i = 2; i < N; i += 2) x = (p.tail & 6u) == i ? w[i] : x;
                __builtin_amdgcn_raw_buffer_store_b32(x, row.buf, from + 4u * (p.tail & 6u), 0, 0);
            }
        } else {
            if (p.tail & 4u) {
                Vec<uint32_t, 2> x;
                x[0] = w[0]; x[1] = w[1];
                __builtin_amdgcn_raw_buffer_store_b64(x, row.buf, from, 0, 0);
            }
            if (p.tail & 2u) __builtin_amdgcn_raw_buffer_store_b32(p.tail & 4u ? w[2] : w[0], row.buf, from + 2u * (p.tail & 4u), 0, 0);
            if (p.tail & 1u) {
                uint32_t x = w[0];
#pragma unroll
                for (uint32_t i = 1; i < 4; ++i) x = (p.tail & 6u) == 2u * i ? w[i] : x;
                __builtin_amdgcn_raw_buffer_store_b16((uint16_t)x, row.buf, from + 2u * (p.tail & 6u), 0, 0);
            }
        }
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

// host side: threads of one launch (it has fewer than 2^32); what needs more goes in several
constexpr uint64_t RK_LAUNCH_THREADS = 1ull << 31;
// a matrix of the operators
static inline bool rk_matrix_ok(const rk_matrix *m, uint64_t n_rows, uint64_t width) {
    if (!m || m->type > RK_F16) return false;
    if (n_rows == 0) return true;
    const uint64_t align = m->type == RK_F32 ? 4 : 2;
    return m->data && ((uintptr_t)m->data & (align - 1)) == 0 && (m->stride >= width || n_rows == 1) && m->stride < (1ull << 40);
}
