// A student's loss against a teacher's largest logits and the labels, and its gradient (rk_distill_loss,
// rk_distill_backward, rk_distill_loss_backward).
#include <cmath>
#include <type_traits>

#include "rk_vec.h"

namespace {

struct DistillArgs {
    const void *student;
    void *d_student;
    uint64_t st, d_st, n_rows, first;   // first: the launch's first row
    uint32_t vocab, top_k, t_type;
    const void *teacher;
    uint64_t t_st;
    const int32_t *index, *label;
    const float *row_weight, *d_total;
    float *loss, *lse, *total;
    float temperature, kd, ce;
    uint32_t slices, slice;             // of a row, where several workgroups share it, and their elements
    float4 *part;                       // [row][slice]: largest logit, sums of the exponentials relative to it
    float4 *cross;                      // [row]: what teacher and label add to the loss; then the row's largest logit and its sums' logarithms
};

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));        // (no quieting before: NaN come out of the sums)
    return r;
}

// a product that is rounded by itself, not fused with what is added to it
__device__ __forceinline__ float times(float a, float b) {
#pragma clang fp contract(off)
    return a * b;
}

// The exponentials of a row: one stream where the two terms of the loss share it (T = 1) or one of them is all there is, two
// streams otherwise, of which the second is the first's square if T = 2.
enum { ONE, TWO, SQUARE };

// A 16-bit student's are taken to base 2, e^(x/T - r) = 2^(x log2(e)/T - r'): one fused product and one instruction.  r' is rounded by up to
// 2^-24 of itself, and the exponent with it: below 2^11 that is 2^-14 at most, an eighth of a float16's half step.  Rows whose largest logit is
// further from zero (all of them masked by a large value, say) and a 32-bit student take differences of logits first, which lose nothing
// (and which the largest of 32-bit logits, beyond HUGE_LOGIT, would overflow while the largest of the row is not known).
constexpr float FUSED_EXPONENT = 2048.f, HUGE_LOGIT = 1e30f;
template <typename T> struct Exp {
    static constexpr bool EXACT = sizeof(T) == 4;
    static __device__ __forceinline__ float of(float x) { return EXACT ? exp_f32(x) : __builtin_amdgcn_exp2f(x); }
    static __device__ __forceinline__ float log(float x) { return EXACT ? logf(x) : __builtin_amdgcn_logf(x); }
    static __device__ __forceinline__ float unit() { return EXACT ? 1.f : 1.4426950408889634f; }
    static __device__ __forceinline__ float natural(float x) { return EXACT ? x : x * 0.6931471805599453f; }
};
// what a logit is multiplied by, the first also without the base; the largest that goes the short way
struct Streams {
    float ka, kb, inv_a, most;
    __device__ __forceinline__ bool huge(float top) const { return fabsf(top) > most && top != -INFINITY; }
};
template <typename T, int SUMS> __device__ __forceinline__ Streams streams_of(const DistillArgs &A) {
    const float inv = A.kd > 0.f ? 1.f / A.temperature : 1.f, ka = inv * Exp<T>::unit(), kb = Exp<T>::unit();
    return Streams{ka, kb, inv, Exp<T>::EXACT ? HUGE_LOGIT : FUSED_EXPONENT / (SUMS == ONE ? ka : fmaxf(ka, kb))};
}

// the sums of a stretch of logits, relative to the largest of them seen so far
template <typename T, int SUMS> struct Running {
    float m = -INFINITY, ref = 0.f, ra = 0.f, rb = 0.f, sa = 0.f, sb = 0.f;     // (nothing above -inf yet: relative to 0)
    __device__ __forceinline__ void rebase(const Streams &S, float top) {
        const float r = fminf(fmaxf(top, -S.most), S.most);     // (a part that is huge: of a row that is not, its sums count from -most; a row that is takes sum_huge)
        if (m != -INFINITY) {
            const float f = Exp<T>::of((ref - r) * S.ka);
            sa *= f;
            if constexpr (SUMS == TWO) sb *= Exp<T>::of((ref - r) * S.kb);
            if constexpr (SUMS == SQUARE) sb *= f * f;
        }
        ref = r; ra = r * S.ka; rb = r * S.kb;
    }
    __device__ __forceinline__ void add(const Streams &S, float x) {
        const float d = x - ref;
        const float e = Exp<T>::of(Exp<T>::EXACT ? d * S.ka : __builtin_fmaf(x, S.ka, -ra));
        sa += e;
        if constexpr (SUMS == TWO) sb += Exp<T>::of(Exp<T>::EXACT ? d * S.kb : __builtin_fmaf(x, S.kb, -rb));
        if constexpr (SUMS == SQUARE) sb += e * e;
    }
    template <int CH> __device__ __forceinline__ void take(const Streams &S, const float (&v)[CH]) {
        float top = v[0];
#pragma unroll
        for (int i = 1; i + 1 < CH; i += 2) top = max3(top, v[i], v[i + 1]);
        top = max3(top, v[CH - 1], m);
        if (top > m) { rebase(S, top); m = top; }
#pragma unroll
        for (int i = 0; i < CH; ++i) add(S, v[i]);
    }
    // relative to the largest of all; a thread that saw nothing has zeros
    __device__ __forceinline__ void move(const Streams &S, float top) {
        if (m != -INFINITY) rebase(S, top);
    }
};

// Calls f(first, words) for a thread's vectors of [begin, end), four of which are under way at once, and tail(place, words) for those of
// the last round; end is the row's end or a multiple of CH.
template <bool CUTS, int THREADS, typename T, int CH, int HINT, typename F, typename G>
__device__ __forceinline__ void stream_row(const Row<T> &row, uint32_t begin, uint32_t end, F f, G tail) {
    constexpr uint32_t U = 4, STEP = THREADS * CH;
    uint32_t base = begin + threadIdx.x * CH, round = begin;
    for (; round + U * STEP <= end; round += U * STEP, base += U * STEP) {
        Words<T, CH> w[U];
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) w[u] = fetch_at<T, CH, HINT>(row, base + u * STEP);
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) f(base + u * STEP, w[u]);
    }
    if (round >= end) return;
    Words<T, CH> w[U];
    Place p[U];
#pragma unroll
    for (uint32_t u = 0; u < U; ++u) {
        p[u] = Place(base + u * STEP, end, CH);
        w[u] = fetch_row<CUTS, T, CH, HINT>(row, p[u]);
    }
#pragma unroll
    for (uint32_t u = 0; u < U; ++u)
        if (round + u * STEP < end) tail(p[u], w[u]);
}
template <bool CUTS, int THREADS, typename T, int CH, int SUMS>
__device__ __forceinline__ void sum_row(const Row<T> &row, uint32_t begin, uint32_t end, const Streams &S, Running<T, SUMS> &R) {
    stream_row<CUTS, THREADS, T, CH, KEEP>(row, begin, end,
        [&](uint32_t, const Words<T, CH> &w) {
            float v[CH];
#pragma unroll
            for (int i = 0; i < CH; ++i) v[i] = element<T>(w, i);
            R.take(S, v);
        },
        [&](const Place &p, const Words<T, CH> &w) {
            float v[CH];
#pragma unroll
            for (int i = 0; i < CH; ++i) v[i] = i < p.valid ? element<T>(w, i) : -INFINITY;
            R.take(S, v);
        });
}

// the same of a stretch whose largest logit is huge, in differences from it
template <bool CUTS, int THREADS, typename T, int CH, int SUMS>
__device__ __forceinline__ void sum_huge(const Row<T> &row, uint32_t begin, uint32_t end, const Streams &S, float top, Running<T, SUMS> &R) {
    R.sa = 0.f; R.sb = 0.f;
    for (uint32_t c = begin + threadIdx.x * CH; c < end; c += THREADS * CH) {
        const Place p(c, end, CH);
        float v[CH];
        load_row<CUTS, T, CH>(row, p, v);
        for (int i = 0; i < CH; ++i) {
            if (i >= p.valid) continue;
            const float d = v[i] - top, e = Exp<T>::of(d * S.ka);
            R.sa += e;
            if constexpr (SUMS == TWO) R.sb += Exp<T>::of(d * S.kb);
            if constexpr (SUMS == SQUARE) R.sb += e * e;
        }
    }
}

// What a row's teacher and label say: a thread holds kept logits tid, tid + THREADS, ...
template <int THREADS, int MOST = (int)RK_MAX_TEACHER_LOGITS> struct Wanted {
    static constexpr int N = MOST / THREADS;
    int32_t at[N], label;
    float t[N], s[N], label_s;
    // what teacher and label name; then, when that is there, the student's logits at their places.  Loads return in their order: what is
    // asked for between the two calls does not wait for the first, nor the second's answers hold it up.
    __device__ __forceinline__ void ask(const DistillArgs &A, uint64_t r) {
        label = A.ce > 0.f ? A.label[r] : -1;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const uint32_t k = threadIdx.x + n * THREADS;
            at[n] = -1; t[n] = -INFINITY;
            if (A.kd > 0.f && k < A.top_k) {
                const uint64_t p = r * A.t_st + k;
                at[n] = A.index[r * A.top_k + k];
                t[n] = A.t_type == RK_F32 ? ((const float *)A.teacher)[p] : A.t_type == RK_BF16 ? (float)((const __bf16 *)A.teacher)[p] : (float)((const _Float16 *)A.teacher)[p];
            }
        }
    }
    // Logits are looked up in [begin, end) only, where they are wanted for what is written there: others may be gradients by now.
    template <typename T> __device__ __forceinline__ void look(const DistillArgs &A, uint64_t r, uint32_t begin, uint32_t end) {
        const T *const row = (const T *)A.student + r * A.st;
        if ((uint32_t)label >= A.vocab) label = -1;
        auto logit = [&](int32_t i) { return (uint32_t)i >= begin && (uint32_t)i < end ? (float)row[i] : 0.f; };
        label_s = logit(label);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            at[n] = (uint32_t)at[n] < A.vocab && t[n] != -INFINITY ? at[n] : -1;
            if (at[n] < 0) t[n] = -INFINITY;
            s[n] = logit(at[n]);
        }
    }
    __device__ __forceinline__ float top() const {
        float m = t[0];
#pragma unroll
        for (int n = 1; n < N; ++n) m = fmaxf(m, t[n]);
        return m;
    }
    // t becomes e^((t - top) / T) (0 where nothing is kept); sum and cross are the thread's parts of sum e and sum e ((t - s - top) / T)
    __device__ __forceinline__ void weigh(const DistillArgs &A, float top, float &sum, float &cross) {
        const float inv = 1.f / A.temperature;
        sum = 0.f; cross = 0.f;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const float x = (t[n] - top) * inv, e = at[n] >= 0 ? exp_f32(x) : 0.f;
            t[n] = e;
            sum += e;
            if (e != 0.f) cross += e * (x - s[n] * inv);
        }
    }
};

// sums (or maxima) over a workgroup, two barriers
template <int WAVES, bool MAX> __device__ __forceinline__ void block_all(float4 &v, float4 *lds) {
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    auto one = [](float x) { return MAX ? wave_max(x) : wave_sum(x); };
    v = make_float4(one(v.x), one(v.y), one(v.z), one(v.w));
    __syncthreads();
    if (lane == 0) lds[wave] = v;
    __syncthreads();
    const float none = MAX ? -INFINITY : 0.f;
    const float4 o = (lane & 15u) < (uint32_t)WAVES ? lds[lane & 15u] : make_float4(none, none, none, none);
    auto row = [](float x) { return MAX ? row_max(x) : row_sum(x); };
    v = make_float4(row(o.x), row(o.y), row(o.z), row(o.w));
}

// d s of a logit.  The streams' exponentials are e^(k (s - top) - l) in the streams' units, top the row's largest logit and l the
// logarithms of the sums relative to it; or, from the log sums, e^(s / T - lse_T) and e^(s - lse_1): each stream from its own, since what
// lse_T T has beyond the largest logit grows with T and would take the second stream's digits.  EITHER: which of them is known at the call.
template <typename T, int SUMS, bool EITHER> struct Slope {
    float ka, kb, ba, bb, ca, cb;       // fused: e^(ka s - ba), e^(kb s - bb)
    float pre, pa, a, la, b, lb;        // from differences: e^(pa (pre s - a) - la), e^(kb (s - b) - lb)
    float ft, f1;                       // of a kept logit's share, of the label
    bool apart;                         // a 16-bit student's exponents are too large for one fused product
    __device__ __forceinline__ Slope(const DistillArgs &A, const Streams &S, float weight, bool kept, bool labelled) : ka(S.ka), kb(S.kb) {
        const float scale = weight * (A.d_total ? A.d_total[0] : 1.f);
        ft = kept ? scale * A.kd * A.temperature : 0.f;
        f1 = labelled ? scale * A.ce : 0.f;
        // (a stream that both terms share, or that is the only term's)
        ca = SUMS == ONE ? ft + f1 : ft;
    }
    __device__ __forceinline__ void from_sums(const Streams &S, float top, float la_, float lb_) {
        pre = 1.f; pa = ka;
        a = b = top; la = la_; lb = lb_;
        ba = top * ka + la; bb = top * kb + lb;
        cb = SUMS == SQUARE ? f1 * Exp<T>::of(la + la - lb) : f1;
        apart = S.huge(top);
    }
    __device__ __forceinline__ void from_lse(const Streams &S, float lse_a, float lse_b) {
        static_assert(EITHER, "");
        pre = S.inv_a; pa = kb;
        a = lse_a; b = lse_b; la = lb = 0.f;
        ba = lse_a * kb; bb = lse_b * kb;
        cb = SUMS == SQUARE ? f1 * Exp<T>::of((lse_a + lse_a - lse_b) * kb) : f1;
        apart = !Exp<T>::EXACT && fmaxf(fabsf(ba), SUMS == ONE ? 0.f : fabsf(bb)) > FUSED_EXPONENT;
    }
    template <bool APART> __device__ __forceinline__ float of(float x) const {
        // (the product with 1 / T is rounded as that of the largest logit in its log sum: no probability is beyond one)
        const float e = Exp<T>::of(!APART ? __builtin_fmaf(x, ka, -ba) : __builtin_fmaf((EITHER ? times(x, pre) : x) - a, EITHER ? pa : ka, -la));
        if constexpr (SUMS == ONE) return ca * e;
        if constexpr (SUMS == SQUARE && !APART) return e * (ca + cb * e);
        return ft * e + f1 * Exp<T>::of(!APART ? __builtin_fmaf(x, kb, -bb) : __builtin_fmaf(x - b, kb, -lb));
    }
    __device__ __forceinline__ float operator()(float x) const { return of<Exp<T>::EXACT>(x); }
};
// The teacher's shares q of the kept logits, by their places, for all threads; then t becomes what those of the same place have
// together (indices may repeat), and label_q what those at the label have, in its thread.
template <int MOST> struct Shares { float4 q[MOST / 4]; int4 at[MOST / 4]; };
template <int THREADS, int MOST> __device__ __forceinline__ float share_wanted(const DistillArgs &A, Wanted<THREADS, MOST> &W, float t_sum, Shares<MOST> &lds) {
    const float inv_sum = t_sum != 0.f ? 1.f / t_sum : 0.f;
    const uint32_t K = A.kd > 0.f ? A.top_k : 0u;
#pragma unroll
    for (int n = 0; n < Wanted<THREADS, MOST>::N; ++n) {
        const uint32_t k = threadIdx.x + n * THREADS;
        if (k < ((K + 3u) & ~3u)) {                     // (behind the last one there is none: at is -1)
            ((float *)lds.q)[k] = W.t[n] * inv_sum;
            ((int32_t *)lds.at)[k] = W.at[n];
        }
    }
    __syncthreads();                    // d_student may be student: what is needed of other places has been read
    auto together = [&](int32_t i) {
        float mass = 0.f;
#pragma unroll 4
        for (uint32_t k = 0; k < (K + 3u) / 4u; ++k) {
            const float4 q = lds.q[k];
            const int4 at = lds.at[k];
            mass += (at.x == i ? q.x : 0.f) + (at.y == i ? q.y : 0.f) + (at.z == i ? q.z : 0.f) + (at.w == i ? q.w : 0.f);
        }
        return mass;
    };
#pragma unroll
    for (int n = 0; n < Wanted<THREADS, MOST>::N; ++n)
        if (W.at[n] >= 0) W.t[n] = together(W.at[n]);
    return threadIdx.x == THREADS - 1 && W.label >= 0 ? together(W.label) : 0.f;
}
// where teacher or label have something in [begin, end): the whole value, once more (equal indices get equal values)
template <int THREADS, int MOST, typename T, int SUMS, bool EITHER>
__device__ __forceinline__ void write_wanted(const Wanted<THREADS, MOST> &W, const Slope<T, SUMS, EITHER> &slope, T *out, uint32_t begin, uint32_t end, float label_q) {
    auto again = [&](int32_t i, float s, float mass) {
        if ((uint32_t)i < begin || (uint32_t)i >= end) return;
        out[i] = (T)((slope.apart ? slope.template of<true>(s) : slope(s)) - slope.ft * mass - (i == W.label ? slope.f1 : 0.f));
    };
#pragma unroll
    for (int n = 0; n < Wanted<THREADS, MOST>::N; ++n)
        if (W.at[n] >= 0) again(W.at[n], W.s[n], W.t[n]);
    if (threadIdx.x == THREADS - 1 && W.label >= 0) again(W.label, W.label_s, label_q);
}
template <bool CUTS, int THREADS, typename T, int CH, int SUMS, bool EITHER>
__device__ __forceinline__ void write_huge(const Row<T> &from, const Row<T> &to, uint32_t begin, uint32_t end, const Slope<T, SUMS, EITHER> &slope) {
    for (uint32_t c = begin + threadIdx.x * CH; c < end; c += THREADS * CH) {
        const Place p(c, end, CH);
        float v[CH];
        load_row<CUTS, T, CH>(from, p, v);
#pragma unroll
        for (int i = 0; i < CH; ++i) v[i] = slope.template of<true>(v[i]);
        store_row<CUTS, T, CH>(to, p, v);
    }
}
template <bool CUTS, int THREADS, typename T, int CH, int SUMS>
__device__ __forceinline__ void write_gradient(const DistillArgs &A, const Row<T> &from, const Row<T> &to, T *out, uint32_t begin, uint32_t end, const Slope<T, SUMS, true> &slope,
                                               Wanted<THREADS> &W, float t_sum, Shares<(int)RK_MAX_TEACHER_LOGITS> &lds) {
    const float label_q = share_wanted(A, W, t_sum, lds);
    if (slope.apart) write_huge<CUTS, THREADS, T, CH>(from, to, begin, end, slope);
    else stream_row<CUTS, THREADS, T, CH, STREAM>(from, begin, end,
        [&](uint32_t first, const Words<T, CH> &w) {
            float v[CH];
#pragma unroll
            for (int i = 0; i < CH; ++i) v[i] = slope(element<T>(w, i));
            store_at<T, CH, STREAM>(to, first, words_of<T, CH>(v));
        },
        [&](const Place &p, const Words<T, CH> &w) {
            float v[CH];
#pragma unroll
            for (int i = 0; i < CH; ++i) v[i] = slope(element<T>(w, i));
            store_row<CUTS, T, CH, STREAM>(to, p, v);
        });
    __syncthreads();
    write_wanted(W, slope, out, begin, end, label_q);
}
template <bool CUTS, int THREADS, typename T, int CH> __device__ __forceinline__ void write_zeros(const Row<T> &to, uint32_t begin, uint32_t end) {
    const float zero[CH] = {};
    for (uint32_t c = begin + threadIdx.x * CH; c < end; c += THREADS * CH) store_row<CUTS, T, CH, STREAM>(to, Place(c, end, CH), zero);
}

// a row's loss and log sums from the joined sums; cross: teacher's cross term and sum, the label's logit and whether there is one
struct RowLoss { float loss, lse_a, lse_b, la, lb; bool left; };
template <typename T, int SUMS> __device__ __forceinline__ RowLoss row_loss(const DistillArgs &A, const Streams &S, float top, float sa, float sb, float4 cross) {
    if (top == -INFINITY && sa == 0.f) return RowLoss{0.f, -INFINITY, -INFINITY, 0.f, 0.f, true};
    RowLoss L;
    L.left = false;
    L.la = Exp<T>::log(sa);
    L.lb = SUMS == ONE ? L.la : Exp<T>::log(sb);
    L.lse_a = times(top, S.inv_a) + Exp<T>::natural(L.la);
    L.lse_b = SUMS == ONE ? L.lse_a : top + Exp<T>::natural(L.lb);
    L.loss = 0.f;
    if (A.kd > 0.f && cross.y != 0.f) L.loss = A.kd * A.temperature * A.temperature * (cross.x / cross.y - logf(cross.y) + L.lse_a);
    if (A.ce > 0.f && cross.w != 0.f) L.loss += A.ce * (L.lse_b - cross.z);
    return L;
}
__device__ __forceinline__ void keep_row(const DistillArgs &A, uint64_t r, const RowLoss &L) {
    A.loss[r] = L.loss;
    A.lse[2 * r] = A.kd > 0.f ? L.lse_a : 0.f;
    A.lse[2 * r + 1] = A.ce > 0.f ? L.lse_b : 0.f;
}

// A workgroup a row: its sums, its loss and, if there is a d_student, its gradient.  Of what a thread reads, its first NR vectors stay in
// registers and its next NL in LDS until then; only what is beyond them is read again.  Bound by HBM: 2048 x 128000 bfloat16, T = 2, both terms, 207 us,
// 1.0 GB that has to move (a tenth of the rows has no weight and is only written), 1.2 GB that does (nine of sixteen vectors a thread are read twice), 5.9 TB/s; 1024 x 32000 float32 52 us, 262 MB, 5.0 TB/s.
// Short rows, of which several fit a compute unit, have registers for eight vectors at five wavefronts a SIMD (at eight: 4096 x 32000 losses
// 74 us, now 51).
template <bool CUTS, int THREADS, int NR, int NL, int MOST, typename T, int CH, int SUMS>
__global__ __launch_bounds__(THREADS, NL > 0 ? 8 : 5) void k_distill_rows(DistillArgs A) {
    extern __shared__ float4 kept_lds[];
    __shared__ float4 red[16];
    __shared__ Shares<MOST> lds;
    constexpr uint32_t STEP = THREADS * CH, MORE = 4;              // vectors under way at once of what is beyond
    const uint64_t r = A.first + blockIdx.x;
    const Row<T> from(A.student, r, A.st, A.vocab), to(A.d_student, r, A.d_st, A.vocab);
    const float weight = A.row_weight ? A.row_weight[r] : 1.f;
    Wanted<THREADS, MOST> W;
    // whole rounds of vectors, and one that the row's end cuts off
    const uint32_t whole = A.vocab / STEP, first = threadIdx.x * CH;
    const Place last(first + whole * STEP, A.vocab, CH);
    auto fetch = [&](uint32_t k, auto hint) {
        constexpr int HINT = decltype(hint)::value;
        return k < whole ? fetch_at<T, CH, HINT>(from, first + k * STEP) : fetch_row<CUTS, T, CH, HINT>(from, last);
    };
    const auto keep = std::integral_constant<int, KEEP>();
    const auto stream = std::integral_constant<int, STREAM>();
    Words<T, CH> w[NR];
    auto begin = [&] {
        W.ask(A, r);
#pragma unroll
        for (int k = 0; k < NR; ++k)
            if ((uint32_t)k <= whole) w[k] = fetch(k, stream);
    };
    if (NL == 0) begin();                   // (a short row is fetched before its weight is there)
    if (weight == 0.f) {
        if (threadIdx.x == 0) { A.loss[r] = 0.f; A.lse[2 * r] = 0.f; A.lse[2 * r + 1] = 0.f; }
        write_zeros<CUTS, THREADS, T, CH>(to, 0, A.vocab);          // (nothing, if there is no d_student)
        return;
    }
    if (NL > 0) begin();
    W.template look<T>(A, r, 0, A.vocab);
    const Streams S = streams_of<T, SUMS>(A);
    Running<T, SUMS> R;
    auto take = [&](uint32_t k, const Words<T, CH> &x) {
        float v[CH];
        if (k < whole) {
#pragma unroll
            for (int i = 0; i < CH; ++i) v[i] = element<T>(x, i);
        } else {
#pragma unroll
            for (int i = 0; i < CH; ++i) v[i] = i < last.valid ? element<T>(x, i) : -INFINITY;
        }
        R.take(S, v);
    };
    constexpr uint32_t W4 = CH * (int)sizeof(T) / 16;
    static_assert(W4 == 1, "a vector is 16 bytes");
#pragma unroll
    for (int k = 0; k < NR; ++k)
        if ((uint32_t)k <= whole) take(k, w[k]);
    if constexpr (NL > 0) {
        Words<T, CH> x[NL];
#pragma unroll
        for (int k = 0; k < NL; ++k)
            if (NR + (uint32_t)k <= whole) x[k] = fetch(NR + k, stream);
#pragma unroll
        for (int k = 0; k < NL; ++k) {
            if (NR + (uint32_t)k > whole) continue;
            if (A.d_student) kept_lds[k * THREADS + threadIdx.x] = __builtin_bit_cast(float4, x[k]);
            take(NR + k, x[k]);
        }
        for (uint32_t k = NR + NL; k <= whole; k += MORE) {
            Words<T, CH> y[MORE];
#pragma unroll
            for (uint32_t u = 0; u < MORE; ++u)
                if (k + u <= whole) y[u] = fetch(k + u, keep);
#pragma unroll
            for (uint32_t u = 0; u < MORE; ++u)
                if (k + u <= whole) take(k + u, y[u]);
        }
    }
    float4 v = make_float4(R.m, W.top(), -INFINITY, -INFINITY);
    block_all<THREADS / 64, true>(v, red);
    const float top = v.x;
    R.move(S, top);
    if (S.huge(top)) sum_huge<CUTS, THREADS, T, CH, SUMS>(from, 0, A.vocab, S, top, R);
    float sum, cross;
    W.weigh(A, v.y, sum, cross);
    v = make_float4(R.sa, R.sb, sum, cross);
    block_all<THREADS / 64, false>(v, red);
    const RowLoss L = row_loss<T, SUMS>(A, S, top, v.x, v.y, make_float4(v.w, v.z, W.label_s, W.label >= 0 ? 1.f : 0.f));
    if (threadIdx.x == 0) keep_row(A, r, L);
    if (!A.d_student) return;
    // (without a kept logit and a label there is no term, whatever the logits hold)
    if (L.left || (v.z == 0.f && W.label < 0)) {
        write_zeros<CUTS, THREADS, T, CH>(to, 0, A.vocab);
        return;
    }
    Slope<T, SUMS, false> slope(A, S, weight, v.z != 0.f, W.label >= 0);
    slope.from_sums(S, top, L.la, L.lb);
    const float label_q = share_wanted(A, W, v.z, lds);
    if (slope.apart) {
        write_huge<CUTS, THREADS, T, CH>(from, to, 0, A.vocab, slope);
    } else {
        auto give = [&](uint32_t k, const Words<T, CH> &x) {
            float g[CH];
#pragma unroll
            for (int i = 0; i < CH; ++i) g[i] = slope(element<T>(x, i));
            if (k < whole) store_at<T, CH, STREAM>(to, first + k * STEP, words_of<T, CH>(g));
            else store_row<CUTS, T, CH, STREAM>(to, last, g);
        };
        if constexpr (NL > 0)
            for (uint32_t k = NR + NL; k <= whole; k += MORE) {
                Words<T, CH> y[MORE];
#pragma unroll
                for (uint32_t u = 0; u < MORE; ++u)
                    if (k + u <= whole) y[u] = fetch(k + u, stream);
#pragma unroll
                for (uint32_t u = 0; u < MORE; ++u)
                    if (k + u <= whole) give(k + u, y[u]);
            }
#pragma unroll
        for (int k = 0; k < NR; ++k)
            if ((uint32_t)k <= whole) give(k, w[k]);
        if constexpr (NL > 0)
#pragma unroll
            for (int k = 0; k < NL; ++k)
                if (NR + (uint32_t)k <= whole) give(NR + k, __builtin_bit_cast(Vec<uint32_t, 4>, kept_lds[k * THREADS + threadIdx.x]));
    }
    __syncthreads();
    write_wanted(W, slope, (T *)A.d_student + r * A.d_st, 0, A.vocab, label_q);
}

// The sums of a slice of a row, for k_distill_join; the first slice's workgroup also looks up what teacher and label want.  For few rows:
// 5 x 128000 4.8 us, then 2.3 in the join, both bound by latency.
template <bool CUTS, int THREADS, typename T, int CH, int SUMS>
__global__ __launch_bounds__(THREADS) void k_distill_part(DistillArgs A) {
    __shared__ float4 red[16];
    const uint64_t r = blockIdx.x / A.slices;
    const uint32_t slice = blockIdx.x - (uint32_t)r * A.slices, begin = slice * A.slice;
    const uint32_t end = slice + 1 == A.slices ? A.vocab : begin + A.slice;
    if (A.row_weight && A.row_weight[r] == 0.f) return;
    const Row<T> from(A.student, r, A.st, A.vocab);
    Wanted<THREADS> W;
    W.at[0] = -1; W.t[0] = -INFINITY;
    if (slice == 0) { W.ask(A, r); W.template look<T>(A, r, 0, A.vocab); }
    const Streams S = streams_of<T, SUMS>(A);
    Running<T, SUMS> R;
    sum_row<CUTS, THREADS, T, CH, SUMS>(from, begin, end, S, R);
    float4 v = make_float4(R.m, slice == 0 ? W.top() : -INFINITY, -INFINITY, -INFINITY);
    block_all<THREADS / 64, true>(v, red);
    const float top = v.x;
    R.move(S, top);
    if (S.huge(top)) sum_huge<CUTS, THREADS, T, CH, SUMS>(from, begin, end, S, top, R);
    float sum = 0.f, cross = 0.f;
    if (slice == 0) W.weigh(A, v.y, sum, cross);
    v = make_float4(R.sa, R.sb, sum, cross);
    block_all<THREADS / 64, false>(v, red);
    if (threadIdx.x) return;
    A.part[r * A.slices + slice] = make_float4(top, v.x, v.y, 0.f);
    if (slice == 0) A.cross[r] = make_float4(v.w, v.z, W.label_s, W.label >= 0 ? 1.f : 0.f);
}

// The slices of the rows joined, a wavefront a row (at most 64 slices); one workgroup also adds the rows' losses up, in one order.
constexpr int JOIN_WAVES = 16;
template <typename T, int SUMS> __global__ __launch_bounds__(64 * JOIN_WAVES) void k_distill_join(DistillArgs A) {
    __shared__ double lds[JOIN_WAVES];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const Streams S = streams_of<T, SUMS>(A);
    double total = 0.0;
    for (uint64_t r = (uint64_t)blockIdx.x * JOIN_WAVES + wave; r < A.n_rows; r += (uint64_t)gridDim.x * JOIN_WAVES) {
        const float weight = A.row_weight ? A.row_weight[r] : 1.f;
        const float4 p = lane < A.slices ? A.part[r * A.slices + lane] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
        const float4 cross = A.cross[r];
        if (weight == 0.f) {
            if (lane == 0) { A.loss[r] = 0.f; A.lse[2 * r] = 0.f; A.lse[2 * r + 1] = 0.f; }
            continue;
        }
        const float top = wave_max(p.x);
        const bool some = p.x != -INFINITY;
        const float d = p.x - top, f = Exp<T>::of(d * S.ka);
        const float sa = some ? p.y * f : p.y, sb = some ? p.z * (SUMS == SQUARE ? f * f : Exp<T>::of(d * S.kb)) : p.z;
        const RowLoss L = row_loss<T, SUMS>(A, S, top, wave_sum(sa), wave_sum(sb), cross);
        if (lane == 0) {
            keep_row(A, r, L);
            if (A.d_student) A.cross[r] = make_float4(top, L.la, L.lb, 0.f);    // (the gradient of these very sums follows)
        }
        total += (double)weight * (double)L.loss;
    }
    if (gridDim.x > 1) return;
    if (lane == 0) lds[wave] = total;
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 1; w < JOIN_WAVES; ++w) total += lds[w];
    A.total[0] = (float)total;
}

// The gradient of a slice of a row (or of all of it) from the row's log sums.  Bound by HBM: 777 x 50021 float16 31 us, 141 MB (a quarter
// of the rows has no weight and is only written), 4.6 TB/s.
template <bool CUTS, int THREADS, typename T, int CH, int SUMS>
__global__ __launch_bounds__(THREADS) void k_distill_gradient(DistillArgs A) {
    __shared__ float4 red[16];
    __shared__ Shares<(int)RK_MAX_TEACHER_LOGITS> lds;
    const uint64_t r = A.first + blockIdx.x / A.slices;
    const uint32_t slice = blockIdx.x % A.slices, begin = slice * A.slice;
    const uint32_t end = slice + 1 == A.slices ? A.vocab : begin + A.slice;
    const Row<T> from(A.student, r, A.st, A.vocab), to(A.d_student, r, A.d_st, A.vocab);
    const float weight = A.row_weight ? A.row_weight[r] : 1.f;
    const float la = A.lse[2 * r + (A.kd > 0.f ? 0 : 1)], lb = A.lse[2 * r + 1];
    if (weight == 0.f || la == -INFINITY) {
        write_zeros<CUTS, THREADS, T, CH>(to, begin, end);
        return;
    }
    Wanted<THREADS> W;
    W.ask(A, r);
    W.template look<T>(A, r, begin, end);
    float4 v = make_float4(W.top(), -INFINITY, -INFINITY, -INFINITY);
    float sum = 0.f, cross = 0.f;
    if (A.kd > 0.f) {
        block_all<THREADS / 64, true>(v, red);
        W.weigh(A, v.x, sum, cross);
        v = make_float4(sum, 0.f, 0.f, 0.f);
        block_all<THREADS / 64, false>(v, red);
        sum = v.x;
    }
    if (sum == 0.f && W.label < 0) {
        write_zeros<CUTS, THREADS, T, CH>(to, begin, end);
        return;
    }
    const Streams S = streams_of<T, SUMS>(A);
    Slope<T, SUMS, true> slope(A, S, weight, sum != 0.f, W.label >= 0);
    if (A.cross) slope.from_sums(S, A.cross[r].x, A.cross[r].y, A.cross[r].z);
    else slope.from_lse(S, la, lb);
    write_gradient<CUTS, THREADS, T, CH, SUMS>(A, from, to, (T *)A.d_student + r * A.d_st, begin, end, slope, W, sum, lds);
}

// the rows' losses added up, in one order
constexpr int TOTAL_THREADS = 1024;
__global__ __launch_bounds__(TOTAL_THREADS) void k_distill_total(DistillArgs A) {
    __shared__ double lds[TOTAL_THREADS / 64];
    double s = 0.0;
    for (uint64_t r = threadIdx.x; r < A.n_rows; r += 4 * TOTAL_THREADS) {
        float w[4], l[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {                           // four under way at once
            const uint64_t q = r + TOTAL_THREADS * i < A.n_rows ? r + TOTAL_THREADS * i : r;
            w[i] = A.row_weight ? A.row_weight[q] : 1.f;
            l[i] = A.loss[q];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) s += r + TOTAL_THREADS * i < A.n_rows && w[i] != 0.f ? (double)w[i] * (double)l[i] : 0.0;
    }
#pragma unroll
    for (int off = 32; off; off >>= 1) s += __shfl_xor(s, off, 64);
    if ((threadIdx.x & 63u) == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x) return;
    s = 0.0;
#pragma unroll
    for (int w = 0; w < TOTAL_THREADS / 64; ++w) s += lds[w];
    A.total[0] = (float)s;
}

// ---- host
// Vectors that a thread of a long row keeps in registers and in LDS: 64 KB a workgroup, two of which fit a compute unit, at 64 registers
// a lane.  A fourth in registers goes to scratch memory instead: 2048 x 128000 both at once 211 us with three, 219 with four, 512 x 64000 31 and 35.
constexpr int DS_REGISTERS = 3, DS_LDS = 4;
// Rows that are cut into slices where there are fewer.  Losses (four times as many): 300 x 20000 13.0 us, 500 x 32000 16.6 (cut below 2,048 rows 26.6
// and 44.4; only below 512, 900 x 128000 55 instead of 69).  With the gradient: 5 x 128000 13 us; but above half as many a workgroup a row is faster, 200 x 128000 56 us
// in slices and 30 in rows, 150 x 10000 23 and 9.
constexpr uint64_t DS_FEW = 256;
// Elements up to which 256 threads take a row or slice, beyond 1,024: gradient of 300 x 50000 16.5 us, with half as many elements
// 26, with twice as many the same, but losses of 900 x 128000 57 instead of 69.
constexpr uint32_t DS_SMALL = 16384;

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
enum Step { STEP_ROWS, STEP_PART, STEP_JOIN, STEP_GRADIENT };
template <typename T, int SUMS> hipError_t launch(hipStream_t st, DistillArgs A, Step step) {
    constexpr int CH = sizeof(T) == 4 ? 4 : 8;
    if (step == STEP_JOIN) {
        k_distill_join<T, SUMS><<<A.n_rows < DS_FEW ? 1 : (uint32_t)((A.n_rows + JOIN_WAVES - 1) / JOIN_WAVES), 64 * JOIN_WAVES, 0, st>>>(A);
        return hipSuccess;
    }
    // f(workgroups) for as many rows as a launch holds, `each` workgroups a row
    auto by_rows = [&](uint64_t threads, uint64_t each, auto f) {
        const uint64_t most = RK_LAUNCH_THREADS / (threads * each);
        for (A.first = 0; A.first < A.n_rows; A.first += most) f((uint32_t)((A.n_rows - A.first < most ? A.n_rows - A.first : most) * each));
    };
    auto go = [&](auto cuts, auto threads) {
        constexpr bool CUTS = decltype(cuts)::value;
        constexpr int N = decltype(threads)::value;
        if (step == STEP_PART) k_distill_part<CUTS, N, T, CH, SUMS><<<(uint32_t)(A.n_rows * A.slices), N, 0, st>>>(A);
        else by_rows(N, A.slices, [&](uint32_t blocks) { k_distill_gradient<CUTS, N, T, CH, SUMS><<<blocks, N, 0, st>>>(A); });
    };
    auto rows = [&](auto cuts) {
        constexpr bool CUTS = decltype(cuts)::value;
        const uint32_t vectors = (A.vocab + CH - 1) / CH;
        constexpr int MOST = (int)RK_MAX_TEACHER_LOGITS;
        if (vectors <= 128 * 4 && A.top_k <= 256) by_rows(128, 1, [&](uint32_t n) { k_distill_rows<CUTS, 128, 4, 0, 256, T, CH, SUMS><<<n, 128, 0, st>>>(A); });
        else if (vectors <= 256 * 8) by_rows(256, 1, [&](uint32_t n) { k_distill_rows<CUTS, 256, 8, 0, MOST, T, CH, SUMS><<<n, 256, 0, st>>>(A); });
        else if (vectors <= 512 * 8) by_rows(512, 1, [&](uint32_t n) { k_distill_rows<CUTS, 512, 8, 0, MOST, T, CH, SUMS><<<n, 512, 0, st>>>(A); });
        else {
            const auto kernel = k_distill_rows<CUTS, 1024, DS_REGISTERS, DS_LDS, MOST, T, CH, SUMS>;
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, DS_LDS * 1024 * 16);
            if (e != hipSuccess) return e;
            by_rows(1024, 1, [&](uint32_t n) { kernel<<<n, 1024, DS_LDS * 1024 * 16, st>>>(A); });
        }
        return hipSuccess;
    };
    if (step == STEP_ROWS) return A.vocab % CH ? rows(std::true_type()) : rows(std::false_type());
    auto sized = [&](auto cuts) {
        if (A.slice <= DS_SMALL) go(cuts, std::integral_constant<int, 256>());
        else go(cuts, std::integral_constant<int, 1024>());
    };
    if (A.vocab % CH) sized(std::true_type()); else sized(std::false_type());
    return hipSuccess;
}
int32_t send(rk_ctx *ctx, uint32_t type, const DistillArgs &A, Step step) {
    const int sums = A.kd == 0.f || A.ce == 0.f || A.temperature == 1.f ? ONE : A.temperature == 2.f && type != RK_F32 ? SQUARE : TWO;
    auto go = [&](auto t) {
        typedef decltype(t) T;
        if (sums == ONE) return launch<T, ONE>(ctx->stream, A, step);
        if constexpr (sizeof(T) == 2)
            if (sums == SQUARE) return launch<T, SQUARE>(ctx->stream, A, step);
        return launch<T, TWO>(ctx->stream, A, step);
    };
    const hipError_t e = type == RK_F32 ? go(float()) : type == RK_BF16 ? go(__bf16()) : go(_Float16());
    if (e != hipSuccess) return rk_fail(ctx, RK_ERR_DEVICE, "k_distill_rows: %s", hipGetErrorString(e));
    RK_CHECK_LAUNCH(ctx, step == STEP_JOIN ? "k_distill_join" : step == STEP_PART ? "k_distill_part" : step == STEP_GRADIENT ? "k_distill_gradient" : "k_distill_rows");
    return RK_OK;
}
// rows in as many slices as bring `want` workgroups together, of `least` elements at least
void cut_rows(DistillArgs &A, uint64_t want, uint32_t least) {
    uint64_t n = A.n_rows ? want / A.n_rows : 1;
    if (n > A.vocab / least) n = A.vocab / least;
    if (n > 64) n = 64;                                         // k_distill_join: a lane a slice
    if (n < 1) n = 1;
    A.slice = (uint32_t)(((A.vocab + n - 1) / n + 7) / 8 * 8);
    A.slices = (A.vocab + A.slice - 1) / A.slice;
}
int32_t run(rk_ctx *ctx, uint32_t type, DistillArgs &A, bool want_loss, bool want_grad) {
    RK_HIP(ctx, hipSetDevice(ctx->device));
    int32_t rc;
    A.slices = 1; A.slice = A.vocab;
    bool gradient = want_grad && !want_loss;
    if (want_loss && A.n_rows) {
        // Rows that would leave compute units without one are cut into slices: fewer than DS_FEW of them, or, where the loss is all and
        // the slices need no second reading, up to four times as many.  512 workgroups with the gradient: 60 x 32000 17.8 us, 200 x 32000 33.3; 1,024
        // 17.8 and 32.3.  4,096 without: 900 x 128000 69 us, 2,048 59, 8,192 55, others the same.  Slices of at least 4,096 elements with it: 60 x 32000
        // 17.8 us, 2,048 18.5, 8,192 16.5; of 8,192 without: 500 x 32000 16.6 us, 4,096 19.4, 16,384 14.0, but 5 x 128000 6.8, 7.0 and 7.7.
        cut_rows(A, want_grad ? 512 : 4096, want_grad ? 4096 : 8192);
        if (A.slices > 1 && A.n_rows < (want_grad ? DS_FEW : 4 * DS_FEW)) {
            const size_t parts = (size_t)(A.n_rows * A.slices);
            float4 *room;
            if ((rc = rk_scratch(ctx, SL_DISTILL_PARTS, (parts + A.n_rows) * 16, (void **)&room)) != RK_OK) return rc;
            A.part = room; A.cross = room + parts;
            if ((rc = send(ctx, type, A, STEP_PART)) != RK_OK || (rc = send(ctx, type, A, STEP_JOIN)) != RK_OK) return rc;
            gradient = want_grad;
            want_loss = A.n_rows >= DS_FEW;                     // (otherwise the join has the total)
        } else {
            A.slices = 1; A.slice = A.vocab;
            if ((rc = send(ctx, type, A, STEP_ROWS)) != RK_OK) return rc;
        }
    }
    if (gradient && A.n_rows) {
        // (300 x 50000 16.5 us, of 4,096 elements at least 19.4, of 16,384 18.4; 777 x 50000 with 8,192 workgroups 36 instead of 38, 1500 x 32000
        // with 2,048 41 instead of 43)
        cut_rows(A, 4096, 8192);
        if ((rc = send(ctx, type, A, STEP_GRADIENT)) != RK_OK) return rc;
    }
    if (want_loss) {
        k_distill_total<<<1, TOTAL_THREADS, 0, ctx->stream>>>(A);
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
