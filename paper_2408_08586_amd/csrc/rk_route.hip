// The router of a mixture of experts: top-k choice and weights, counts per expert, balance and z loss, and the gradient of the
// logits (rk_route_forward, rk_route_backward).
#include <cmath>
#include <initializer_list>
#include <type_traits>

#include "rk_vec.h"

namespace {

constexpr int RT_THREADS = 512, RT_WAVES = RT_THREADS / 64;

struct RouteArgs {
    const void *logits;
    uint64_t st, n_tokens, group_tokens, n_groups;
    uint32_t n_experts, top_k, renorm;
    const uint8_t *mask;
    int32_t *expert;
    float *weight, *lse;
    uint32_t *counts;
    float *prob_sum;
    uint32_t *tokens;
    float *loss;
    uint64_t chunk, per_group;          // tokens of a workgroup; workgroups of a group
    uint32_t *part_counts;              // [workgroup][expert]
    float *part_probs;
    float2 *part_z;                     // [workgroup]: tokens, sum of lse^2
    float4 *tile_z;                     // [group][tile of experts]: sum of counts * prob_sum, sum of lse^2, tokens
    uint32_t *done;                     // workgroups that have ended; 0 between calls
    uint32_t tiles;
    // backward
    void *d_logits;
    uint64_t d_st;
    const float *d_loss, *d_weight;
};

// ---- A token's logits lie in L lanes next to each other (8, or the 16 of a DPP row), in vectors of four: vector j + L i is the i-th
// of lane j.  A wavefront works on 64 / L tokens at once, and what is summed over a token never leaves its row.
template <int CTRL> __device__ __forceinline__ uint32_t dpp_u(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false);
}
// quad_perm 1,0,3,2 and 2,3,0,1; row_half_mirror; row_mirror: after each, twice as many lanes have the same
template <int L> __device__ __forceinline__ float lanes_sum(float v) {
    v += dpp_of<0xB1>(v); v += dpp_of<0x4E>(v); v += dpp_of<0x141>(v);
    if constexpr (L == 16) v += dpp_of<0x140>(v);
    return v;
}
template <int L> __device__ __forceinline__ float lanes_max(float v) {
    v = fmaxf(v, dpp_of<0xB1>(v)); v = fmaxf(v, dpp_of<0x4E>(v)); v = fmaxf(v, dpp_of<0x141>(v));
    if constexpr (L == 16) v = fmaxf(v, dpp_of<0x140>(v));
    return v;
}
__device__ __forceinline__ uint32_t max_u(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ double max_d(double a, double b) {
    double r;
    asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));                 // (keys are never NaN)
    return r;
}
template <int CTRL> __device__ __forceinline__ double dpp_d(double v) {
    const unsigned long long u = (unsigned long long)__double_as_longlong(v);
    return __longlong_as_double((long long)((unsigned long long)dpp_u<CTRL>((uint32_t)(u >> 32)) << 32 | dpp_u<CTRL>((uint32_t)u)));
}

// four logits from `first` on, as they lie in memory; behind the last expert -inf
template <typename T, bool CUTS> __device__ __forceinline__ Words<T, 4> fetch4(const T *row, uint32_t first, uint32_t n, bool live) {
    typedef Words<T, 4> Any __attribute__((aligned(sizeof(T))));
    constexpr uint32_t NONE = sizeof(T) == 4 ? 0xFF800000u : __is_same(T, __bf16) ? 0xFF80FF80u : 0xFC00FC00u;
    Words<T, 4> w;
    if (live && first + 4 <= n) {
        w = *reinterpret_cast<const Any *>(row + first);
    } else {
        w = NONE;
        if constexpr (CUTS)
            if (live)
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (first + i < n) {
                        if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(row[first + i]);
                        else w[i / 2] = (w[i / 2] & (i & 1 ? 0xFFFFu : 0xFFFF0000u)) | (uint32_t)__builtin_bit_cast(uint16_t, row[first + i]) << (i & 1 ? 16 : 0);
                    }
    }
    return w;
}
template <typename T, bool CUTS> __device__ __forceinline__ void store4(T *row, uint32_t first, uint32_t n, const float (&v)[4]) {
    typedef Words<T, 4> Any __attribute__((aligned(sizeof(T))));
    if (first + 4 <= n) {
        *reinterpret_cast<Any *>(row + first) = words_of<T, 4>(v);
    } else if constexpr (CUTS) {
#pragma unroll
        for (int i = 0; i < 3; ++i) if (first + i < n) row[first + i] = (T)v[i];
    }
}

// Logits as keys that differ for every expert, larger for larger logits and, among equal ones, for lower indices: the largest key
// names the expert.  A 16-bit logit and ten bits of index go into a word; the next key below the last is found by one subtraction
// each, what lies below it becoming large by wrapping.  A 32-bit logit is a double whose last bits hold the index.
template <typename T> struct Keys {
    typedef uint32_t Key;
    static __device__ __forceinline__ Key of(float l, uint32_t e) {
        const float v = l + 0.f;                                            // (zeros of both signs are equal)
        uint32_t u;
        if constexpr (__is_same(T, __bf16)) u = __float_as_uint(v) >> 16;
        else u = __builtin_bit_cast(uint16_t, (_Float16)v);
        u = u & 0x8000u ? ~u & 0xFFFFu : u | 0x8000u;
        return v > -INFINITY ? u << 10 | (1023u - e) : 0u;
    }
    static __device__ __forceinline__ float value(Key k) {
        uint32_t u = k >> 10;
        u = u & 0x8000u ? u & 0x7FFFu : ~u & 0xFFFFu;
        if constexpr (__is_same(T, __bf16)) return __uint_as_float(u << 16);
        else return (float)__builtin_bit_cast(_Float16, (uint16_t)u);
    }
    static __device__ __forceinline__ int32_t expert(Key k) { return k ? (int32_t)(1023u - (k & 1023u)) : -1; }
    static __device__ __forceinline__ Key none() { return 0u; }
    static __device__ __forceinline__ Key before() { return 0x7FFFFFFFu; }
    template <int L, int N> static __device__ __forceinline__ Key next(Key (&key)[N], Key last) {
        uint32_t c = 0u;
#pragma unroll
        for (int i = 0; i < N; ++i) c = max_u(c, key[i] - last);
        c = max_u(c, dpp_u<0xB1>(c)); c = max_u(c, dpp_u<0x4E>(c)); c = max_u(c, dpp_u<0x141>(c));
        if constexpr (L == 16) c = max_u(c, dpp_u<0x140>(c));
        return c >= 0x80000000u ? c + last : 0u;
    }
};
template <> struct Keys<float> {
    typedef double Key;
    static __device__ __forceinline__ Key none() { return -1.7e308; }
    static __device__ __forceinline__ Key before() { return 1.7e308; }
    static __device__ __forceinline__ Key of(float l, uint32_t e) {
        const double d = (double)(l + 0.f);
        unsigned long long u = (unsigned long long)__double_as_longlong(d);
        if (l == INFINITY) u = 0x7FE0000000000000ull;                       // (above every finite float)
        u |= l < 0.f ? e : 1023u - e;
        return l > -INFINITY ? __longlong_as_double((long long)u) : none();
    }
    static __device__ __forceinline__ float value(Key k) {
        const unsigned long long u = (unsigned long long)__double_as_longlong(k);
        return (u >> 32) == 0x7FE00000ull ? INFINITY : (float)__longlong_as_double((long long)(u & ~1023ull));
    }
    static __device__ __forceinline__ int32_t expert(Key k) {
        const uint32_t low = (uint32_t)__double_as_longlong(k) & 1023u;
        return k == none() ? -1 : (int32_t)(k < 0.0 ? low : 1023u - low);
    }
    template <int L, int N> static __device__ __forceinline__ Key next(Key (&key)[N], Key last) {
        double c = none();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (key[i] == last) key[i] = none();
            c = max_d(c, key[i]);
        }
        c = max_d(c, dpp_d<0xB1>(c)); c = max_d(c, dpp_d<0x4E>(c)); c = max_d(c, dpp_d<0x141>(c));
        if constexpr (L == 16) c = max_d(c, dpp_d<0x140>(c));
        return c;
    }
};

// balance of a group from sum counts * prob_sum
__device__ __forceinline__ float balance_of(uint32_t n_experts, uint32_t top_k, float cp, float n) {
    return n > 0.f ? (float)n_experts / ((float)top_k * n) * (cp / n) : 0.f;
}

// A workgroup's tokens belong to one group.  The only workgroup of a call ends it; otherwise k_route_join follows.  Bound by the chain of
// top_k largest keys of a row and, of few tokens, by latency: 8192 x 256 bfloat16, k = 8, 7.6 us (4 MB of logits), 16 x 64 5.4 us.
template <typename T, int L, int NV, bool CUTS>
__global__ __launch_bounds__(RT_THREADS) void k_route_forward(RouteArgs A) {
    constexpr int SLOTS = 64 / L, V = 4 * NV, KEPT = (int)RK_MAX_TOP_K / L;
    extern __shared__ uint32_t lds[];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, E = A.n_experts, K = A.top_k, j = lane & (L - 1), slot = lane / L;
    uint32_t *const hist = lds;                                 // [n_experts]
    float *const probs = (float *)(lds + E);                    // [waves * slots][n_experts]
    float *const zs = probs + RT_WAVES * SLOTS * E;             // [waves][3]
    for (uint32_t e = threadIdx.x; e < E; e += RT_THREADS) hist[e] = 0u;
    __syncthreads();
    const uint64_t g = blockIdx.x / A.per_group;
    const uint64_t t0 = g * A.group_tokens + (blockIdx.x - g * A.per_group) * A.chunk;
    uint64_t t1 = t0 + A.chunk, end = (g + 1) * A.group_tokens;
    end = end < A.n_tokens ? end : A.n_tokens;
    t1 = t1 < end ? t1 : end;
    float sum[V] = {};
    float z = 0.f, n = 0.f;
    for (uint64_t base = t0 + wave * SLOTS; base < t1; base += RT_WAVES * SLOTS) {
        const uint64_t t = base + slot;
        const bool live = t < t1;
        const T *const row = (const T *)A.logits + t * A.st;
        float l[V], m = -INFINITY;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const Words<T, 4> x = fetch4<T, CUTS>(row, (j + L * i) * 4, E, live);
#pragma unroll
            for (int q = 0; q < 4; ++q) { l[4 * i + q] = element<T>(x, q); m = fmaxf(m, l[4 * i + q]); }
        }
        bool there = live;
        if (A.mask && live) there = A.mask[t] != 0;
        m = lanes_max<L>(m);
        const float ref = there && m > -INFINITY ? m : 0.f;
        typename Keys<T>::Key key[V];
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint32_t e = (j + L * (i / 4)) * 4 + i % 4;
            key[i] = there ? Keys<T>::of(l[i], e) : Keys<T>::none();
            l[i] = there ? exp_f32(l[i] - ref) : 0.f;
            s += l[i];
        }
        s = lanes_sum<L>(s);
        there = there && s != 0.f;                          // (nothing but -inf: no exponential; a NaN stays one)
        const float lse = there ? ref + logf(s) : 0.f, inv = there ? 1.f / s : 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) sum[i] += l[i] * inv;
        z += lse * lse; n += there ? 1.f : 0.f;
        typename Keys<T>::Key last = Keys<T>::before(), mine[KEPT];
#pragma unroll
        for (int h = 0; h < KEPT; ++h) {
            mine[h] = Keys<T>::none();
            for (uint32_t k = 0; k < (uint32_t)L && h * L + k < K; ++k) {
                last = Keys<T>::template next<L, V>(key, last);
                if (j == k) mine[h] = last;
            }
        }
        float w[KEPT], ws = 0.f;
#pragma unroll
        for (int h = 0; h < KEPT; ++h) {
            w[h] = 0.f;
            if (h && h * L >= K) continue;                      // (the same for all: few ask for more than a row's lanes hold)
            w[h] = Keys<T>::expert(mine[h]) >= 0 ? exp_f32(Keys<T>::value(mine[h]) - lse) : 0.f;
            ws += w[h];
        }
        const float scale = A.renorm && there ? 1.f / lanes_sum<L>(ws) : 1.f;
#pragma unroll
        for (int h = 0; h < KEPT; ++h) {
            if (h && h * L >= K) continue;
            const uint32_t k = h * L + j;
            const int32_t e = Keys<T>::expert(mine[h]);
            if (live && k < K) {
                A.expert[t * K + k] = e;
                A.weight[t * K + k] = e >= 0 ? w[h] * scale : 0.f;     // (scale is NaN beside a NaN)
                if (e >= 0) atomicAdd(&hist[e], 1u);
            }
        }
        if (live && j == 0) A.lse[t] = lse;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const uint32_t e = (j + L * (i / 4)) * 4 + i % 4;
        if (e < E) probs[(wave * SLOTS + slot) * E + e] = sum[i];
    }
    z = wave_sum(j == 0 ? z : 0.f); n = wave_sum(j == 0 ? n : 0.f);
    if (lane == 0) { zs[wave] = n; zs[RT_WAVES + wave] = z; }
    __syncthreads();
    const bool only = gridDim.x == 1;
    float cp = 0.f;
    for (uint32_t e = threadIdx.x; e < E; e += RT_THREADS) {
        float p = 0.f;
        for (int r = 0; r < RT_WAVES * SLOTS; ++r) p += probs[r * E + e];
        const uint64_t at = only ? e : (uint64_t)blockIdx.x * E + e;
        (only ? A.counts : A.part_counts)[at] = hist[e];
        (only ? A.prob_sum : A.part_probs)[at] = p;
        cp += (float)hist[e] * p;
    }
    n = 0.f; z = 0.f;
#pragma unroll
    for (int w = 0; w < RT_WAVES; ++w) { n += zs[w]; z += zs[RT_WAVES + w]; }
    if (!only) {
        if (threadIdx.x == 0) A.part_z[blockIdx.x] = make_float2(n, z);
        return;
    }
    cp = wave_sum(cp);
    if (lane == 0) zs[2 * RT_WAVES + wave] = cp;
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 1; w < RT_WAVES; ++w) cp += zs[2 * RT_WAVES + w];
    A.tokens[0] = (uint32_t)n;
    A.loss[0] = balance_of(E, K, cp, n);
    A.loss[1] = n > 0.f ? z / n : 0.f;
}

// The workgroups' parts of a group added up in their order: a workgroup has 16 experts, and 64 threads of it share an expert's parts.
// Bound by latency, its launch and three trips to the device's scope one after the other: 6.6 us for 8192 x 256 in four groups.
constexpr uint32_t RT_COLS = 16, RT_SHARE = 64;
__global__ __launch_bounds__(RT_COLS * RT_SHARE) void k_route_join(RouteArgs A) {
    __shared__ float lds_p[RT_SHARE][RT_COLS], lds_n[16], lds_z[16];
    __shared__ uint32_t lds_c[RT_SHARE][RT_COLS];
    const uint64_t g = blockIdx.x / A.tiles, first = g * A.per_group;
    const uint32_t E = A.n_experts, lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, part = threadIdx.x / RT_COLS;
    uint32_t e = (blockIdx.x - (uint32_t)g * A.tiles) * RT_COLS + threadIdx.x % RT_COLS;
    float n = 0.f, z = 0.f, p = 0.f;
    uint32_t count = 0;
    for (uint64_t c = threadIdx.x; c < A.per_group; c += RT_COLS * RT_SHARE) { n += A.part_z[first + c].x; z += A.part_z[first + c].y; }
    if (e < E)
#pragma unroll 4
        for (uint64_t c = part; c < A.per_group; c += RT_SHARE) {
            count += A.part_counts[(first + c) * E + e];
            p += A.part_probs[(first + c) * E + e];
        }
    n = wave_sum(n); z = wave_sum(z);
    if (lane == 0) { lds_n[wave] = n; lds_z[wave] = z; }
    lds_p[part][threadIdx.x % RT_COLS] = p; lds_c[part][threadIdx.x % RT_COLS] = count;
    __syncthreads();
    if (wave) return;
    // the first wavefront: lane l has the parts l / 16, l / 16 + 4, ... of expert l % 16
    n = 0.f; z = 0.f; p = 0.f; count = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) { n += lds_n[w]; z += lds_z[w]; }
#pragma unroll
    for (uint32_t s = 0; s < RT_SHARE; s += 4) { p += lds_p[s + lane / RT_COLS][lane % RT_COLS]; count += lds_c[s + lane / RT_COLS][lane % RT_COLS]; }
    p += __shfl_xor(p, 16, 64); count += (uint32_t)__shfl_xor((int)count, 16, 64);
    p += __shfl_xor(p, 32, 64); count += (uint32_t)__shfl_xor((int)count, 32, 64);
    if (lane >= RT_COLS) e = E;                             // (the others have the same)
    if (e < E) { A.counts[g * E + e] = count; A.prob_sum[g * E + e] = p; }
    const float cp = wave_sum(e < E ? (float)count * p : 0.f);
    // The workgroup that ends last adds the groups up, in their order.  What it needs of the others goes through stores and loads at the
    // device's scope (the workgroups sit on several L2 caches), which are written through and read where all of the device sees
    // them; when the wait before the counter is over they have arrived, and no cache has to be written back.
    uint32_t ends = 0;
    if (lane == 0) {
        if (e == 0) A.tokens[g] = (uint32_t)n;
        float *const mine = (float *)&A.tile_z[blockIdx.x];
        __hip_atomic_store(mine, cp, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(mine + 1, z, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(mine + 2, n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        ends = __hip_atomic_fetch_add(A.done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if ((uint32_t)__builtin_amdgcn_readfirstlane((int)ends) != gridDim.x - 1u) return;
    asm volatile("" ::: "memory");
    if (lane == 0) __hip_atomic_store(A.done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);     // (for the next call)
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    for (uint64_t q = lane; q < A.n_groups; q += 64) {
        const float *const of = (const float *)&A.tile_z[q * A.tiles];
        float sum = 0.f;
        for (uint32_t i = 0; i < A.tiles; ++i) sum += __hip_atomic_load(of + 4 * i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const float zq = __hip_atomic_load(of + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const float nq = __hip_atomic_load(of + 2, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        s[0] += balance_of(E, A.top_k, sum, nq); s[1] += zq; s[2] += nq; s[3] += nq > 0.f ? 1.0 : 0.0;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int off = 32; off; off >>= 1) s[i] += __shfl_xor(s[i], off, 64);
    if (lane) return;
    A.loss[0] = s[3] > 0.0 ? (float)(s[0] / s[3]) : 0.f;
    A.loss[1] = s[2] > 0.0 ? (float)(s[1] / s[2]) : 0.f;
}

// no token: nothing but zeros (of the one group, if the tokens are not in groups)
__global__ __launch_bounds__(256) void k_route_nothing(RouteArgs A) {
    for (uint64_t e = threadIdx.x; e < A.n_groups * A.n_experts; e += 256) { A.counts[e] = 0u; A.prob_sum[e] = 0.f; }
    if (threadIdx.x < A.n_groups) A.tokens[threadIdx.x] = 0u;
    if (threadIdx.x < 2) A.loss[threadIdx.x] = 0.f;
}

// d l = p (A - sum A p - sum y + d_z 2 lse / n) + y at the chosen experts, where y = p d weight, or, of renormalised weights,
// w (d weight - sum w d weight), and then not in the sum.  y reaches its experts' lanes over LDS: zeros but for what a
// token's lanes put there and take away again; the tokens of a wavefront use places of their own, in program order.  131072 x 160 float32,
// k = 6, 41.5 us, 174 MB, 4.2 TB/s: bound by HBM and, behind it, by the exponentials (about 350 instructions of a wavefront for four tokens).
template <typename T, int L, int NV, bool CUTS>
__global__ __launch_bounds__(RT_THREADS) void k_route_backward(RouteArgs A) {
    constexpr int SLOTS = 64 / L, KEPT = (int)RK_MAX_TOP_K / L;
    extern __shared__ float4 lds4[];
    __shared__ float red[RT_WAVES][2];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, E = A.n_experts, K = A.top_k, j = lane & (L - 1), slot = lane / L;
    float *const y = (float *)lds4 + (wave * SLOTS + slot) * (L * NV * 4);
    const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < NV; ++i) ((float4 *)y)[j + L * i] = zero;
    const uint64_t t0 = (uint64_t)blockIdx.x * A.chunk;
    const uint64_t t1 = t0 + A.chunk < A.n_tokens ? t0 + A.chunk : A.n_tokens;
    // the next token's data are on their way while one is worked on, the first's while the groups are counted (not of so many
    // experts that registers for it would cost wavefronts)
    constexpr bool AHEAD = NV <= 4;
    Words<T, 4> next_l[NV];
    int32_t next_e[KEPT];
    float next_dw[KEPT], next_lse;
    auto fetch = [&](uint64_t t) {
        const bool live = t < t1;
        const T *const row = (const T *)A.logits + t * A.st;
#pragma unroll
        for (int h = 0; h < KEPT; ++h) {
            next_e[h] = -1; next_dw[h] = 0.f;
            if (h && h * L >= K) continue;                      // (the same for all)
            const uint32_t k = h * L + j;
            if (live && k < K) {
                next_e[h] = A.expert[t * K + k];
                if (A.d_weight) next_dw[h] = A.d_weight[t * K + k];
            }
        }
        next_lse = live ? A.lse[t] : 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) next_l[i] = fetch4<T, CUTS>(row, (j + L * i) * 4, E, live);
    };
    if constexpr (AHEAD) fetch(t0 + wave * SLOTS + slot);
    float n = 0.f, some = 0.f;
    for (uint64_t g = threadIdx.x; g < A.n_groups; g += RT_THREADS) {
        const uint32_t c = A.tokens[g];
        n += (float)c; some += c ? 1.f : 0.f;
    }
    n = wave_sum(n); some = wave_sum(some);
    if (lane == 0) { red[wave][0] = n; red[wave][1] = some; }
    __syncthreads();
    n = 0.f; some = 0.f;
#pragma unroll
    for (int w = 0; w < RT_WAVES; ++w) { n += red[w][0]; some += red[w][1]; }
    const float bal = some > 0.f ? A.d_loss[0] * (float)E / ((float)K * some) : 0.f;
    const float dz = n > 0.f ? A.d_loss[1] * 2.f / n : 0.f;
    uint64_t g_end = 0;                                     // first token behind the group that `a` is of
    float a[4 * NV] = {};
    for (uint64_t base = t0 + wave * SLOTS; base < t1; base += RT_WAVES * SLOTS) {
        const uint64_t t = base + slot;
        const bool live = t < t1;
        if (live && t >= g_end) {
            const uint64_t g = t / A.group_tokens;
            g_end = (g + 1) * A.group_tokens;
            const float c = (float)A.tokens[g], s = c > 0.f ? bal / c / c : 0.f;
#pragma unroll
            for (int i = 0; i < 4 * NV; ++i) {
                const uint32_t e = (j + L * (i / 4)) * 4 + i % 4;
                a[i] = e < E ? s * (float)A.counts[g * E + e] : 0.f;
            }
        }
        const T *const row = (const T *)A.logits + t * A.st;
        T *const out = (T *)A.d_logits + t * A.d_st;
        if constexpr (!AHEAD) fetch(t);
        int32_t e[KEPT];
        float dw[KEPT], p[4 * NV];
#pragma unroll
        for (int h = 0; h < KEPT; ++h) { e[h] = (uint32_t)next_e[h] < E ? next_e[h] : -1; dw[h] = next_dw[h]; }
#pragma unroll
        for (int i = 0; i < 4 * NV; ++i) p[i] = element<T>(next_l[i / 4], i % 4);
        const float lse = next_lse;
        if constexpr (AHEAD) fetch(t + RT_WAVES * SLOTS);
        // a token that counts has its first choice, unless all its logits are -inf and NaN
        const bool there = __shfl(e[0], lane & ~(L - 1), 64) >= 0 || lse != lse;
        float yk[KEPT], ws = 0.f, wd = 0.f;
        if (A.d_weight) {
#pragma unroll
            for (int h = 0; h < KEPT; ++h) {
                yk[h] = 0.f;
                if (h && h * L >= K) continue;
                yk[h] = e[h] >= 0 ? exp_f32((float)row[e[h]] - lse) : 0.f;
                ws += yk[h]; wd += e[h] >= 0 ? yk[h] * dw[h] : 0.f;
            }
            ws = lanes_sum<L>(ws); wd = lanes_sum<L>(wd);
#pragma unroll
            for (int h = 0; h < KEPT; ++h) {
                if (h && h * L >= K) continue;
                yk[h] = A.renorm ? yk[h] / ws * (dw[h] - wd / ws) : yk[h] * dw[h];
                if (e[h] >= 0) y[e[h]] = yk[h];
            }
        }
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 4 * NV; ++i) {
            p[i] = there ? exp_f32(p[i] - lse) : 0.f;
            s += a[i] * p[i];
        }
        s = lanes_sum<L>(s) + (A.renorm ? 0.f : wd) - dz * lse;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float4 add = zero;
            if (A.d_weight) add = ((const float4 *)y)[j + L * i];
            float d[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float v = q == 0 ? add.x : q == 1 ? add.y : q == 2 ? add.z : add.w;
                d[q] = there ? p[4 * i + q] * (a[4 * i + q] - s) + v : 0.f;
            }
            if (live) store4<T, CUTS>(out, (j + L * i) * 4, E, d);
        }
        __builtin_amdgcn_wave_barrier();
        if (A.d_weight)
#pragma unroll
            for (int h = 0; h < KEPT; ++h) if (e[h] >= 0) y[e[h]] = 0.f;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// ---- host
// f(type, lanes of a token, vectors of a lane, whether four divide the experts)
template <typename F> void with_lanes(uint32_t type, uint32_t n_experts, F f) {
    auto cut = [&](auto t, auto l, auto v) {
        if (n_experts % 4) f(t, l, v, std::true_type()); else f(t, l, v, std::false_type());
    };
    auto sized = [&](auto t) {
        const auto L8 = std::integral_constant<int, 8>();
        const auto L16 = std::integral_constant<int, 16>();
        if (n_experts <= 32) cut(t, L8, std::integral_constant<int, 1>());
        else if (n_experts <= 64) cut(t, L8, std::integral_constant<int, 2>());
        else if (n_experts <= 128) cut(t, L16, std::integral_constant<int, 2>());
        else if (n_experts <= 192) cut(t, L16, std::integral_constant<int, 3>());
        else if (n_experts <= 256) cut(t, L16, std::integral_constant<int, 4>());
        else if (n_experts <= 512) cut(t, L16, std::integral_constant<int, 8>());
        else cut(t, L16, std::integral_constant<int, 16>());
    };
    if (type == RK_F32) sized(float());
    else if (type == RK_BF16) sized(__bf16());
    else sized(_Float16());
}
uint32_t lanes_of(uint32_t n_experts) { return n_experts <= 64 ? 8 : 16; }

int32_t check_router(rk_ctx *ctx, const rk_router *r, uint64_t n_tokens, const rk_matrix *logits) {
    if (!r) return rk_fail(ctx, RK_ERR_INVALID_ARG, "router is null");
    if (r->n_experts < 1 || r->top_k < 1 || r->top_k > r->n_experts || r->renormalise > 1)
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "n_experts, top_k or renormalise out of range");
    if (r->n_experts > RK_MAX_EXPERTS || r->top_k > RK_MAX_TOP_K)
        return rk_fail(ctx, RK_ERR_UNSUPPORTED, "%u experts, %u chosen: %u and %u at most", r->n_experts, r->top_k, RK_MAX_EXPERTS, RK_MAX_TOP_K);
    if (n_tokens > 0xFFFFFFull) return rk_fail(ctx, RK_ERR_UNSUPPORTED, "more than 2^24 - 1 tokens");     // counts are exact in a float
    if (!rk_matrix_ok(logits, n_tokens, r->n_experts)) return rk_fail(ctx, RK_ERR_INVALID_ARG, "logits null, misaligned or of a stride below n_experts");
    return RK_OK;
}
void fill_router(RouteArgs &A, const rk_router *r, uint64_t n_tokens, const rk_matrix *logits) {
    A.logits = logits->data; A.st = logits->stride;
    A.n_tokens = n_tokens;
    A.group_tokens = r->group_tokens && r->group_tokens < n_tokens ? r->group_tokens : n_tokens;
    A.n_groups = n_tokens ? (n_tokens + A.group_tokens - 1) / A.group_tokens : (r->group_tokens ? 0 : 1);
    A.n_experts = r->n_experts; A.top_k = r->top_k; A.renorm = r->renormalise;
}
bool misaligned4(std::initializer_list<const void *> ps) {
    for (const void *p : ps) if (((uintptr_t)p & 3u)) return true;
    return false;
}

}  // namespace

extern "C" int32_t rk_route_forward(rk_ctx *ctx, const rk_router *router, uint64_t n_tokens, const rk_matrix *logits, const uint8_t *mask,
                                    int32_t *expert, float *weight, float *lse, uint32_t *counts, float *prob_sum, uint32_t *tokens,
                                    float *loss) {
    if (!ctx) return RK_ERR_INVALID_ARG;
    int32_t rc = check_router(ctx, router, n_tokens, logits);
    if (rc != RK_OK) return rc;
    RouteArgs A{};
    fill_router(A, router, n_tokens, logits);
    if ((n_tokens && (!expert || !weight || !lse)) || (A.n_groups && (!counts || !prob_sum || !tokens)) || !loss ||
        misaligned4({expert, weight, lse, counts, prob_sum, tokens, loss}))
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "an output is null or misaligned");
    A.tiles = (A.n_experts + RT_COLS - 1) / RT_COLS;
    if (A.n_groups * A.tiles * RT_COLS * RT_SHARE > 0xFFFFFFFFull) return rk_fail(ctx, RK_ERR_UNSUPPORTED, "2^26 groups times experts or more");
    RK_HIP(ctx, hipSetDevice(ctx->device));
    A.mask = mask; A.expert = expert; A.weight = weight; A.lse = lse; A.counts = counts; A.prob_sum = prob_sum; A.tokens = tokens; A.loss = loss;
    // up to four workgroups a compute unit share the tokens, each in rounds of as many as its wavefronts hold (65536 x 256 bfloat16 32.8 us; eight 37.7, two 31.5, one
    // 36.6; 19883 x 160 17.3, 17.4, 18.3, 17.8); few tokens, of up to four rounds, are one's (128 x 64 7.4 us, in two kernels 10.1; 256 x 64 11.1 and
    // 10.2; of eight rounds 512 x 64 18.7 us, in two kernels 10.2)
    const uint64_t at_once = RT_WAVES * 64 / lanes_of(A.n_experts);
    A.chunk = (n_tokens + 1024 * at_once - 1) / (1024 * at_once) * at_once;
    if (A.n_groups == 1 && n_tokens <= 4 * at_once) A.chunk = 4 * at_once;      // (then there is nothing to join)
    A.per_group = n_tokens ? (A.group_tokens + A.chunk - 1) / A.chunk : 0;
    const uint64_t blocks = A.per_group * (n_tokens ? A.n_groups : 0);
    if (blocks == 0) {
        k_route_nothing<<<1, 256, 0, ctx->stream>>>(A);
        RK_CHECK_LAUNCH(ctx, "k_route_nothing");
        return RK_OK;
    }
    if (blocks > 1) {
        if ((rc = rk_scratch(ctx, SL_ROUTE_COUNTS, blocks * A.n_experts * 4, (void **)&A.part_counts)) != RK_OK) return rc;
        if ((rc = rk_scratch(ctx, SL_ROUTE_PROBS, blocks * A.n_experts * 4, (void **)&A.part_probs)) != RK_OK) return rc;
        if ((rc = rk_scratch(ctx, SL_ROUTE_Z, blocks * 8, (void **)&A.part_z)) != RK_OK) return rc;
        if ((rc = rk_scratch(ctx, SL_ROUTE_GROUPS, A.n_groups * A.tiles * 16, (void **)&A.tile_z)) != RK_OK) return rc;
        if ((rc = rk_scratch(ctx, SL_ROUTE_DONE, 4, (void **)&A.done)) != RK_OK) return rc;
        if (!ctx->route_clear) {                                // (once, and never in a graph: the wait would fail there)
            RK_HIP(ctx, hipMemsetAsync(A.done, 0, 4, ctx->stream));
            RK_HIP(ctx, hipStreamSynchronize(ctx->stream));
            ctx->route_clear = true;
        }
    }
    const size_t lds = (size_t)A.n_experts * 4 * (1 + at_once) + RT_WAVES * 12;
    with_lanes(logits->type, A.n_experts, [&](auto t, auto l, auto v, auto c) {
        const auto kernel = k_route_forward<decltype(t), decltype(l)::value, decltype(v)::value, decltype(c)::value>;
        if (lds > 65536)
            rc = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) == hipSuccess ? RK_OK : RK_ERR_DEVICE;
        if (rc == RK_OK) kernel<<<(uint32_t)blocks, RT_THREADS, lds, ctx->stream>>>(A);
    });
    if (rc != RK_OK) return rk_fail(ctx, rc, "k_route_forward: no room in LDS");
    RK_CHECK_LAUNCH(ctx, "k_route_forward");
    if (blocks > 1) {
        k_route_join<<<(uint32_t)(A.n_groups * A.tiles), RT_COLS * RT_SHARE, 0, ctx->stream>>>(A);
        RK_CHECK_LAUNCH(ctx, "k_route_join");
    }
    return RK_OK;
}

extern "C" int32_t rk_route_backward(rk_ctx *ctx, const rk_router *router, uint64_t n_tokens, const rk_matrix *logits, const int32_t *expert,
                                     const float *lse, const uint32_t *counts, const uint32_t *tokens, const float *d_loss,
                                     const float *d_weight, const rk_matrix *d_logits) {
    if (!ctx) return RK_ERR_INVALID_ARG;
    int32_t rc = check_router(ctx, router, n_tokens, logits);
    if (rc != RK_OK) return rc;
    if (!rk_matrix_ok(d_logits, n_tokens, router->n_experts) || d_logits->type != logits->type)
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "d_logits null, misaligned, of a stride below n_experts or of another type than the logits");
    if (n_tokens == 0) return RK_OK;
    if (!expert || !lse || !counts || !tokens || !d_loss || misaligned4({expert, lse, counts, tokens, d_loss, d_weight}))
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "an input is null or misaligned");
    RK_HIP(ctx, hipSetDevice(ctx->device));
    RouteArgs A{};
    fill_router(A, router, n_tokens, logits);
    A.expert = const_cast<int32_t *>(expert); A.lse = const_cast<float *>(lse); A.counts = const_cast<uint32_t *>(counts);
    A.tokens = const_cast<uint32_t *>(tokens);
    A.d_loss = d_loss; A.d_weight = d_weight; A.d_logits = d_logits->data; A.d_st = d_logits->stride;
    // two workgroups a compute unit, as many as fit at once, each at least as many tokens as its wavefronts hold at once (131072 x 160 in 32
    // bits 42.9 us, with twice as many 44.0; 60000 x 250 23.9 and 28.4)
    const uint64_t at_once = RT_WAVES * 64 / lanes_of(A.n_experts);
    A.chunk = (n_tokens + 511) / 512;
    A.chunk = (A.chunk + at_once - 1) / at_once * at_once;
    const uint64_t blocks = (n_tokens + A.chunk - 1) / A.chunk;
    with_lanes(logits->type, A.n_experts, [&](auto t, auto l, auto v, auto c) {
        constexpr int L = decltype(l)::value, NV = decltype(v)::value;
        const size_t lds = (size_t)RT_WAVES * 64 * NV * 16;
        const auto kernel = k_route_backward<decltype(t), L, NV, decltype(c)::value>;
        if (lds > 65536 - 1024)
            rc = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) == hipSuccess ? RK_OK : RK_ERR_DEVICE;
        if (rc == RK_OK) kernel<<<(uint32_t)blocks, RT_THREADS, lds, ctx->stream>>>(A);
    });
    if (rc != RK_OK) return rk_fail(ctx, rc, "k_route_backward: no room in LDS");
    RK_CHECK_LAUNCH(ctx, "k_route_backward");
    return RK_OK;
}
