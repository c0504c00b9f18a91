// The router of a mixture of experts: top-k choice and weights, counts per expert, balance and z loss, and the gradient of the
// logits (rk_route_forward, rk_route_backward).
#include <cmath>

#include "rk_vec.h"

namespace {

constexpr int RT_THREADS = 256, RT_WAVES = 4;

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
    float4 *group_z;                    // [group]: its balance, sum of lse^2, tokens, 1 if any
    // backward
    void *d_logits;
    uint64_t d_st;
    const float *d_loss, *d_weight;
};

// A wavefront holds a token's logits, expert e in lane e & 63; a workgroup's tokens belong to one group.
template <typename T, int VPL>
__global__ __launch_bounds__(RT_THREADS) void k_route_forward(RouteArgs A) {
    extern __shared__ uint32_t lds[];
    uint32_t *const hist = lds;                                 // [n_experts]
    float *const probs = (float *)(lds + A.n_experts);          // [waves][n_experts]
    float *const zs = probs + RT_WAVES * A.n_experts;           // [waves][2]
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, E = A.n_experts, K = A.top_k;
    for (uint32_t e = threadIdx.x; e < E; e += RT_THREADS) hist[e] = 0u;
    __syncthreads();
    const uint64_t g = blockIdx.x / A.per_group;
    const uint64_t t0 = g * A.group_tokens + (blockIdx.x - g * A.per_group) * A.chunk;
    uint64_t t1 = t0 + A.chunk, end = (g + 1) * A.group_tokens;
    end = end < A.n_tokens ? end : A.n_tokens;
    t1 = t1 < end ? t1 : end;
    float sum[VPL] = {};
    float z = 0.f, n = 0.f;
    for (uint64_t t = t0 + wave; t < t1; t += RT_WAVES) {
        const T *const row = (const T *)A.logits + t * A.st;
        float l[VPL], m = -INFINITY;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            const uint32_t e = lane + 64u * i;
            l[i] = e < E ? (float)row[e] : -INFINITY;
            m = fmaxf(m, l[i]);
        }
        m = wave_max(m);
        const bool there = (!A.mask || A.mask[t]) && m > -INFINITY;
        float lse = 0.f, mine = 0.f;
        int32_t chosen = -1;
        if (there) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < VPL; ++i) s += exp_f32(l[i] - m);
            lse = m + logf(wave_sum(s));
#pragma unroll
            for (int i = 0; i < VPL; ++i) sum[i] += exp_f32(l[i] - lse);
            z += lse * lse; n += 1.f;
            for (uint32_t k = 0; k < K; ++k) {
                float best = -INFINITY;
                uint32_t at = 0xFFFFFFFFu;
#pragma unroll
                for (int i = 0; i < VPL; ++i)
                    if (l[i] > best) { best = l[i]; at = lane + 64u * i; }
                const float top = wave_max(best);
                if (!(top > -INFINITY)) break;
                uint32_t who = best == top ? at : 0xFFFFFFFFu;
#pragma unroll
                for (int off = 1; off < 64; off <<= 1) { const uint32_t o = (uint32_t)__shfl_xor((int)who, off, 64); who = o < who ? o : who; }
#pragma unroll
                for (int i = 0; i < VPL; ++i)
                    if (lane + 64u * i == who) l[i] = -INFINITY;
                if (lane == k) { chosen = (int32_t)who; mine = exp_f32(top - lse); }
                if (lane == 0) atomicAdd(&hist[who], 1u);
            }
            if (A.renorm) mine /= wave_sum(mine);
        }
        if (lane < K) {
            A.expert[t * K + lane] = chosen;
            A.weight[t * K + lane] = chosen < 0 ? 0.f : mine;
        }
        if (lane == 0) A.lse[t] = lse;
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i)
        if (lane + 64u * i < E) probs[wave * E + lane + 64u * i] = sum[i];
    if (lane == 0) { zs[2 * wave] = n; zs[2 * wave + 1] = z; }
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < E; e += RT_THREADS) {
        A.part_counts[(uint64_t)blockIdx.x * E + e] = hist[e];
        A.part_probs[(uint64_t)blockIdx.x * E + e] = (probs[e] + probs[E + e]) + (probs[2 * E + e] + probs[3 * E + e]);
    }
    if (threadIdx.x == 0)
        A.part_z[blockIdx.x] = make_float2((zs[0] + zs[2]) + (zs[4] + zs[6]), (zs[1] + zs[3]) + (zs[5] + zs[7]));
}

// the workgroups' parts of a group added up in their order, and the group's balance
__global__ __launch_bounds__(RT_THREADS) void k_route_join(RouteArgs A) {
    __shared__ float lds[RT_WAVES][3];
    const uint64_t g = blockIdx.x, first = g * A.per_group;
    const uint32_t E = A.n_experts, lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    float n = 0.f, z = 0.f, cp = 0.f;
    for (uint64_t c = threadIdx.x; c < A.per_group; c += RT_THREADS) { n += A.part_z[first + c].x; z += A.part_z[first + c].y; }
    for (uint32_t e = threadIdx.x; e < E; e += RT_THREADS) {
        uint32_t count = 0;
        float p = 0.f;
        for (uint64_t c = 0; c < A.per_group; ++c) {
            count += A.part_counts[(first + c) * E + e];
            p += A.part_probs[(first + c) * E + e];
        }
        A.counts[g * E + e] = count;
        A.prob_sum[g * E + e] = p;
        cp += (float)count * p;
    }
    n = wave_sum(n); z = wave_sum(z); cp = wave_sum(cp);
    if (lane == 0) { lds[wave][0] = n; lds[wave][1] = z; lds[wave][2] = cp; }
    __syncthreads();
    if (threadIdx.x) return;
    n = (lds[0][0] + lds[1][0]) + (lds[2][0] + lds[3][0]);
    z = (lds[0][1] + lds[1][1]) + (lds[2][1] + lds[3][1]);
    cp = (lds[0][2] + lds[1][2]) + (lds[2][2] + lds[3][2]);
    A.tokens[g] = (uint32_t)n;
    A.group_z[g] = make_float4(n > 0.f ? (float)E / ((float)A.top_k * n) * (cp / n) : 0.f, z, n, n > 0.f ? 1.f : 0.f);
}

__global__ __launch_bounds__(RT_THREADS) void k_route_loss(RouteArgs A) {
    __shared__ double lds[RT_THREADS][4];
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    for (uint64_t g = threadIdx.x; g < A.n_groups; g += RT_THREADS) {
        const float4 v = A.group_z[g];
        s[0] += v.x; s[1] += v.y; s[2] += v.z; s[3] += v.w;
    }
    for (int i = 0; i < 4; ++i) lds[threadIdx.x][i] = s[i];
    for (uint32_t off = RT_THREADS / 2; off; off >>= 1) {
        __syncthreads();
        if (threadIdx.x < off)
            for (int i = 0; i < 4; ++i) lds[threadIdx.x][i] += lds[threadIdx.x + off][i];
    }
    if (threadIdx.x) return;
    A.loss[0] = lds[0][3] > 0.0 ? (float)(lds[0][0] / lds[0][3]) : 0.f;
    A.loss[1] = lds[0][2] > 0.0 ? (float)(lds[0][1] / lds[0][2]) : 0.f;
}

// d l = p (A - sum A p + d_z 2 lse / n) (+ what comes through renormalised weights), a wavefront a token
template <typename T, int VPL>
__global__ __launch_bounds__(RT_THREADS) void k_route_backward(RouteArgs A) {
    __shared__ float lds[RT_WAVES][2];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, E = A.n_experts, K = A.top_k;
    float n = 0.f, some = 0.f;
    for (uint64_t g = threadIdx.x; g < A.n_groups; g += RT_THREADS) {
        const uint32_t c = A.tokens[g];
        n += (float)c; some += c ? 1.f : 0.f;
    }
    n = wave_sum(n); some = wave_sum(some);
    if (lane == 0) { lds[wave][0] = n; lds[wave][1] = some; }
    __syncthreads();
    n = (lds[0][0] + lds[1][0]) + (lds[2][0] + lds[3][0]);
    some = (lds[0][1] + lds[1][1]) + (lds[2][1] + lds[3][1]);
    const float bal = some > 0.f ? A.d_loss[0] * (float)E / ((float)K * some) : 0.f;
    const float dz = n > 0.f ? A.d_loss[1] * 2.f / n : 0.f;
    uint64_t t0 = ((uint64_t)blockIdx.x * RT_WAVES + wave) * A.chunk, t1 = t0 + A.chunk, of = ~0ull;
    t1 = t1 < A.n_tokens ? t1 : A.n_tokens;
    float a[VPL] = {};
    for (uint64_t t = t0; t < t1; ++t) {
        const uint64_t g = t / A.group_tokens;
        if (g != of) {
            of = g;
            const float c = (float)A.tokens[g];
            const float s = c > 0.f ? bal / c / c : 0.f;
#pragma unroll
            for (int i = 0; i < VPL; ++i)
                if (lane + 64u * i < E) a[i] = s * (float)A.counts[g * E + lane + 64u * i];
        }
        const int32_t mine = lane < K ? A.expert[t * K + lane] : -1;
        const bool there = __builtin_amdgcn_readfirstlane(mine) >= 0;
        T *const out = (T *)A.d_logits + t * A.d_st;
        float d[VPL];
        if (there) {
            const T *const row = (const T *)A.logits + t * A.st;
            const float lse = A.lse[t];
            float p[VPL], x[VPL] = {}, w[VPL] = {};
#pragma unroll
            for (int i = 0; i < VPL; ++i) p[i] = lane + 64u * i < E ? exp_f32((float)row[lane + 64u * i] - lse) : 0.f;
            if (A.d_weight) {
                const float dw = lane < K && mine >= 0 ? A.d_weight[t * K + lane] : 0.f;
                for (uint32_t k = 0; k < K; ++k) {
                    const int32_t e = __builtin_amdgcn_readlane(mine, k);
                    const float v = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(dw), k));
#pragma unroll
                    for (int i = 0; i < VPL; ++i)
                        if ((int32_t)(lane + 64u * i) == e) { x[i] = v; w[i] = p[i]; }
                }
            }
            float s = 0.f, ws = 0.f, wx = 0.f;
#pragma unroll
            for (int i = 0; i < VPL; ++i) {
                s += (A.renorm ? a[i] : a[i] + x[i]) * p[i];
                ws += w[i]; wx += w[i] * x[i];
            }
            s = wave_sum(s);
            if (A.renorm && A.d_weight) {
                ws = wave_sum(ws); wx = wave_sum(wx) / ws;
            }
#pragma unroll
            for (int i = 0; i < VPL; ++i) {
                d[i] = p[i] * ((A.renorm ? a[i] : a[i] + x[i]) - s + dz * lse);
                if (A.renorm && A.d_weight && w[i] != 0.f) d[i] += w[i] / ws * (x[i] - wx);
            }
        } else {
#pragma unroll
            for (int i = 0; i < VPL; ++i) d[i] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < VPL; ++i)
            if (lane + 64u * i < E) out[lane + 64u * i] = (T)d[i];
    }
}

// ---- host
template <typename F> void with_lanes(uint32_t type, uint32_t n_experts, F f) {
    auto sized = [&](auto t) {
        if (n_experts <= 64) f(t, std::integral_constant<int, 1>());
        else if (n_experts <= 128) f(t, std::integral_constant<int, 2>());
        else if (n_experts <= 256) f(t, std::integral_constant<int, 4>());
        else if (n_experts <= 512) f(t, std::integral_constant<int, 8>());
        else f(t, std::integral_constant<int, 16>());
    };
    if (type == RK_F32) sized(float());
    else if (type == RK_BF16) sized(__bf16());
    else sized(_Float16());
}

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
    RK_HIP(ctx, hipSetDevice(ctx->device));
    A.mask = mask; A.expert = expert; A.weight = weight; A.lse = lse; A.counts = counts; A.prob_sum = prob_sum; A.tokens = tokens; A.loss = loss;
    // four workgroups a compute unit share the tokens, eight tokens each at least
    uint64_t chunk = (n_tokens + 1023) / 1024;
    if (chunk < 8) chunk = 8;
    A.per_group = n_tokens ? (A.group_tokens + chunk - 1) / chunk : 0;
    A.chunk = A.per_group ? (A.group_tokens + A.per_group - 1) / A.per_group : 0;
    const uint64_t blocks = A.per_group * (n_tokens ? A.n_groups : 0);
    if ((rc = rk_scratch(ctx, SL_ROUTE_COUNTS, blocks * A.n_experts * 4, (void **)&A.part_counts)) != RK_OK) return rc;
    if ((rc = rk_scratch(ctx, SL_ROUTE_PROBS, blocks * A.n_experts * 4, (void **)&A.part_probs)) != RK_OK) return rc;
    if ((rc = rk_scratch(ctx, SL_ROUTE_Z, blocks * 8, (void **)&A.part_z)) != RK_OK) return rc;
    if ((rc = rk_scratch(ctx, SL_ROUTE_GROUPS, A.n_groups * 16, (void **)&A.group_z)) != RK_OK) return rc;
    if (blocks) {
        const size_t lds = (size_t)A.n_experts * 4 * (1 + RT_WAVES) + RT_WAVES * 8;
        with_lanes(logits->type, A.n_experts, [&](auto t, auto v) {
            k_route_forward<decltype(t), decltype(v)::value><<<(uint32_t)blocks, RT_THREADS, lds, ctx->stream>>>(A);
        });
        RK_CHECK_LAUNCH(ctx, "k_route_forward");
    }
    if (A.n_groups) {
        k_route_join<<<(uint32_t)A.n_groups, RT_THREADS, 0, ctx->stream>>>(A);
        RK_CHECK_LAUNCH(ctx, "k_route_join");
    }
    k_route_loss<<<1, RT_THREADS, 0, ctx->stream>>>(A);
    RK_CHECK_LAUNCH(ctx, "k_route_loss");
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
    A.chunk = (n_tokens + 8191) / 8192;                     // tokens of a wavefront
    const uint64_t blocks = (n_tokens + A.chunk * RT_WAVES - 1) / (A.chunk * RT_WAVES);
    with_lanes(logits->type, A.n_experts, [&](auto t, auto v) {
        k_route_backward<decltype(t), decltype(v)::value><<<(uint32_t)blocks, RT_THREADS, 0, ctx->stream>>>(A);
    });
    RK_CHECK_LAUNCH(ctx, "k_route_backward");
    return RK_OK;
}
