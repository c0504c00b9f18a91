// The loss of rows under a vocabulary's weights and its gradients, without keeping the logits (rk_head in rubick.h).
//
// Rows that count are gathered first, so that products take no others, and padded with zeros to whole steps of k.  The loss
// takes the logits' tiles out of the product's registers: of every row the largest and the sum of exponentials over a tile's
// words, joined in fixed order.  The gradients go through the vocabulary in pieces, from the last to the first: a piece's logits are made again and become
// g = row_weight (p (1 + 2 z lse) - onehot), rounded to the rows' type and scaled by a power of two that keeps float16 in its range (rows far below the
// largest one by their own, for dx; d_weight takes them under the largest one's again);
// dx adds up g W over the pieces in float32, and the piece's rows of d_weight are g^T x.  By far the largest element of a row is its label's: what
// rounding to 16 bits takes off it is kept and its products are added to dx and d_weight in float32 (777 x 50021 x 1111 in float16: both are
// 2.1e-4 from the definition, all of it their own rounding, and 3.5e-4 without).  Where the loss is made along with
// them, it leaves the exponentials of the piece that it ends with, which then only have to be scaled: of a vocabulary of one piece all of them, of a longer one
// what is left for the last piece.
//
// The products' kernels are bound by the matrix units (figures in rk_gemm.h), what stands around them by memory: for 2,048 x 128,000 x 5,248 in bfloat16 the rows'
// gathering takes 10 us, k_head_join 9, k_head_scale 147 (0.94 GB, 6.4 TB/s) instead of the 2.2 ms of another product, k_head_dx_out 40.
// Five rows are bound by the weights: 235 to 243 us for 1.34 GB, 5.6 TB/s.
#include "rk_gemm.h"

namespace {

constexpr uint32_t HD_THREADS = 1024;
constexpr uint64_t HD_BUDGET = 1ull << 30;                  // bytes of a piece's gradients, and weights where they are padded
constexpr uint64_t HD_PARTS = 1ull << 28;                   // ... of the sums of the loss's tiles
constexpr int HD_TA = 256;                                  // words, or columns, of a tile

struct RowInfo { float lse, factor, share, unit; };         // g = (p factor - onehot) share, which stands for room / unit times the gradient

// what the device keeps of the rows that count
struct Rows {
    uint32_t *count;            // [0] how many, [1] bits of the largest unit of a row
    int32_t *row, *place;       // a kept row's place in the matrix; a row's place among the kept, or -1
    int32_t *label;
    float *weight, *label_logit, *top, *sum;
    float *lost, *lost_dw;      // what rounding takes off the gradient of a row's label; float16: for d_weight, under the largest unit
    RowInfo *info;
};

struct RowsArgs {
    Rows R;
    const int32_t *label;
    const float *row_weight;
    float *loss, *lse;          // zeros for rows that are left out, or null
    uint64_t n_rows;
    uint32_t vocab;
};

__global__ __launch_bounds__(HD_THREADS) void k_head_rows(const RowsArgs A) {
    __shared__ uint32_t in_wave[HD_THREADS / 64];
    constexpr uint32_t EACH = 4;
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    uint32_t before = 0;
    for (uint64_t begin = 0; begin < A.n_rows; begin += HD_THREADS * EACH) {
        int32_t label[EACH];
        float weight[EACH];
        uint32_t n = 0;
#pragma unroll
        for (uint32_t e = 0; e < EACH; ++e) {
            const uint64_t r = begin + threadIdx.x * EACH + e;
            label[e] = r < A.n_rows ? A.label[r] : -1;
            weight[e] = r < A.n_rows ? A.row_weight ? A.row_weight[r] : 1.f : 0.f;
            if (label[e] < 0 || (uint32_t)label[e] >= A.vocab || weight[e] == 0.f) label[e] = -1;
            n += label[e] >= 0;
        }
        uint32_t upto = n;                                  // inclusive over the wavefront
#pragma unroll
        for (uint32_t d = 1; d < 64; d *= 2) {
            const uint32_t o = __shfl_up(upto, d, 64);
            upto += lane >= d ? o : 0u;
        }
        if (lane == 63) in_wave[wave] = upto;
        __syncthreads();
        uint32_t at = before + upto - n, all = 0;
#pragma unroll
        for (uint32_t w = 0; w < HD_THREADS / 64; ++w) {
            at += w < wave ? in_wave[w] : 0u;
            all += in_wave[w];
        }
        before += all;
#pragma unroll
        for (uint32_t e = 0; e < EACH; ++e) {
            const uint64_t r = begin + threadIdx.x * EACH + e;
            if (r >= A.n_rows) continue;
            const bool there = label[e] >= 0;
            A.R.place[r] = there ? (int32_t)at : -1;
            if (there) {
                A.R.row[at] = (int32_t)r;
                A.R.label[at] = label[e];
                A.R.weight[at] = weight[e];
                ++at;
            } else if (A.loss) {
                A.loss[r] = 0.f;
                A.lse[r] = 0.f;
            }
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) A.R.count[0] = before;
}

// Rows one behind the other, each padded with zeros to out_width (a multiple of 16 bytes): the kept ones of x (count rows of R), or n_rows as they lie
// (count null).  A lane takes 16 bytes of the result, whatever the alignment of what it reads.
template <typename T> __global__ __launch_bounds__(256) void k_head_pad(const int32_t *row, const uint32_t *count, uint32_t n_rows, const T *x, uint64_t stride, uint32_t width, T *out, uint32_t out_width) {
    constexpr uint32_t EACH = 16 / sizeof(T);
    const uint32_t per_row = out_width / EACH, rows = count ? *count : n_rows;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < (uint64_t)rows * per_row; i += (uint64_t)gridDim.x * 256) {
        const uint32_t r = (uint32_t)(i / per_row), c = (uint32_t)(i - (uint64_t)r * per_row) * EACH;
        const T *const from = x + (uint64_t)(row ? (uint32_t)row[r] : r) * stride + c;
        Vec<uint32_t, 4> w;
        if (c + EACH <= width) {
            w = *(const Loose<Vec<uint32_t, 4>, T> *)from;
        } else {
            Vec<T, EACH> v = (T)0.f;
#pragma unroll
            for (uint32_t e = 0; e < EACH; ++e) if (c + e < width) v[e] = from[e];
            w = __builtin_bit_cast(Vec<uint32_t, 4>, v);
        }
        *(Vec<uint32_t, 4> *)(out + (uint64_t)r * out_width + c) = w;
    }
}

struct LogitsArgs {
    Rows R;
    Side W, X;                  // of this piece; the kept rows
    uint32_t width, tiles_b;
    uint32_t first, words;      // the piece's first word, how many it has
    float scale, room;
    float2 *parts;              // loss: [words / TA][kept rows]
    uint64_t parts_stride;
    void *g;                    // [kept rows][g_stride]: gradients, or what the loss leaves of them (null: nothing)
    uint64_t g_stride;
};
template <typename T> __device__ __forceinline__ float exp_of(float x) {
    if constexpr (sizeof(T) == 4) return exp_f32(x);
    else return __builtin_amdgcn_exp2f(x * 1.4426950408889634f);
}

// LOSS: a tile's largest logit and sum of exponentials of every row, and its label's logit (and, with g, the exponentials themselves, `room` times as
// large); otherwise the gradients of the logits
template <typename T, int TA, int TB, int WA, bool LOSS> __global__ __launch_bounds__(GM_THREADS) void k_head_logits(const LogitsArgs A) {
    typedef Tile<T, TA, TB, WA, ALONG, ALONG> Tl;
    const uint32_t n = A.R.count[0];
    const Turn at_turn = turn_of(in_runs(blockIdx.x, gridDim.x), gridDim.x / A.tiles_b, A.tiles_b);
    const uint32_t a0 = at_turn.a * TA, b0 = at_turn.b * TB;
    if (b0 >= n) return;
    Side X = A.X;
    X.count = n;
    Tl t;
    t.run(A.W, X, a0, b0, 0, A.width);
    const typename Tl::At at = Tl::place();
    const uint32_t a_of = a0 + at.a, b_of = b0 + at.b;
    if constexpr (LOSS) {
        float *const tops = (float *)t.shared, *const sums = tops + WA * TB;
        const uint32_t wa = at.a / (TA / WA), in_tile = at.b;           // (the wavefront's place, and its rows' in the tile)
        float top[Tl::MB];
#pragma unroll
        for (int j = 0; j < Tl::MB; ++j) {
            const uint32_t b = b_of + 16 * j;
            const int64_t label = b < n ? (int64_t)A.R.label[b] - (int64_t)A.first : -1;
            float own = 0.f;
            top[j] = -INFINITY;
#pragma unroll
            for (int i = 0; i < Tl::MA; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t a = a_of + 16 * i + q;
                    float l = t.acc[i][j][q] * A.scale;
                    l = a < A.words ? l : -INFINITY;
                    t.acc[i][j][q] = l;
                    top[j] = fmaxf(top[j], l);
                    own = label == (int64_t)a ? l : own;
                }
            const uint32_t d = (uint32_t)(label - (int64_t)a_of);
            if (label >= 0 && d < 16 * Tl::MA && (d & 15u) < 4) A.R.label_logit[b] = own;
            top[j] = fmaxf(top[j], __shfl_xor(top[j], 16, 64));
            top[j] = fmaxf(top[j], __shfl_xor(top[j], 32, 64));
            if (at.lane < 16) tops[wa * TB + in_tile + 16 * j] = top[j];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < Tl::MB; ++j) {
#pragma unroll
            for (uint32_t w = 0; w < WA; ++w) top[j] = fmaxf(top[j], tops[w * TB + in_tile + 16 * j]);
            const float from = top[j] == -INFINITY ? 0.f : top[j];
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < Tl::MA; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float e = exp_of<T>(t.acc[i][j][q] - from);
                    t.acc[i][j][q] = e;
                    sum += e;
                }
            sum += __shfl_xor(sum, 16, 64);
            sum += __shfl_xor(sum, 32, 64);
            if (at.lane < 16) sums[wa * TB + in_tile + 16 * j] = sum;
            __builtin_amdgcn_sched_barrier(0);
        }
        __syncthreads();
        for (uint32_t b = threadIdx.x; b < TB && b0 + b < n; b += GM_THREADS) {
            float m = tops[b], s = sums[b];
            for (uint32_t w = 1; w < WA; ++w) { m = fmaxf(m, tops[w * TB + b]); s += sums[w * TB + b]; }
            A.parts[(uint64_t)at_turn.a * A.parts_stride + b0 + b] = make_float2(m, s);
        }
    }
    if constexpr (!LOSS) {
#pragma unroll
        for (int j = 0; j < Tl::MB; ++j) {
            const uint32_t b = b_of + 16 * j;
            const bool there = b < n;
            const int64_t label = there ? (int64_t)A.R.label[b] - (int64_t)A.first : -1;
            const RowInfo info = there ? A.R.info[b] : RowInfo{0.f, 0.f, 0.f, 0u};
            float own = 0.f;
#pragma unroll
            for (int i = 0; i < Tl::MA; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t a = a_of + 16 * i + q;
                    const float p = exp_of<T>(t.acc[i][j][q] * A.scale - info.lse) * info.factor;
                    const float g = there && a < A.words ? (label == (int64_t)a ? p - 1.f : p) * info.share : 0.f;
                    own = label == (int64_t)a ? g : own;
                    t.acc[i][j][q] = g;
                }
            const uint32_t d = (uint32_t)(label - (int64_t)a_of);
            if (label >= 0 && d < 16 * Tl::MA && (d & 15u) < 4) A.R.lost[b] = own - (float)(T)own;
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    if (A.g)
        t.rows([&](int i, int j) { return LOSS ? t.acc[i][j] * A.room : t.acc[i][j]; },
               [&](uint32_t a, uint32_t b, const Vec<uint32_t, 4> &w) {
                   if (b0 + b < n) *(Vec<uint32_t, 4> *)((T *)A.g + (uint64_t)(b0 + b) * A.g_stride + a0 + a) = w;
               });
}

// What the loss left of a piece becomes its gradients: each tile's words had their own largest logit.  A workgroup takes rows of 2,048 words.
// (In 16 bits these gradients are rounded twice, the others once: a step of half a unit more in an element of a sum over all words or rows, whose own
// rounding is as large; the label's comes from its logit in 32 bits.)
struct ScaleArgs {
    Rows R;
    const float2 *parts;
    uint64_t parts_stride, g_stride;
    void *g;
    uint32_t first, words, part;
    float room;
};
template <typename T> __global__ __launch_bounds__(256) void k_head_scale(const ScaleArgs A) {
    constexpr uint32_t EACH = 16 / sizeof(T);
    const uint32_t n = A.R.count[0], a = (blockIdx.x * 256u + threadIdx.x) * EACH;
    if (a >= A.words) return;                               // (words behind the piece's last are zeros already)
    for (uint32_t b = blockIdx.y; b < n; b += gridDim.y) {
        const RowInfo info = A.R.info[b];
        const int64_t label = (int64_t)A.R.label[b] - (int64_t)A.first - (int64_t)a;
        const float top = A.parts[(uint64_t)(a / A.part) * A.parts_stride + b].x;
        const float f = exp_f32((top == -INFINITY ? 0.f : top) - info.lse) * info.factor * (1.f / A.room);
        Vec<uint32_t, 4> *const at = (Vec<uint32_t, 4> *)((T *)A.g + (uint64_t)b * A.g_stride + a);
        const Vec<uint32_t, 4> w = *at;
        Vec<T, EACH> v;
#pragma unroll
        for (uint32_t e = 0; e < EACH; ++e) v[e] = (T)(element<T>(w, e) * f * info.share);
        if (label >= 0 && label < (int64_t)EACH) {          // (the label's logit is there in 32 bits)
            const float own = (exp_f32(A.R.label_logit[b] - info.lse) * info.factor - 1.f) * info.share;
#pragma unroll
            for (uint32_t e = 0; e < EACH; ++e) v[e] = label == (int64_t)e ? (T)own : v[e];
            A.R.lost[b] = own - (float)(T)own;
        }
        *at = __builtin_bit_cast(Vec<uint32_t, 4>, v);
    }
}

struct JoinArgs {
    Rows R;
    const float2 *parts;
    uint64_t parts_stride;
    uint32_t n_parts;
    bool first, last;           // of the pieces
    float z_weight;
    float *loss, *lse;
};
// 64 lanes a row: a row's parts in as many runs, joined in fixed order
constexpr uint32_t HD_RUNS = 64;
__global__ __launch_bounds__(16 * HD_RUNS) void k_head_join(const JoinArgs A) {
    __shared__ float2 runs[HD_RUNS][16];
    const uint32_t n = A.R.count[0];
    const uint32_t x = threadIdx.x & 15u, y = threadIdx.x >> 4;
    const uint32_t i = blockIdx.x * 16u + x;
    auto add = [](float &m, float &s, float2 o) {
        const float top = fmaxf(m, o.x), from = top == -INFINITY ? 0.f : top;
        s = s * exp_f32(m - from) + o.y * exp_f32(o.x - from);
        m = top;
    };
    if (blockIdx.x * 16u >= n) return;
    float m = -INFINITY, s = 0.f;
    if (i < n) {
        const uint32_t each = (A.n_parts + HD_RUNS - 1) / HD_RUNS, end = min(A.n_parts, (y + 1) * each);
        for (uint32_t p = y * each; p < end; ++p) add(m, s, A.parts[(uint64_t)p * A.parts_stride + i]);
    }
    runs[y][x] = make_float2(m, s);
    for (uint32_t d = HD_RUNS / 2; d; d /= 2) {
        __syncthreads();
        if (y < d) {
            add(m, s, runs[y + d][x]);
            runs[y][x] = make_float2(m, s);
        }
    }
    if (y || i >= n) return;
    if (!A.first) add(m, s, make_float2(A.R.top[i], A.R.sum[i]));
    A.R.top[i] = m; A.R.sum[i] = s;
    if (!A.last) return;
    const float lse = m + logf(s), loss = lse - A.R.label_logit[i] + A.z_weight * lse * lse;
    A.loss[A.R.row[i]] = loss;
    A.lse[A.R.row[i]] = lse;
}
// sums over one workgroup, every thread's part in fixed order
__device__ __forceinline__ double block_sum(double v, double *lds) {
    lds[threadIdx.x] = v;
    __syncthreads();
    for (uint32_t d = HD_THREADS / 2; d; d /= 2) {
        if (threadIdx.x < d) lds[threadIdx.x] += lds[threadIdx.x + d];
        __syncthreads();
    }
    return lds[0];
}
// 2^n with 2^n >= v (1 for what is no positive finite number)
__device__ __forceinline__ float power_above(float v) {
    if (!(v > 0.f) || !(v < 1e38f)) return 1.f;
    int e;
    const float m = frexpf(v, &e);
    return ldexpf(1.f, m == 0.5f ? e - 1 : e);
}
// What one workgroup does behind the loss: the total (null: there was none), and, with room > 0, the numbers that g is made with; room: what g's
// largest element may be (a power of two).  own_units: rows whose gradients are below a 64th of the largest row's are made under a unit of their own, so that
// float16 keeps them for dx whatever other rows weigh; others share the largest, and need no k_head_shared.
struct EndArgs {
    Rows R;
    const float *loss, *lse;
    float *total;
    float z_weight, room;
    bool own_units;
};
__global__ __launch_bounds__(HD_THREADS) void k_head_end(const EndArgs A) {
    __shared__ double lds[HD_THREADS];
    const uint32_t n = A.R.count[0];
    if (A.total) {
        double v = 0.0;
        for (uint32_t i = threadIdx.x; i < n; i += HD_THREADS) v += (double)A.R.weight[i] * (double)A.loss[A.R.row[i]];
        v = block_sum(v, lds);
        if (threadIdx.x == 0) *A.total = (float)v;
    }
    if (!(A.room > 0.f)) return;
    float most = 0.f;
    for (uint32_t i = threadIdx.x; i < n; i += HD_THREADS) {
        const float factor = 1.f + 2.f * A.z_weight * A.lse[A.R.row[i]], v = fabsf(A.R.weight[i]) * fmaxf(1.f, fabsf(factor));
        if (v < 1e38f) most = fmaxf(most, v);
    }
    __syncthreads();
    float *const tops = (float *)lds;
    tops[threadIdx.x] = most;
    __syncthreads();
    for (uint32_t d = HD_THREADS / 2; d; d /= 2) {
        if (threadIdx.x < d) tops[threadIdx.x] = fmaxf(tops[threadIdx.x], tops[threadIdx.x + d]);
        __syncthreads();
    }
    const float unit = power_above(tops[0]);
    if (threadIdx.x == 0) A.R.count[1] = __float_as_uint(unit);
    for (uint32_t i = threadIdx.x; i < n; i += HD_THREADS) {
        const float lse = A.lse[A.R.row[i]], factor = 1.f + 2.f * A.z_weight * lse, own = power_above(fabsf(A.R.weight[i]) * fmaxf(1.f, fabsf(factor)));
        const float of = A.own_units && own < unit * 0.015625f ? own : unit;
        A.R.info[i] = RowInfo{lse, factor, A.R.weight[i] / of * A.room, of};
    }
}

// d_weight sums over rows, under one unit: those that had their own are brought to the largest (exactly, but for what is then below float16's smallest).  A
// workgroup's second index is its row; most have nothing to do but the label's.
template <typename T> __global__ __launch_bounds__(256) void k_head_shared(Rows R, T *g, uint64_t g_stride, uint32_t first, uint32_t words) {
    constexpr uint32_t EACH = 16 / sizeof(T);
    const uint32_t n = R.count[0];
    const float largest = __uint_as_float(R.count[1]);
    for (uint32_t b = blockIdx.y; b < n; b += gridDim.y) {
        const float down = R.info[b].unit / largest;
        const int64_t label = (int64_t)R.label[b] - (int64_t)first;
        if (down == 1.f) {
            if (blockIdx.x == 0 && threadIdx.x == 0) R.lost_dw[b] = R.lost[b];
            continue;
        }
        for (uint32_t a = (blockIdx.x * 256u + threadIdx.x) * EACH; a < words; a += gridDim.x * 256u * EACH) {
            Vec<uint32_t, 4> *const at = (Vec<uint32_t, 4> *)(g + (uint64_t)b * g_stride + a);
            const Vec<uint32_t, 4> w = *at;
            Vec<T, EACH> v;
#pragma unroll
            for (uint32_t e = 0; e < EACH; ++e) {
                const bool own = label == (int64_t)(a + e);
                const float x = (element<T>(w, e) + (own ? R.lost[b] : 0.f)) * down;
                v[e] = (T)x;
                if (own) R.lost_dw[b] = x - (float)v[e];
            }
            *at = __builtin_bit_cast(Vec<uint32_t, 4>, v);
        }
    }
}

struct OutArgs {
    Rows R;
    Side A, B;
    uint32_t tiles_b, ks;
    uint32_t splits;
    float *sums;                // dx: [splits][rows][stride]
    uint64_t stride, split_stride;
    bool first;
    void *out;                  // d_weight
    uint32_t width, words, word0;
    const float *d_total;
    float scale, room;
};
// dx: sums over the piece's words, one share of them a split, added to those of the pieces before
template <typename T, int TA, int TB, int WA> __global__ __launch_bounds__(GM_THREADS) void k_head_dx(const OutArgs A) {
    typedef Tile<T, TA, TB, WA, ACROSS, ALONG> Tl;
    const uint32_t n = A.R.count[0];
    const uint32_t i = in_runs(blockIdx.x, gridDim.x), tiles = gridDim.x / A.splits, split = i / tiles;
    const Turn at_turn = turn_of(i - split * tiles, tiles / A.tiles_b, A.tiles_b);
    const uint32_t a0 = at_turn.a * TA, b0 = at_turn.b * TB;
    if (b0 >= n) return;
    Side B = A.B;
    B.count = n;
    const uint32_t turns = (A.ks + Tl::GRAIN - 1) / Tl::GRAIN;
    const uint32_t from = (uint32_t)((uint64_t)turns * split / A.splits) * Tl::GRAIN, to = (uint32_t)((uint64_t)turns * (split + 1) / A.splits) * Tl::GRAIN;
    Tl t;
    t.run(A.A, B, a0, b0, from, (to < A.ks ? to : A.ks) - from);
    const typename Tl::At at = Tl::place();
    const uint32_t a_of = a0 + at.a, b_of = b0 + at.b;
#pragma unroll
    for (int j = 0; j < Tl::MB; ++j)
#pragma unroll
        for (int i = 0; i < Tl::MA; ++i) {
            const uint32_t a = a_of + 16 * i, b = b_of + 16 * j;
            if (b >= n || a >= A.stride) continue;
            Vec<float, 4> *const to = (Vec<float, 4> *)(A.sums + split * A.split_stride + (uint64_t)b * A.stride + a);
            *to = A.first ? t.acc[i][j] : *to + t.acc[i][j];
        }
}
// a lane four columns of a row, a workgroup's first index its columns
template <typename T> __global__ __launch_bounds__(256) void k_head_dx_out(const OutArgs A, const T *weight, uint64_t w_st, T *dx, uint64_t dx_st, uint64_t n_rows) {
    const uint32_t c = (blockIdx.x * 256u + threadIdx.x) * 4u;
    if (c >= A.width) return;
    for (uint64_t r = blockIdx.y; r < n_rows; r += gridDim.y) {
        const int32_t i = A.R.place[r];
        Vec<float, 4> v = 0.f;
        if (i >= 0) {
            if constexpr (sizeof(T) == 2) {
                const T *const own = weight + (uint64_t)A.R.label[i] * w_st + c;
                const float lost = A.R.lost[i];
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e) v[e] = c + e < A.width ? lost * (float)own[e] : 0.f;
            }
            const float *const from = A.sums + (uint64_t)i * A.stride + c;
#pragma unroll 8
            for (uint32_t s = 0; s < A.splits; ++s) v += *(const Vec<float, 4> *)(from + s * A.split_stride);
            v *= (A.d_total ? *A.d_total : 1.f) * A.scale * (A.R.info[i].unit / A.room);
        }
        T *const to = dx + r * dx_st + c;
        if (c + 4 <= A.width) {
            *(Loose<Words<T, 4>, T> *)to = words_of<T, 4>({v[0], v[1], v[2], v[3]});
        } else {
#pragma unroll
            for (uint32_t e = 0; e < 3; ++e) if (c + e < A.width) to[e] = (T)v[e];
        }
    }
}
template <typename T, int TA, int TB, int WA> __global__ __launch_bounds__(GM_THREADS) void k_head_dw(const OutArgs A) {
    typedef Tile<T, TA, TB, WA, ACROSS, ACROSS> Tl;
    const uint32_t n = A.R.count[0];
    const Turn at_turn = turn_of(in_runs(blockIdx.x, gridDim.x), gridDim.x / A.tiles_b, A.tiles_b);
    const uint32_t a0 = at_turn.a * TA, b0 = at_turn.b * TB;
    Tl t;
    t.run(A.A, A.B, a0, b0, 0, n);
    if constexpr (sizeof(T) == 2) {
        // What rounding took off the labels of the tile: rows are looked through in order, 2,048 at a time, and those whose label lies in the tile make
        // further steps, 32 of them each, as their x and a side that has one element of each k: what was lost, rounded to the rows' type itself (the
        // label's gradient then has a 512th of its rounding, of float16 a 4,096th).  A tile takes as many steps as its labels are, however they lie.
        constexpr uint32_t EVERY = 4, KS = GM_STEP / sizeof(T), EL = 16 / sizeof(T), PA = TA / EL, PB = TB / EL;
        uint32_t *const found = (uint32_t *)t.shared, *const counts = found + EVERY * GM_THREADS;
        static_assert((EVERY * GM_THREADS + EVERY * GM_WAVES) * 4 <= TB * GM_STEP, "");
        const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        for (uint32_t begin = 0; begin < n; begin += EVERY * GM_THREADS) {
            uint32_t v[EVERY], before[EVERY];
            uint64_t hits[EVERY];
#pragma unroll
            for (uint32_t e = 0; e < EVERY; ++e) {
                const uint32_t r = begin + e * GM_THREADS + threadIdx.x;
                v[e] = r < n ? (uint32_t)A.R.label[r] - A.word0 - b0 : ~0u;
                hits[e] = __builtin_amdgcn_ballot_w64(v[e] < (uint32_t)TB);
                before[e] = (uint32_t)__popcll(hits[e] & ((1ull << lane) - 1ull));
                if (lane == 0) counts[e * GM_WAVES + wave] = (uint32_t)__popcll(hits[e]);
            }
            __syncthreads();
            uint32_t all = 0;
#pragma unroll
            for (uint32_t e = 0; e < EVERY; ++e)
#pragma unroll
                for (uint32_t w = 0; w < GM_WAVES; ++w) {
                    if (w == wave && v[e] < (uint32_t)TB) found[all + before[e]] = (begin + e * GM_THREADS + threadIdx.x) << 8 | v[e];
                    all += counts[e * GM_WAVES + w];
                }
            __syncthreads();
            for (uint32_t step = 0; step < all; step += KS) {
                for (uint32_t i = threadIdx.x; i < KS * PA; i += GM_THREADS) {
                    const uint32_t k = i / PA, piece = i % PA;
                    Vec<uint32_t, 4> w = 0u;
                    if (step + k < all && a0 * sizeof(T) + piece * 16 < A.A.count)
                        w = *(const Vec<uint32_t, 4> *)(A.A.data + (uint64_t)(found[step + k] >> 8) * A.A.stride + a0 * sizeof(T) + piece * 16);
                    *(Vec<uint32_t, 4> *)(t.step_a + k * (TA * sizeof(T)) + (piece ^ order_of<T, PA>(k)) * 16) = w;
                }
                for (uint32_t i = threadIdx.x; i < KS * PB; i += GM_THREADS) {
                    const uint32_t k = i / PB, piece = i % PB, of = step + k < all ? found[step + k] : 0u;
                    Vec<T, EL> w = (T)0.f;
                    if (step + k < all && (of & 255u) / EL == piece) {
                        const T lost = (T)A.R.lost[of >> 8];
#pragma unroll
                        for (uint32_t e = 0; e < EL; ++e) w[e] = (of & 255u) % EL == e ? lost : (T)0.f;
                    }
                    *(Vec<T, EL> *)(t.step_b + k * (TB * sizeof(T)) + (piece ^ order_of<T, PB>(k)) * 16) = w;
                }
                __syncthreads();
                t.step_alone();
                __syncthreads();
            }
        }
    }
    const float f = n ? (A.d_total ? *A.d_total : 1.f) * A.scale * (__uint_as_float(A.R.count[1]) / A.room) : 0.f;
    constexpr uint32_t EACH = 16 / sizeof(T);
    T *const out = (T *)A.out;
    t.rows([&](int i, int j) { return n ? t.acc[i][j] * f : Vec<float, 4>(0.f); },
           [&](uint32_t a, uint32_t b, const Vec<uint32_t, 4> &w) {
               if (b0 + b >= A.words) return;
               T *const to = out + (uint64_t)(b0 + b) * A.stride + a0 + a;
               if (a0 + a + EACH <= A.width) {
                   __builtin_nontemporal_store(w, (Loose<Vec<uint32_t, 4>, T> *)to);
               } else {
                   const Vec<T, EACH> v = __builtin_bit_cast(Vec<T, EACH>, w);
#pragma unroll
                   for (uint32_t e = 0; e < EACH; ++e) if (a0 + a + e < A.width) to[e] = v[e];
               }
           });
}

// ---- host
struct Call {
    const rk_head *head;
    uint64_t n_rows;
    uint32_t width, vocab;
    const rk_matrix *x, *weight;
    const int32_t *label;
    const float *row_weight, *d_total;
    float *loss, *lse, *total;
    const rk_matrix *dx, *d_weight;
    const float *given_lse;
};
// f(rows of a tile, wavefronts along its words)
template <typename T, typename F> void with_rows(uint32_t tile, F f) {
    if (tile == 32) f(std::integral_constant<int, 32>(), std::integral_constant<int, 8>());
    else if (tile == 64) f(std::integral_constant<int, 64>(), std::integral_constant<int, 8>());
    else if (tile == 128) f(std::integral_constant<int, 128>(), std::integral_constant<int, 4>());
    else if (tile == 256) f(std::integral_constant<int, 256>(), std::integral_constant<int, 2>());
    else if constexpr (sizeof(T) == 4) f(std::integral_constant<int, 192>(), std::integral_constant<int, 2>());
}
// Rows of a tile.  Few take small tiles, which leave LDS for two workgroups a compute unit (5 x 128000 x 5248: 258 us, with tiles of 256 rows 368).
// More of 16 bits take the largest, even where it is half empty (300 x 64000 x 4096: 238 us, of 192 rows 244, of 128 rows 263); of 32 bits, where only
// the matrix units' time counts, the one that has the fewest rows in all turns of the compute units (300 x 64000 x 4096: 1,867, 1,451 and 1,420 us).  Neither is
// made for vocabularies of fewer tiles than compute units, which leave many of these without work (1000 x 1000 x 1000 in 16 bits, loss and gradients: 128 us).
template <typename T> uint32_t rows_of_tile(uint64_t n_rows, uint64_t tiles_a) {
    if (n_rows <= 128) return n_rows <= 32 ? 32 : n_rows <= 64 ? 64 : 128;
    uint32_t best = 256;
    if (sizeof(T) == 4) {
        auto cost = [&](uint64_t tile) { return (tiles_a * ((n_rows + tile - 1) / tile) + 255) / 256 * tile; };
        for (uint32_t tile : {192u, 128u}) if (cost(tile) < cost(best)) best = tile;
    }
    return best;
}
uint64_t up_to(uint64_t v, uint64_t m) { return (v + m - 1) / m * m; }
uint32_t blocks_of(uint64_t n) { return (uint32_t)(n < (1u << 20) ? n : 1u << 20); }

template <typename T> int32_t run_typed(rk_ctx *ctx, const Call &C) {
    constexpr uint32_t ES = sizeof(T), STEP = 128 / ES;
    const hipStream_t stream = ctx->stream;
    const uint32_t wide = (uint32_t)up_to(C.width, STEP);
    const uint64_t rows_pad = up_to(C.n_rows, 256);
    int32_t rc;
    Rows R{};
    {
        char *p;
        if ((rc = rk_scratch(ctx, SL_HEAD_ROWS, 256 + rows_pad * (9 * 4 + sizeof(RowInfo)), (void **)&p)) != RK_OK) return rc;
        R.count = (uint32_t *)p; p += 256;
        R.info = (RowInfo *)p; p += rows_pad * sizeof(RowInfo);
        R.row = (int32_t *)p; p += rows_pad * 4;
        R.place = (int32_t *)p; p += rows_pad * 4;
        R.label = (int32_t *)p; p += rows_pad * 4;
        R.weight = (float *)p; p += rows_pad * 4;
        R.label_logit = (float *)p; p += rows_pad * 4;
        R.top = (float *)p; p += rows_pad * 4;
        R.sum = (float *)p; p += rows_pad * 4;
        R.lost = (float *)p; p += rows_pad * 4;
        R.lost_dw = (float *)p;
    }
    T *xc;
    if ((rc = rk_scratch(ctx, SL_HEAD_X, C.n_rows * wide * ES, (void **)&xc)) != RK_OK) return rc;
    k_head_rows<<<1, HD_THREADS, 0, stream>>>(RowsArgs{R, C.label, C.row_weight, C.loss, C.lse, C.n_rows, C.vocab});
    RK_CHECK_LAUNCH(ctx, "k_head_rows");
    if (C.n_rows) {
        k_head_pad<T><<<blocks_of((C.n_rows * wide * ES / 16 + 255) / 256), 256, 0, stream>>>(R.row, R.count, 0, (const T *)C.x->data, C.x->stride, C.width, xc, wide);
        RK_CHECK_LAUNCH(ctx, "k_head_pad");
    }
    const Side X = {(const char *)xc, (uint64_t)wide * ES, 0};
    const T *const w = (const T *)C.weight->data;
    const uint64_t w_st = C.weight->stride;
    // rows of W go into the product as they lie where their vectors do not straddle; others are padded first, piece by piece
    const bool direct = ((uintptr_t)w % 16 == 0 && w_st * ES % 16 == 0 && (uint64_t)C.width * ES % 16 == 0 && w_st * ES * 256 < GM_NOWHERE);
    const uint32_t tile_b = rows_of_tile<T>(C.n_rows, (C.vocab + 255) / 256);
    const uint32_t tiles_b = (uint32_t)((C.n_rows + tile_b - 1) / tile_b);
    const uint64_t most_tiles = (1u << 22) / (tiles_b ? tiles_b : 1);
    const bool back = C.dx || C.d_weight;
    // words of a piece: what the budget holds of their gradients, of W padded, and of the sums of tiles
    uint64_t words = up_to(C.vocab, 256);
    const uint64_t each = (back ? rows_pad * ES : 0) + (direct ? 0 : (uint64_t)wide * ES), sums_each = C.total ? rows_pad * 8 / HD_TA : 0;
    if (each && HD_BUDGET / each < words) words = HD_BUDGET / each / 256 * 256;
    if (sums_each && HD_PARTS / sums_each < words) words = HD_PARTS / sums_each / 256 * 256;
    if (words > most_tiles * 256) words = most_tiles * 256;
    if (words < 256) words = 256;
    T *padded = nullptr;
    if (!direct && (rc = rk_scratch(ctx, SL_HEAD_W, words * wide * ES, (void **)&padded)) != RK_OK) return rc;
    // the piece from word `first` on
    uint32_t n_words = 0;
    Side W{};
    auto piece = [&](uint64_t first) -> int32_t {
        n_words = (uint32_t)(C.vocab - first < words ? C.vocab - first : words);
        if (direct) {
            W = Side{(const char *)(w + first * w_st), w_st * ES, 0};
            return RK_OK;
        }
        k_head_pad<T><<<blocks_of(((uint64_t)n_words * wide * ES / 16 + 255) / 256), 256, 0, stream>>>(nullptr, nullptr, n_words, w + first * w_st, w_st, C.width, padded, wide);
        RK_CHECK_LAUNCH(ctx, "k_head_pad");
        W = Side{(const char *)padded, (uint64_t)wide * ES, 0};
        return RK_OK;
    };
    // float16 has 30 powers of two between one and its smallest: what is at most one is moved up by fourteen
    const float room = __is_same(T, _Float16) ? 16384.f : 1.f;
    const bool own_units = __is_same(T, _Float16) && C.dx;
    LogitsArgs L{};
    L.R = R; L.X = X; L.width = C.width; L.tiles_b = tiles_b; L.scale = C.head->logit_scale; L.room = room;
    if (back && (rc = rk_scratch(ctx, SL_HEAD_G, rows_pad * words * ES, (void **)&L.g)) != RK_OK) return rc;
    L.g_stride = words;
    void *const g = L.g;
    const uint64_t last_piece = (C.vocab - 1) / words * words;

    if (C.total) {
        if ((rc = rk_scratch(ctx, SL_HEAD_PARTS, words * sums_each, (void **)&L.parts)) != RK_OK) return rc;
        L.parts_stride = rows_pad;
        JoinArgs J{R, L.parts, rows_pad, 0, false, false, C.head->z_weight, C.loss, C.lse};
        for (uint64_t first = 0; first < C.vocab && C.n_rows; first += words) {
            if ((rc = piece(first)) != RK_OK) return rc;
            L.first = (uint32_t)first; L.words = n_words;
            L.W = W; L.W.count = n_words;
            L.g = first == last_piece ? g : nullptr;
            const uint32_t tiles_a = (n_words + 255) / 256;
            with_rows<T>(tile_b, [&](auto tb, auto wa) {
                k_head_logits<T, HD_TA, decltype(tb)::value, decltype(wa)::value, true><<<tiles_a * tiles_b, GM_THREADS, 0, stream>>>(L);
            });
            RK_CHECK_LAUNCH(ctx, "k_head_logits");
            J.n_parts = tiles_a;
            J.first = first == 0; J.last = first == last_piece;
            k_head_join<<<(uint32_t)((C.n_rows + 15) / 16), 16 * HD_RUNS, 0, stream>>>(J);
            RK_CHECK_LAUNCH(ctx, "k_head_join");
        }
    }
    k_head_end<<<1, HD_THREADS, 0, stream>>>(EndArgs{R, C.loss, C.given_lse ? C.given_lse : C.lse, C.total, C.head->z_weight, back ? room : 0.f, own_units});
    RK_CHECK_LAUNCH(ctx, "k_head_end");
    if (!back) return RK_OK;
    const uint32_t tiles_w = (uint32_t)((C.width + 255) / 256);
    OutArgs O{};
    O.R = R; O.d_total = C.d_total; O.scale = C.head->logit_scale; O.room = room; O.width = C.width;
    if (C.dx) {
        // the words in as many shares as leave the fewest compute units idle in the last turn; none shorter than 1,024 words
        const uint64_t tiles = (uint64_t)tiles_w * (tiles_b ? tiles_b : 1);
        double best = 0.0;
        for (uint32_t n = 1; n <= 64 && n <= words / 1024 + 1; ++n) {
            const uint64_t turns = (tiles * n + 255) / 256;
            const double filled = (double)(tiles * n) / (double)(turns * 256) * (1.0 - 0.002 * n);
            if (filled > best) { best = filled; O.splits = n; }
        }
        O.stride = up_to(C.width, 4);
        O.split_stride = C.n_rows * O.stride;
        if ((rc = rk_scratch(ctx, SL_HEAD_DX, O.splits * O.split_stride * 4, (void **)&O.sums)) != RK_OK) return rc;
    }
    const uint64_t row_bytes = direct ? (uint64_t)C.width * ES : (uint64_t)wide * ES;
    L.g = g;
    for (uint64_t first = last_piece;; first -= words) {
        if ((rc = piece(first)) != RK_OK) return rc;        // (padded once more where the loss has been through all pieces)
        const uint32_t tiles_a = (n_words + 255) / 256;
        if (C.n_rows && C.total && first == last_piece) {
            const uint32_t across = (n_words + 256 * 16 / ES - 1) / (256 * 16 / ES);
            k_head_scale<T><<<dim3(across, (uint32_t)(C.n_rows < 4096 ? C.n_rows : 4096)), 256, 0, stream>>>(
                ScaleArgs{R, L.parts, rows_pad, words, g, (uint32_t)first, n_words, HD_TA, room});
            RK_CHECK_LAUNCH(ctx, "k_head_scale");
        } else if (C.n_rows) {
            L.first = (uint32_t)first; L.words = n_words;
            L.W = W; L.W.count = n_words;
            with_rows<T>(tile_b, [&](auto tb, auto wa) {
                k_head_logits<T, HD_TA, decltype(tb)::value, decltype(wa)::value, false><<<tiles_a * tiles_b, GM_THREADS, 0, stream>>>(L);
            });
            RK_CHECK_LAUNCH(ctx, "k_head_logits");
        }
        if (C.dx && C.n_rows) {
            O.A = W; O.A.count = row_bytes;
            O.B = Side{(const char *)g, words * ES, 0};
            O.ks = n_words; O.tiles_b = tiles_b; O.first = first == last_piece;
            with_rows<T>(tile_b, [&](auto tb, auto wa) {
                k_head_dx<T, HD_TA, decltype(tb)::value, decltype(wa)::value><<<tiles_w * tiles_b * O.splits, GM_THREADS, 0, stream>>>(O);
            });
            RK_CHECK_LAUNCH(ctx, "k_head_dx");
        }
        if (C.d_weight) {
            OutArgs D = O;
            if constexpr (__is_same(T, _Float16)) {
                if (own_units && C.n_rows) {
                    const uint32_t across = (n_words + 2047) / 2048;
                    k_head_shared<T><<<dim3(across < 4 ? across : 4, (uint32_t)(C.n_rows < 4096 ? C.n_rows : 4096)), 256, 0, stream>>>(R, (T *)g, words, (uint32_t)first, n_words);
                    RK_CHECK_LAUNCH(ctx, "k_head_shared");
                    D.R.lost = R.lost_dw;
                }
            }
            D.A = X; D.A.count = (uint64_t)wide * ES;
            D.B = Side{(const char *)g, words * ES, words * ES};
            D.tiles_b = tiles_a; D.words = n_words; D.word0 = (uint32_t)first;
            D.out = (T *)C.d_weight->data + first * C.d_weight->stride; D.stride = C.d_weight->stride;
            // (tiles of 64 words, two workgroups a compute unit, were slower for few rows too: 5 x 128000 x 5248 566 instead of 436 us)
            k_head_dw<T, HD_TA, 256, 2><<<tiles_w * tiles_a, GM_THREADS, 0, stream>>>(D);
            RK_CHECK_LAUNCH(ctx, "k_head_dw");
        }
        if (first == 0) break;
    }
    if (C.dx && C.n_rows) {
        k_head_dx_out<T><<<dim3((C.width + 1023) / 1024, (uint32_t)(C.n_rows < 32768 ? C.n_rows : 32768)), 256, 0, stream>>>(O, w, w_st, (T *)C.dx->data, C.dx->stride, C.n_rows);
        RK_CHECK_LAUNCH(ctx, "k_head_dx_out");
    }
    return RK_OK;
}

bool misaligned4(std::initializer_list<const void *> ps) {
    for (const void *p : ps) if (((uintptr_t)p & 3u)) return true;
    return false;
}

int32_t run_head(rk_ctx *ctx, const Call &C, bool loss, bool back) {
    if (!ctx) return RK_ERR_INVALID_ARG;
    if (!C.head || !(C.head->z_weight >= 0.f) || !(C.head->z_weight < INFINITY) || !(fabsf(C.head->logit_scale) < INFINITY) || C.head->logit_scale == 0.f)
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "head is null, its z_weight negative or not finite, or its logit_scale 0 or not finite");
    if (C.width < 1 || C.vocab < 1) return rk_fail(ctx, RK_ERR_INVALID_ARG, "rows or the vocabulary are empty");
    if (C.width > RK_HEAD_MAX_WIDTH || C.vocab > (1u << 28) || C.n_rows > (1ull << 20))
        return rk_fail(ctx, RK_ERR_UNSUPPORTED, "more than 2^20 rows, 2^28 words or %u columns", RK_HEAD_MAX_WIDTH);
    if (!rk_matrix_ok(C.x, C.n_rows, C.width) || !rk_matrix_ok(C.weight, C.vocab, C.width))
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "x or weight null, misaligned or of a stride below the width");
    if (C.x->type != C.weight->type) return rk_fail(ctx, RK_ERR_INVALID_ARG, "weight has another type than x");
    if ((C.n_rows && !C.label) || misaligned4({C.label, C.row_weight})) return rk_fail(ctx, RK_ERR_INVALID_ARG, "label null, or it or row_weight misaligned");
    if (loss && ((C.n_rows && (!C.loss || !C.lse)) || !C.total || misaligned4({C.loss, C.lse, C.total})))
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "loss, lse or total null or misaligned");
    if (back) {
        if (!C.dx && !C.d_weight) return rk_fail(ctx, RK_ERR_INVALID_ARG, "no gradient is wanted");
        if ((C.dx && (!rk_matrix_ok(C.dx, C.n_rows, C.width) || C.dx->type != C.x->type)) ||
            (C.d_weight && (!rk_matrix_ok(C.d_weight, C.vocab, C.width) || C.d_weight->type != C.x->type)))
            return rk_fail(ctx, RK_ERR_INVALID_ARG, "dx or d_weight misaligned, of a stride below the width or of another type than x");
        if ((!loss && C.n_rows && !C.given_lse) || misaligned4({C.given_lse, C.d_total})) return rk_fail(ctx, RK_ERR_INVALID_ARG, "lse null, or it or d_total misaligned");
    }
    RK_HIP(ctx, hipSetDevice(ctx->device));
    if (C.x->type == RK_F32) return run_typed<float>(ctx, C);
    if (C.x->type == RK_BF16) return run_typed<__bf16>(ctx, C);
    return run_typed<_Float16>(ctx, C);
}

}  // namespace

extern "C" int32_t rk_head_loss(rk_ctx *ctx, const rk_head *head, uint64_t n_rows, uint32_t width, uint32_t vocab, const rk_matrix *x,
                                const rk_matrix *weight, const int32_t *label, const float *row_weight, float *loss, float *lse,
                                float *total) {
    return run_head(ctx, Call{head, n_rows, width, vocab, x, weight, label, row_weight, nullptr, loss, lse, total, nullptr, nullptr, nullptr}, true, false);
}

extern "C" int32_t rk_head_backward(rk_ctx *ctx, const rk_head *head, uint64_t n_rows, uint32_t width, uint32_t vocab, const rk_matrix *x,
                                    const rk_matrix *weight, const int32_t *label, const float *row_weight, const float *lse,
                                    const float *d_total, const rk_matrix *dx, const rk_matrix *d_weight) {
    return run_head(ctx, Call{head, n_rows, width, vocab, x, weight, label, row_weight, d_total, nullptr, nullptr, nullptr, dx, d_weight, lse}, false, true);
}

extern "C" int32_t rk_head_loss_backward(rk_ctx *ctx, const rk_head *head, uint64_t n_rows, uint32_t width, uint32_t vocab, const rk_matrix *x,
                                         const rk_matrix *weight, const int32_t *label, const float *row_weight, const float *d_total,
                                         float *loss, float *lse, float *total, const rk_matrix *dx, const rk_matrix *d_weight) {
    return run_head(ctx, Call{head, n_rows, width, vocab, x, weight, label, row_weight, d_total, loss, lse, total, dx, d_weight, nullptr}, true, true);
}
