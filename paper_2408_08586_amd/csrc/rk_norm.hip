// The join of a block and its residual stream: norm of the block's output, gate, scaled residual, norm before the next
// block, forward and backward (rk_norm_forward, rk_norm_backward).
#include <cmath>
#include <type_traits>

#include "rk_vec.h"

namespace {

enum { G_POST_W, G_POST_B, G_PRE_W, G_PRE_B, G_GATE, G_VECTORS };

struct NormArgs {
    const void *x, *y, *dxo, *du;       // forward: x; backward: x_out
    void *xo, *u;                       // forward: x_out, u; backward: dx, dy
    uint64_t x_st, y_st, dxo_st, du_st, xo_st, u_st;
    float *stats;
    const void *vec[G_VECTORS];
    uint64_t gate_rows, gate_st;
    uint64_t n_rows, first;             // first: the launch's first row
    uint32_t width;
    uint32_t post, pre, p32;            // p32: the vectors are float32
    float post_eps, pre_eps, scale;
    float4 *row_sums;                   // backward: per row, what its norms' gradients subtract
};

// ---- sums over a row, which `nw` wavefronts hold together
struct RowGroup {
    float *lds;                         // 3 x 16 floats for every exchange that may be under way
    uint32_t nw, wave, lane;
    uint32_t turn;                      // exchanges alternate between two places: one barrier each is enough
    __device__ __forceinline__ float *place() { return lds + 48 * (turn++ & 1u); }
    __device__ __forceinline__ void two(float &a, float &b) {
        a = wave_sum(a); b = wave_sum(b);
        if (nw == 1) return;
        float *const s = place();
        if (lane == 0) { s[wave] = a; s[16 + wave] = b; }
        __syncthreads();
        const uint32_t w = lane & 15u;
        a = row_sum(w < nw ? s[w] : 0.f);
        b = row_sum(w < nw ? s[16 + w] : 0.f);
    }
};

// a lane's part of a weight, bias or gate; `none` in each place if there is none
template <bool CUTS, typename T, int CH>
__device__ __forceinline__ void load_param(const NormArgs &A, int which, uint64_t row, uint64_t stride, const Place &p, float none, float (&v)[CH]) {
    const void *const base = A.vec[which];
    if (!base) {
#pragma unroll
        for (int i = 0; i < CH; ++i) v[i] = none;
    } else if (A.p32) {
        load_row<CUTS, float, CH>(Row<float>(base, row, stride, A.width), p, v);
    } else {
        load_row<CUTS, T, CH>(Row<T>(base, row, stride, A.width), p, v);
    }
}

// Mean and sum of squares about it of a lane's elements v(k, i).  Each wavefront takes its squares about its own mean, and the parts
// are joined by what the means differ: nothing is cancelled, and one exchange is enough.
template <int CH, int NC, typename V>
__device__ __forceinline__ void row_stats(RowGroup &G, V v, uint32_t width, const Place (&at)[NC], uint32_t how, float eps,
                                          float &mean, float &r) {
    mean = 0.f; r = 1.f;
    if (how == RK_NORM_NONE) return;
    if (how == RK_NORM_RMS) {
        float q = 0.f, none = 0.f;
#pragma unroll
        for (int k = 0; k < NC; ++k)
#pragma unroll
            for (int i = 0; i < CH; ++i) q += v(k, i) * v(k, i);
        G.two(q, none);
        r = 1.0f / sqrtf(q / (float)width + eps);
        return;
    }
    float s = 0.f, n = 0.f;
#pragma unroll
    for (int k = 0; k < NC; ++k) {
        const int32_t valid = at[k].valid;
        n += (float)(valid < 0 ? 0 : valid < CH ? valid : CH);
#pragma unroll
        for (int i = 0; i < CH; ++i) s += v(k, i);          // those behind the row's end are zero
    }
    s = wave_sum(s); n = wave_sum(n);
    const float own = n > 0.f ? s / n : 0.f;
    float q = 0.f;
#pragma unroll
    for (int k = 0; k < NC; ++k) {
#pragma unroll
        for (int i = 0; i < CH; ++i) { const float d = i < at[k].valid ? v(k, i) - own : 0.f; q += d * d; }
    }
    q = wave_sum(q);
    if (G.nw > 1) {
        float *const p = G.place();
        if (G.lane == 0) { p[G.wave] = s; p[16 + G.wave] = n; p[32 + G.wave] = q; }
        __syncthreads();
        const uint32_t w = G.lane & 15u;
        const float sw = w < G.nw ? p[w] : 0.f, nn = w < G.nw ? p[16 + w] : 0.f, qw = w < G.nw ? p[32 + w] : 0.f;
        mean = row_sum(sw) / (float)width;
        const float d = nn > 0.f ? sw / nn - mean : 0.f;
        q = row_sum(qw + nn * d * d);
    } else {
        mean = own;
    }
    r = 1.0f / sqrtf(q / (float)width + eps);
}

// A lane's vectors are its thread's number and those a stride further.  Only the last of them can be the one that the row's end cuts, since a
// row takes as few threads as hold it (in 32 bits, where vectors are taken in pairs, or the last but one, of narrow rows the first).
template <int CH, int NC> __device__ __forceinline__ void places(Place (&at)[NC], uint32_t tid, uint32_t threads, uint32_t width) {
#pragma unroll
    for (int k = 0; k < NC; ++k) {
        at[k] = Place((tid + k * threads) * CH, width, CH);
        if (k + 1 < NC && !(CH == 4 && (NC == 2 || (NC == 4 && k == 2)))) at[k].cut_here = false;
    }
}

// The rows of a workgroup: one (its wavefronts share it), or one per wavefront for rows that a wavefront holds.
struct RowOf { uint64_t row; uint32_t tid, threads; bool there; };
__device__ __forceinline__ RowOf row_of(uint64_t first, uint64_t n_rows, bool per_wave, RowGroup &G, float *lds) {
    const uint32_t t = threadIdx.x, waves = blockDim.x >> 6;
    G.lane = t & 63u; G.wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(t >> 6)); G.turn = 0; G.lds = lds;
    G.nw = per_wave ? 1u : waves;
    const uint64_t row = first + (per_wave ? (uint64_t)blockIdx.x * waves + G.wave : blockIdx.x);
    return RowOf{row, per_wave ? G.lane : t, per_wave ? 64u : blockDim.x, row < n_rows};
}

// What is behind the row's fetching, of rows of few whole vectors a lane: what the norms multiply and add is asked for before the sums are taken, all of
// it at once.  (Longer rows would pay for the registers with wavefronts: 8192 x 12288 149 us without, 187 with; 4096 x 2048 14.6 and 13.8.)
template <typename T, typename R, int CH, int NC>
__device__ __forceinline__ void forward_early(const NormArgs &A, const RowOf &P, RowGroup &G, const Place (&at)[NC], const Words<R, CH> (&wx)[NC], const Words<T, CH> (&wy)[NC]) {
    Words<T, CH> w[NC], b[NC], g[NC];
    auto ask = [&](int which, uint64_t row, uint64_t stride, Words<T, CH> (&v)[NC]) {
        const Row<T> of(A.vec[which], row, stride, A.width);                    // (zeros, if there is none)
#pragma unroll
        for (int k = 0; k < NC; ++k) v[k] = fetch_at<T, CH>(of, at[k].whole);
    };
    ask(G_POST_W, 0, 0, w); ask(G_GATE, A.gate_rows ? P.row / A.gate_rows : 0, A.gate_st, g); ask(G_POST_B, 0, 0, b);
    float my, ry, mx, rx;
    row_stats<CH, NC>(G, [&](int k, int i) { return element<T>(wy[k], i); }, A.width, at, A.post, A.post_eps, my, ry);
    const bool has_w1 = A.vec[G_POST_W] != nullptr, has_gate = A.vec[G_GATE] != nullptr, has_w2 = A.vec[G_PRE_W] != nullptr;
    float x[NC][CH];
    const Row<R> xo(A.xo, P.row, A.xo_st, A.width);
#pragma unroll
    for (int k = 0; k < NC; ++k) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const float n = (element<T>(wy[k], i) - my) * ry * (has_w1 ? element<T>(w[k], i) : 1.f) + element<T>(b[k], i);
            x[k][i] = i < at[k].valid ? A.scale * element<R>(wx[k], i) + (has_gate ? element<T>(g[k], i) : 1.f) * n : 0.f;
        }
        store_at<R, CH, STREAM>(xo, at[k].whole, words_of<R, CH>(x[k]));
    }
    ask(G_PRE_W, 0, 0, w); ask(G_PRE_B, 0, 0, b);
    row_stats<CH, NC>(G, [&](int k, int i) { return x[k][i]; }, A.width, at, A.pre, A.pre_eps, mx, rx);
    if (P.tid == 0) reinterpret_cast<float4 *>(A.stats)[P.row] = make_float4(my, ry, mx, rx);
    if (A.pre == RK_NORM_NONE) return;
    const Row<T> u(A.u, P.row, A.u_st, A.width);
#pragma unroll
    for (int k = 0; k < NC; ++k) {
#pragma unroll
        for (int i = 0; i < CH; ++i) x[k][i] = (x[k][i] - mx) * rx * (has_w2 ? element<T>(w[k], i) : 1.f) + element<T>(b[k], i);
        store_at<T, CH, STREAM>(u, at[k].whole, words_of<T, CH>(x[k]));
    }
}

// A row forward: all of it in registers between its one reading and its two results, so that both norms cost one pass.  Bound by HBM: 8192 x
// 12288 bfloat16 149 us, 805 MB, 5.4 TB/s; where all rows fit the chip at once, by one row's chain of loads and two exchanges: 1999 x 5003 float16
// 21 us, 3.8 TB/s.
template <bool CUTS, typename T, typename R, int CH, int NC, int MAXT>
__global__ __launch_bounds__(MAXT) void k_norm_forward(NormArgs A, bool per_wave) {
    __shared__ float lds[96];
    RowGroup G;
    const RowOf P = row_of(A.first, A.n_rows, per_wave, G, lds);
    if (!P.there) return;                                   // (per_wave only: whole wavefronts, no barrier follows)
    Place at[NC];
    places<CH, NC>(at, P.tid, P.threads, A.width);
    Words<R, CH> wx[NC];
    Words<T, CH> wy[NC];
    {
        const Row<T> ry(A.y, P.row, A.y_st, A.width);
        const Row<R> rx(A.x, P.row, A.x_st, A.width);
#pragma unroll
        for (int k = 0; k < NC; ++k) wy[k] = fetch_row<CUTS, T, CH>(ry, at[k]);
#pragma unroll
        for (int k = 0; k < NC; ++k) wx[k] = fetch_row<CUTS, R, CH>(rx, at[k]);
    }
    if constexpr (!CUTS && MAXT <= 512)
        if (sizeof(T) == 4 || !A.p32) {                     // (32-bit vectors beside narrow rows take too many registers: 4096 x 4096 26 us, early 28)
            forward_early<T, R, CH, NC>(A, P, G, at, wx, wy);
            return;
        }
    float my, ry, mx, rx;
    row_stats<CH, NC>(G, [&](int k, int i) { return element<T>(wy[k], i); }, A.width, at, A.post, A.post_eps, my, ry);
    float x[NC][CH];
    const uint64_t gate = A.gate_rows ? P.row / A.gate_rows : 0;
    const Row<R> xo(A.xo, P.row, A.xo_st, A.width);
#pragma unroll
    for (int k = 0; k < NC; ++k) {
        float w[CH], b[CH], g[CH];
        load_param<CUTS, T, CH>(A, G_POST_W, 0, 0, at[k], 1.f, w);
        load_param<CUTS, T, CH>(A, G_POST_B, 0, 0, at[k], 0.f, b);
        load_param<CUTS, T, CH>(A, G_GATE, gate, A.gate_st, at[k], 1.f, g);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const float n = (element<T>(wy[k], i) - my) * ry * w[i] + b[i];
            x[k][i] = i < at[k].valid ? A.scale * element<R>(wx[k], i) + g[i] * n : 0.f;
        }
        store_row<CUTS, R, CH, STREAM>(xo, at[k], x[k]);
    }
    row_stats<CH, NC>(G, [&](int k, int i) { return x[k][i]; }, A.width, at, A.pre, A.pre_eps, mx, rx);
    if (P.tid == 0) reinterpret_cast<float4 *>(A.stats)[P.row] = make_float4(my, ry, mx, rx);
    if (A.pre == RK_NORM_NONE) return;
    const Row<T> u(A.u, P.row, A.u_st, A.width);
#pragma unroll
    for (int k = 0; k < NC; ++k) {
        float w[CH], b[CH];
        load_param<CUTS, T, CH>(A, G_PRE_W, 0, 0, at[k], 1.f, w);
        load_param<CUTS, T, CH>(A, G_PRE_B, 0, 0, at[k], 0.f, b);
#pragma unroll
        for (int i = 0; i < CH; ++i) x[k][i] = (x[k][i] - mx) * rx * w[i] + b[i];
        store_row<CUTS, T, CH, STREAM>(u, at[k], x[k]);
    }
}

// One row back: D = dx_out + (what comes through the norm before the next block), dx = scale * D, and dy through gate and the
// block's own norm.  row_sums keeps what D takes off, for the sums over rows.  For calls that want no vector's gradient, and for rows that are too wide
// to keep sums beside them: then k_norm_sums reads everything once more (4096 x 16384 bfloat16: 287 us for both, bound by HBM).
template <bool CUTS, typename T, typename R, int CH, int NC, int MAXT>
__global__ __launch_bounds__(MAXT) void k_norm_backward(NormArgs A, bool per_wave) {
    __shared__ float lds[96];
    RowGroup G;
    const RowOf P = row_of(A.first, A.n_rows, per_wave, G, lds);
    if (!P.there) return;
    Place at[NC];
    places<CH, NC>(at, P.tid, P.threads, A.width);
    const float4 st = reinterpret_cast<const float4 *>(A.stats)[P.row];
    float d[NC][CH], hat[NC][CH];
    float c = 0.f, m = 0.f;
    if (A.pre != RK_NORM_NONE) {
        const Row<R> rx(A.x, P.row, A.x_st, A.width);
        const Row<T> ru(A.du, P.row, A.du_st, A.width);
#pragma unroll
        for (int k = 0; k < NC; ++k) {
            float w[CH];
            load_row<CUTS, R, CH>(rx, at[k], hat[k]);
            load_row<CUTS, T, CH>(ru, at[k], d[k]);
            load_param<CUTS, T, CH>(A, G_PRE_W, 0, 0, at[k], 1.f, w);
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                hat[k][i] = (hat[k][i] - st.z) * st.w;
                d[k][i] *= w[i];                            // zero behind the row's end
                c += d[k][i] * hat[k][i]; m += d[k][i];
            }
        }
        G.two(c, m);
        c /= (float)A.width;
        m = A.pre == RK_NORM_LAYER ? m / (float)A.width : 0.f;
#pragma unroll
        for (int k = 0; k < NC; ++k)
#pragma unroll
            for (int i = 0; i < CH; ++i) d[k][i] = st.w * (d[k][i] - m - hat[k][i] * c);
    } else {
#pragma unroll
        for (int k = 0; k < NC; ++k)
#pragma unroll
            for (int i = 0; i < CH; ++i) d[k][i] = 0.f;
    }
    if (A.row_sums && P.tid == 0) A.row_sums[P.row] = make_float4(c, m, 0.f, 0.f);
    const uint64_t gate = A.gate_rows ? P.row / A.gate_rows : 0;
    const Row<R> rd(A.dxo, P.row, A.dxo_st, A.width), dx(A.xo, P.row, A.xo_st, A.width);
    const Row<T> ry(A.y, P.row, A.y_st, A.width), dy(A.u, P.row, A.u_st, A.width);
    c = 0.f; m = 0.f;
#pragma unroll
    for (int k = 0; k < NC; ++k) {
        float t[CH];
        if (A.dxo) {
            load_row<CUTS, R, CH>(rd, at[k], t);
#pragma unroll
            for (int i = 0; i < CH; ++i) d[k][i] += t[i];
        }
#pragma unroll
        for (int i = 0; i < CH; ++i) t[i] = A.scale * d[k][i];
        store_row<CUTS, R, CH>(dx, at[k], t);
        if (!A.y) continue;
        float w[CH], g[CH];
        load_param<CUTS, T, CH>(A, G_GATE, gate, A.gate_st, at[k], 1.f, g);
        load_param<CUTS, T, CH>(A, G_POST_W, 0, 0, at[k], 1.f, w);
        load_row<CUTS, T, CH>(ry, at[k], hat[k]);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            d[k][i] = i < at[k].valid ? d[k][i] * g[i] * w[i] : 0.f;
            hat[k][i] = (hat[k][i] - st.x) * st.y;
            c += d[k][i] * hat[k][i]; m += d[k][i];
        }
    }
    if (!A.y) return;
    if (A.post != RK_NORM_NONE) {
        G.two(c, m);
        c /= (float)A.width;
        m = A.post == RK_NORM_LAYER ? m / (float)A.width : 0.f;
    }
#pragma unroll
    for (int k = 0; k < NC; ++k) {
        if (A.post != RK_NORM_NONE)
#pragma unroll
            for (int i = 0; i < CH; ++i) d[k][i] = st.y * (d[k][i] - m - hat[k][i] * c);
        store_row<CUTS, T, CH>(dy, at[k], d[k]);
    }
}

// ---- gradients of the vectors: sums over rows
// The rows are cut into chunks, and no chunk holds parts of two gates' rows unless it holds all of each of them.
struct Chunks {
    uint64_t rows;              // of a chunk
    uint64_t per_gate;          // chunks of a gate's rows; 0: chunks hold whole gates, or the gate is one for all
    uint64_t n;
};
struct NormSums {
    NormArgs A;
    Chunks C;
    float *part[G_VECTORS];     // null: not wanted; [chunk][width], or, of the gates, where `gate_direct`, [gate][stride]
    uint64_t gate_out_st;
    bool gate_direct;
};
__device__ __forceinline__ void chunk_rows(const NormArgs &A, const Chunks &C, uint64_t c, uint64_t &r0, uint64_t &r1) {
    uint64_t end = A.n_rows;
    if (C.per_gate) {
        const uint64_t g = c / C.per_gate;
        r0 = g * A.gate_rows + (c - g * C.per_gate) * C.rows;
        const uint64_t last = (g + 1) * A.gate_rows;
        end = last < end ? last : end;
    } else {
        r0 = c * C.rows;
    }
    r1 = r0 + C.rows < end ? r0 + C.rows : end;
    if (r0 > r1) r0 = r1;
}

// A thread has CH columns of a chunk's rows; what it reads of a row's statistics is the same for all.
constexpr int SUM_THREADS = 256;
template <bool CUTS, typename T, typename R, int CH>
__global__ __launch_bounds__(SUM_THREADS) void k_norm_sums(NormSums S, uint32_t tiles) {
    const NormArgs &A = S.A;
    const uint64_t chunk = blockIdx.x / tiles;
    const Place at((blockIdx.x % tiles * SUM_THREADS + threadIdx.x) * CH, A.width, CH);
    if (at.valid <= 0) return;
    uint64_t r0, r1;
    chunk_rows(A, S.C, chunk, r0, r1);
    float acc[G_VECTORS][CH] = {};
    float w1[CH], b1[CH], w2[CH];
    load_param<CUTS, T, CH>(A, G_POST_W, 0, 0, at, 1.f, w1);
    load_param<CUTS, T, CH>(A, G_POST_B, 0, 0, at, 0.f, b1);
    load_param<CUTS, T, CH>(A, G_PRE_W, 0, 0, at, 1.f, w2);
    for (uint64_t r = r0; r < r1; ++r) {
        const float4 st = reinterpret_cast<const float4 *>(A.stats)[r];
        float d[CH] = {};
        if (A.dxo) load_row<CUTS, R, CH>(Row<R>(A.dxo, r, A.dxo_st, A.width), at, d);
        if (A.pre != RK_NORM_NONE) {
            const float4 off = A.row_sums[r];
            float hat[CH], e[CH];
            load_row<CUTS, R, CH>(Row<R>(A.x, r, A.x_st, A.width), at, hat);
            load_row<CUTS, T, CH>(Row<T>(A.du, r, A.du_st, A.width), at, e);
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                hat[i] = (hat[i] - st.z) * st.w;
                acc[G_PRE_W][i] += e[i] * hat[i];
                acc[G_PRE_B][i] += e[i];
                d[i] += st.w * (e[i] * w2[i] - off.y - hat[i] * off.x);
            }
        }
        if (!A.y) continue;
        float g[CH], y[CH];
        const uint64_t gate = A.gate_rows ? r / A.gate_rows : 0;
        load_param<CUTS, T, CH>(A, G_GATE, gate, A.gate_st, at, 1.f, g);
        load_row<CUTS, T, CH>(Row<T>(A.y, r, A.y_st, A.width), at, y);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            y[i] = (y[i] - st.x) * st.y;
            acc[G_GATE][i] += d[i] * (y[i] * w1[i] + b1[i]);
            d[i] *= g[i];
            acc[G_POST_W][i] += d[i] * y[i];
            acc[G_POST_B][i] += d[i];
        }
        if (S.gate_direct && (r + 1 == r1 || (r + 1) % A.gate_rows == 0)) {
            store_row<CUTS, float, CH>(Row<float>(S.part[G_GATE], gate, S.gate_out_st, A.width), at, acc[G_GATE]);
#pragma unroll
            for (int i = 0; i < CH; ++i) acc[G_GATE][i] = 0.f;
        }
    }
#pragma unroll
    for (int s = 0; s < G_VECTORS; ++s)
        if (S.part[s] && !(s == G_GATE && S.gate_direct)) store_row<CUTS, float, CH>(Row<float>(S.part[s], chunk, A.width, A.width), at, acc[s]);
}

// what a lane keeps in LDS of two weights and the gate, in 16 bytes: an odd number of them, so that the lanes' reads spread over the
// banks
constexpr uint32_t sums_lds_of(int ch, int nc) { return (uint32_t)(3 * nc * ch / 4) | 1u; }

// Rows back and the sums over them in one pass: a workgroup takes a chunk of rows and every lane keeps the sums of its columns in
// registers.  Rows that a wavefront holds are shared out to the workgroup's four, which add their sums up at the end, or (`alone`: with
// gates of rows) are a chunk to each of them.  The next row's x_out and du are on their way while this row's first norm is summed,
// its dx_out and y while the second is; LEAN has half of that under way, for rows that take all registers.  Weights and gate,
// which every row needs, lie in LDS: each lane reads only what it wrote itself.  Of the vectors behind the gate only sum D y^ and sum D are kept:
//     d post_weight = gate sum D y^,  d post_bias = gate sum D,  d gate = post_weight sum D y^ + post_bias sum D
// for rows of one gate.  A chunk with several gates' rows adds its first two up in its place in memory, gate by gate.
// Bound by HBM but for the first row's and the sums' latency: wide rows take all registers of a compute unit, one workgroup each.  8192 x 8576 bfloat16
// 169 us, 843 MB, 5.0 TB/s (a pass for the rows and one for the sums: 391 us with the join); 4096 x 5248 with a float32 stream 86 us, 387 MB, 4.5 TB/s.
template <bool CUTS, typename T, typename R, int CH, int NC, int MAXT, bool BIAS>
__global__ __launch_bounds__(MAXT) void k_norm_backward_sums(NormSums S, bool per_wave, bool alone) {
    constexpr bool LEAN = MAXT == 768 && (BIAS || CUTS || sizeof(R) == 4);
    // The pieces of a cut vector stay apart until they are wanted, where there are registers for it: 4096 x 5003 104 -> 69 us, 8192 x 777
    // with biases 43 -> 35; but 4096 x 7777 in 32 bits 194 -> 262, 8192 x 777 52 -> 61, 4096 x 9999 149 -> 185.
    // Elsewhere they are asked for where they are wanted: 4096 x 9999 with biases 254 -> 212 us, in 32 bits 358 -> 277.
    constexpr bool HOLD = CUTS && sizeof(T) == 2 && (MAXT <= 512 || (MAXT == 1024 && sizeof(R) == 2)), LATE = CUTS && !HOLD;
    extern __shared__ float4 param_lds[];
    __shared__ float lds[96];
    const NormArgs &A = S.A;
    RowGroup G;
    const RowOf P = row_of(0, S.C.n, per_wave, G, lds);            // (its "row" is the chunk of one that is alone)
    if (!P.there && alone) return;
    const bool shared = per_wave && !alone;
    const uint64_t chunk = shared ? blockIdx.x : P.row;
    uint64_t r0, r1;
    chunk_rows(A, S.C, chunk, r0, r1);
    const uint64_t stride = shared ? blockDim.x >> 6 : 1, begin = r0 + (shared ? G.wave : 0u);
    Place at[NC];
    places<CH, NC>(at, P.tid, P.threads, A.width);
    Held<HOLD, R, CH> rx[NC], rd[NC];
    Held<HOLD, T, CH> ru[NC], ry[NC];
    float4 st_next = make_float4(0.f, 1.f, 0.f, 1.f);
    auto fetch_first = [&](uint64_t r) {
        const bool there = r < r1;                              // (behind the chunk: a row of no elements)
        if (there) st_next = reinterpret_cast<const float4 *>(A.stats)[r];
        const Row<R> x(there ? A.x : nullptr, r, A.x_st, A.width);
        const Row<T> u(there ? A.du : nullptr, r, A.du_st, A.width);
#pragma unroll
        for (int k = 0; k < NC; ++k) {
            rx[k] = held<HOLD, R, CH, STREAM>(x, at[k]);
            ru[k] = held<HOLD, T, CH, STREAM>(u, at[k]);
        }
    };
    auto fetch_second = [&](uint64_t r) {
        const bool there = r < r1;
        const Row<R> dxo(there ? A.dxo : nullptr, r, A.dxo_st, A.width);
        const Row<T> y(there ? A.y : nullptr, r, A.y_st, A.width);
#pragma unroll
        for (int k = 0; k < NC; ++k) {
            rd[k] = held<HOLD, R, CH, STREAM>(dxo, at[k]);
            ry[k] = held<HOLD, T, CH, STREAM>(y, at[k]);
        }
    };
    fetch_first(begin);
    if (!LEAN) fetch_second(begin);
    constexpr int Q = CH / 4;
    float4 *const mine = param_lds + threadIdx.x * sums_lds_of(CH, NC);
    auto put = [&](int v, int k, const float (&x)[CH]) {
#pragma unroll
        for (int q = 0; q < Q; ++q) mine[(v * NC + k) * Q + q] = make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
    };
    auto get = [&](int v, int k, float (&x)[CH]) {
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const float4 f = mine[(v * NC + k) * Q + q];
            x[4 * q] = f.x; x[4 * q + 1] = f.y; x[4 * q + 2] = f.z; x[4 * q + 3] = f.w;
        }
    };
    enum { L_W1, L_W2, L_GATE };
    uint64_t gate = A.gate_rows ? begin / A.gate_rows : 0, gate_end = A.gate_rows ? (gate + 1) * A.gate_rows : ~0ull;
    // the vectors' parts, all under way before the first is waited for
    auto vectors = [&](auto p) {
        typedef decltype(p) V;
        Held<HOLD, V, CH> w[3][NC];
        auto hold_vector = [&](const Row<V> &of, const Place &p) {
            if constexpr (HOLD) return hold_row<V, CH>(of, p); else return Held<false, V, CH>{fetch_row<CUTS, V, CH>(of, p)};
        };
        const Row<V> w1(A.vec[G_POST_W], 0, 0, A.width), w2(A.vec[G_PRE_W], 0, 0, A.width), g(begin < r1 ? A.vec[G_GATE] : nullptr, gate, A.gate_st, A.width);
#pragma unroll
        for (int k = 0; k < NC; ++k) {
            w[L_W1][k] = hold_vector(w1, at[k]);
            w[L_W2][k] = hold_vector(w2, at[k]);
            w[L_GATE][k] = hold_vector(g, at[k]);
        }
        const bool have[3] = {A.vec[G_POST_W] != nullptr, A.vec[G_PRE_W] != nullptr, A.vec[G_GATE] != nullptr};
#pragma unroll
        for (int v = 0; v < 3; ++v)
#pragma unroll
            for (int k = 0; k < NC; ++k) {
                float x[CH];
                const Words<V, CH> own = whole_of<V, CH>(w[v][k], at[k]);
#pragma unroll
                for (int i = 0; i < CH; ++i) x[i] = have[v] ? element<V>(own, i) : 1.f;
                put(v, k, x);
            }
    };
    if (A.p32) vectors(float()); else vectors(T());
    float sum_dy[NC][CH] = {}, acc_w2[NC][CH] = {}, sum_d[BIAS ? NC : 1][CH] = {}, acc_b2[BIAS ? NC : 1][CH] = {};
    // what the sums since the last gate give
    auto of_gate = [&](int k, float (&w)[CH], float (&b)[CH], float (&g)[CH]) {
        float v[CH];
        get(L_GATE, k, v);
#pragma unroll
        for (int i = 0; i < CH; ++i) { w[i] = v[i] * sum_dy[k][i]; if constexpr (BIAS) b[i] = v[i] * sum_d[k][i]; }
        get(L_W1, k, v);
#pragma unroll
        for (int i = 0; i < CH; ++i) { g[i] = v[i] * sum_dy[k][i]; sum_dy[k][i] = 0.f; }
        if constexpr (BIAS) {
            load_param<CUTS, T, CH>(A, G_POST_B, 0, 0, at[k], 0.f, v);
#pragma unroll
            for (int i = 0; i < CH; ++i) { g[i] += v[i] * sum_d[k][i]; sum_d[k][i] = 0.f; }
        }
    };
    const float inv = 1.f / (float)A.width;
    for (uint64_t r = begin; r < r1; r += stride) {
        const float4 st = st_next;
        if (r >= gate_end) {
            gate = r / A.gate_rows;
            gate_end = (gate + 1) * A.gate_rows;
#pragma unroll
            for (int k = 0; k < NC; ++k) {
                float x[CH];
                load_param<CUTS, T, CH>(A, G_GATE, gate, A.gate_st, at[k], 1.f, x);
                put(L_GATE, k, x);
            }
        }
        float d[NC][CH], hat[NC][CH];
        float c = 0.f, m = 0.f;
#pragma unroll
        for (int k = 0; k < NC; ++k) {
            float w2[CH];
            get(L_W2, k, w2);
            Words<T, CH> wu;
            Words<R, CH> wx;
            if constexpr (LATE) {
                const Held<true, T, CH> hu = with_pieces<T, CH>(Row<T>(A.du, r, A.du_st, A.width), at[k], ru[k].w);
                const Held<true, R, CH> hx = with_pieces<R, CH>(Row<R>(A.x, r, A.x_st, A.width), at[k], rx[k].w);
                wu = whole_of<T, CH>(hu, at[k]); wx = whole_of<R, CH>(hx, at[k]);
            } else {
                wu = whole_of<T, CH>(ru[k], at[k]); wx = whole_of<R, CH>(rx[k], at[k]);
            }
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const float u = element<T>(wu, i);
                hat[k][i] = (element<R>(wx, i) - st.z) * st.w;
                acc_w2[k][i] += u * hat[k][i];
                if constexpr (BIAS) acc_b2[k][i] += u;
                d[k][i] = u * w2[i];
                c += d[k][i] * hat[k][i]; m += d[k][i];
            }
            __builtin_amdgcn_sched_barrier(0);                  // vector by vector: fewer registers at once
        }
        if (LEAN) fetch_second(r); else fetch_first(r + stride);
        G.two(c, m);
        c *= inv;
        m = A.pre == RK_NORM_LAYER ? m * inv : 0.f;
#pragma unroll
        for (int k = 0; k < NC; ++k) {
            Words<R, CH> wd;
            if constexpr (LATE) wd = whole_of<R, CH>(with_pieces<R, CH>(Row<R>(A.dxo, r, A.dxo_st, A.width), at[k], rd[k].w), at[k]);
            else wd = whole_of<R, CH>(rd[k], at[k]);
#pragma unroll
            for (int i = 0; i < CH; ++i) d[k][i] = st.w * (d[k][i] - m - hat[k][i] * c) + element<R>(wd, i);
        }
        c = 0.f; m = 0.f;
        const Row<R> dx(A.xo, r, A.xo_st, A.width);
#pragma unroll
        for (int k = 0; k < NC; ++k) {
            float t[CH], w1[CH], g[CH];
            get(L_W1, k, w1);
            get(L_GATE, k, g);
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                t[i] = A.scale * d[k][i];
            }
            store_row<CUTS, R, CH, STREAM>(dx, at[k], t);
            Words<T, CH> wy;
            if constexpr (LATE) wy = whole_of<T, CH>(with_pieces<T, CH>(Row<T>(A.y, r, A.y_st, A.width), at[k], ry[k].w), at[k]);
            else wy = whole_of<T, CH>(ry[k], at[k]);
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const float y = (element<T>(wy, i) - st.x) * st.y;
                sum_dy[k][i] += d[k][i] * y;
                if constexpr (BIAS) sum_d[k][i] += d[k][i];
                hat[k][i] = y;
                d[k][i] = i < at[k].valid ? d[k][i] * g[i] * w1[i] : 0.f;
                c += d[k][i] * y; m += d[k][i];
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (LEAN) fetch_first(r + stride); else fetch_second(r + stride);
        if (A.post != RK_NORM_NONE) {
            G.two(c, m);
            c *= inv;
            m = A.post == RK_NORM_LAYER ? m * inv : 0.f;
#pragma unroll
            for (int k = 0; k < NC; ++k)
#pragma unroll
                for (int i = 0; i < CH; ++i) d[k][i] = st.y * (d[k][i] - m - hat[k][i] * c);
        }
        const Row<T> dy(A.u, r, A.u_st, A.width);
#pragma unroll
        for (int k = 0; k < NC; ++k) store_row<CUTS, T, CH, STREAM>(dy, at[k], d[k]);
        if (A.gate_rows && (r + 1 == r1 || r + 1 == gate_end)) {
            const bool first = gate_end <= r0 + A.gate_rows;    // (of the chunk's gates)
            const Row<float> pw(S.part[G_POST_W], chunk, A.width, A.width), pb(S.part[G_POST_B], chunk, A.width, A.width);
            const Row<float> pg(S.part[G_GATE], S.gate_direct ? gate : chunk, S.gate_direct ? S.gate_out_st : A.width, A.width);
#pragma unroll
            for (int k = 0; k < NC; ++k) {
                float w[CH], b[CH], g[CH], old[CH];
                of_gate(k, w, b, g);
                store_row<CUTS, float, CH>(pg, at[k], g);
                if (!first) {
                    load_row<CUTS, float, CH>(pw, at[k], old);
#pragma unroll
                    for (int i = 0; i < CH; ++i) w[i] += old[i];
                }
                store_row<CUTS, float, CH>(pw, at[k], w);
                if constexpr (BIAS) {
                    if (!first) {
                        load_row<CUTS, float, CH>(pb, at[k], old);
#pragma unroll
                        for (int i = 0; i < CH; ++i) b[i] += old[i];
                    }
                    store_row<CUTS, float, CH>(pb, at[k], b);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    // the chunk's sums; a shared chunk's wavefronts add them up over LDS, in their order, a vector of each lane at a time
    auto keep = [&](int which, int k, float (&v)[CH]) {
        const Row<float> part(S.part[which], chunk, A.width, A.width);
        if (!shared) {
            store_row<CUTS, float, CH>(part, at[k], v);
            return;
        }
        if (!S.part[which]) return;
        __syncthreads();                                        // (weights and gate are not needed any more)
        if (G.wave) {
#pragma unroll
            for (int q = 0; q < Q; ++q) param_lds[((G.wave - 1) * Q + q) * 64 + G.lane] = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
        }
        __syncthreads();
        if (G.wave) return;
        for (uint32_t w = 0; w + 1 < stride; ++w)
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const float4 f = param_lds[(w * Q + q) * 64 + G.lane];
                v[4 * q] += f.x; v[4 * q + 1] += f.y; v[4 * q + 2] += f.z; v[4 * q + 3] += f.w;
            }
        store_row<CUTS, float, CH>(part, at[k], v);
    };
    float w[NC][CH], b[NC][CH], g[NC][CH];
    if (!A.gate_rows)
#pragma unroll
        for (int k = 0; k < NC; ++k) of_gate(k, w[k], b[k], g[k]);
#pragma unroll
    for (int k = 0; k < NC; ++k) {
        keep(G_PRE_W, k, acc_w2[k]);
        if constexpr (BIAS) keep(G_PRE_B, k, acc_b2[k]);
        if (!A.gate_rows) {
            keep(G_POST_W, k, w[k]);
            if constexpr (BIAS) keep(G_POST_B, k, b[k]);
            keep(G_GATE, k, g[k]);
        } else if (r0 == r1) {                                  // (a chunk behind the last row of the last gate)
            float zero[CH] = {};
            keep(G_POST_W, k, zero);
            keep(G_POST_B, k, zero);
            if (!S.gate_direct) keep(G_GATE, k, zero);
        }
    }
}

// The chunks' sums added up, always in the same order: LANES lanes next to each other have four columns each of a chunk, the
// workgroup's 1,024 / LANES such rows share the chunks; a wavefront's rows are joined by swaps and rotations, the wavefronts over LDS.
// Bound by its launch and one trip to memory: 3 x 256 chunks of 5248 columns (16 MB) 4.6 us, a column a lane took 7.6.
struct Joined { const float *from[G_VECTORS]; float *to[G_VECTORS]; uint64_t count[G_VECTORS]; uint32_t n; uint64_t gate_chunks, gate_out_st; };
template <int LANES> __global__ __launch_bounds__(1024) void k_norm_join(Joined J, uint32_t width, uint32_t tiles) {
    static_assert(LANES == 16 || LANES == 4, "");
    constexpr uint32_t SHARE = 1024 / LANES, COLS = 4 * LANES;
    typedef Vec<float, 4> Any __attribute__((aligned(4)));
    __shared__ float4 lds[16][LANES];
    const uint32_t part = threadIdx.x / LANES;
    const uint64_t job = blockIdx.x / tiles;
    const uint32_t col0 = blockIdx.x % tiles * COLS, col = col0 + threadIdx.x % LANES * 4;
    // the vectors first, then the gates one by one (J.gate_chunks each)
    const uint32_t v = job < J.n ? (uint32_t)job : J.n;
    const float *from = J.from[v];
    float *to = J.to[v];
    uint64_t count = J.count[v];
    if (job >= J.n) { from += (job - J.n) * J.gate_chunks * width; to += (job - J.n) * J.gate_out_st; count = J.gate_chunks; }
    Vec<float, 4> s = {0.f, 0.f, 0.f, 0.f};
    if (col + 4 <= width) {
        uint64_t c = part;
        for (; c + 3 * SHARE < count; c += 4 * SHARE) {         // four under way at once
            Vec<float, 4> x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const Any *>(from + (c + SHARE * i) * width + col);
#pragma unroll
            for (int i = 0; i < 4; ++i) s += x[i];
        }
        for (; c < count; c += SHARE) s += *reinterpret_cast<const Any *>(from + c * width + col);
    } else if (col < width) {                                   // the vector that the width cuts
        for (uint64_t c = part; c < count; c += SHARE)
#pragma unroll
            for (int i = 0; i < 3; ++i) if (col + i < width) s[i] += from[c * width + col + i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float o;
        s[i] = swap32(s[i], o) + o;
        s[i] = swap16(s[i], o) + o;
        if constexpr (LANES == 4) { s[i] += dpp_of<0x128>(s[i]); s[i] += dpp_of<0x124>(s[i]); }      // row_ror:8, 4
    }
    if ((threadIdx.x & 63u) < (uint32_t)LANES) lds[threadIdx.x >> 6][threadIdx.x % LANES] = make_float4(s[0], s[1], s[2], s[3]);
    __syncthreads();
    if (threadIdx.x >= COLS || col0 + threadIdx.x >= width) return;
    float sum = 0.f;
#pragma unroll
    for (uint32_t w = 0; w < 16; ++w) sum += reinterpret_cast<const float *>(lds[w])[threadIdx.x];
    to[col0 + threadIdx.x] = sum;
}

// gates that no row has: their gradients are sums over nothing
__global__ __launch_bounds__(256) void k_norm_no_rows(float *to, uint64_t stride, uint64_t gates, uint32_t width) {
    for (uint64_t i = blockIdx.x * 256ull + threadIdx.x; i < gates * width; i += gridDim.x * 256ull) to[i / width * stride + i % width] = 0.f;
}

// ---- host
struct Shape { int nc; uint32_t threads, rows_per_wg; bool per_wave; };

template <typename T, typename R> constexpr int chunk_of() { return sizeof(T) == 2 ? 8 : 4; }

// A lane holds nc vectors of a row, a row as few wavefronts as that allows; rows that one wavefront holds go four to a workgroup.
Shape shape_of(uint32_t width, int ch) {
    for (int nc = 1; nc <= 2; ++nc)
        if (width <= 64u * ch * nc) return Shape{nc, 256, 4, true};
    int nc = 2;
    while (nc < 8 && width > 1024u * ch * nc) nc *= 2;
    const uint32_t threads = (width + ch * nc * 64 - 1) / (ch * nc * 64) * 64;
    return Shape{nc, threads, 1, false};
}

template <typename T, typename R, int NC, int MAXT>
void launch_nc(hipStream_t st, NormArgs A, const Shape &S, bool back) {
    constexpr int CH = chunk_of<T, R>();
    const uint64_t all = (A.n_rows + S.rows_per_wg - 1) / S.rows_per_wg, most = RK_LAUNCH_THREADS / S.threads;
    auto go = [&](auto cuts) {
        constexpr bool CUTS = decltype(cuts)::value;
        for (uint64_t at = 0; at < all; at += most) {
            const uint32_t blocks = (uint32_t)(all - at < most ? all - at : most);
            A.first = at * S.rows_per_wg;
            if (back) k_norm_backward<CUTS, T, R, CH, NC, MAXT><<<blocks, S.threads, 0, st>>>(A, S.per_wave);
            else k_norm_forward<CUTS, T, R, CH, NC, MAXT><<<blocks, S.threads, 0, st>>>(A, S.per_wave);
        }
    };
    if (A.width % CH) go(std::true_type()); else go(std::false_type());
}
template <typename T, typename R> void launch_rows(hipStream_t st, const NormArgs &A, bool back) {
    const Shape S = shape_of(A.width, chunk_of<T, R>());
    if (S.nc == 1) launch_nc<T, R, 1, 256>(st, A, S, back);
    else if (S.nc == 2 && S.threads <= 512) launch_nc<T, R, 2, 512>(st, A, S, back);
    else if (S.nc == 2) launch_nc<T, R, 2, 1024>(st, A, S, back);
    else if (S.nc == 4) launch_nc<T, R, 4, 1024>(st, A, S, back);
    else if constexpr (chunk_of<T, R>() == 4) launch_nc<T, R, 8, 1024>(st, A, S, back);
}
// How the rows are held where their sums are taken along; nc 0: too wide for a lane's registers or a compute unit's LDS, rows and sums
// are two passes.
Shape sums_shape_of(uint32_t width, int ch) {
    const int per = 8 / ch;                                     // vectors of eight elements
    for (int n8 = 1; n8 <= 2; ++n8)
        if (width <= 512u * n8) return Shape{n8 * per, 256, 4, true};
    const int n8 = width <= 8192u ? 1 : 2;
    const uint32_t threads = (width + 8 * n8 * 64 - 1) / (8 * n8 * 64) * 64;
    if (threads > (n8 == 1 ? 1024u : 768u) || threads * sums_lds_of(8, n8) * 16 > 163840u - 1024u) return Shape{0, 0, 0, false};
    return Shape{n8 * per, threads, 1, false};
}
template <typename T, typename R, int NC, int MAXT> int32_t launch_fused_nc(rk_ctx *ctx, const NormSums &S, const Shape &H, bool bias) {
    constexpr int CH = chunk_of<T, R>();
    const bool alone = !H.per_wave || S.A.gate_rows;
    const uint32_t blocks = (uint32_t)(alone ? (S.C.n + H.rows_per_wg - 1) / H.rows_per_wg : S.C.n);
    const uint32_t lds = H.threads * sums_lds_of(CH, NC) * 16;
    auto go = [&](auto cuts, auto with_bias) -> int32_t {
        const auto kernel = k_norm_backward_sums<decltype(cuts)::value, T, R, CH, NC, MAXT, decltype(with_bias)::value>;
        if (lds > 65536u - 1024u) RK_HIP(ctx, hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
        kernel<<<blocks, H.threads, lds, ctx->stream>>>(S, H.per_wave, alone);
        return RK_OK;
    };
    const bool cuts = S.A.width % CH != 0;
    if (bias) return cuts ? go(std::true_type(), std::true_type()) : go(std::false_type(), std::true_type());
    return cuts ? go(std::true_type(), std::false_type()) : go(std::false_type(), std::false_type());
}
template <typename T, typename R> int32_t launch_fused(rk_ctx *ctx, const NormSums &S, const Shape &H, bool bias) {
    constexpr int PER = 8 / chunk_of<T, R>();
    if (H.nc == PER && H.threads <= 512) return launch_fused_nc<T, R, PER, 512>(ctx, S, H, bias);
    if (H.nc == PER) return launch_fused_nc<T, R, PER, 1024>(ctx, S, H, bias);
    if (H.threads <= 512) return launch_fused_nc<T, R, 2 * PER, 512>(ctx, S, H, bias);
    return launch_fused_nc<T, R, 2 * PER, 768>(ctx, S, H, bias);
}
template <typename T, typename R> void launch_sums(hipStream_t st, const NormSums &S) {
    constexpr int CH = chunk_of<T, R>();
    const uint32_t tiles = (S.A.width + SUM_THREADS * CH - 1) / (SUM_THREADS * CH);
    if (S.A.width % CH) k_norm_sums<true, T, R, CH><<<(uint32_t)(S.C.n * tiles), SUM_THREADS, 0, st>>>(S, tiles);
    else k_norm_sums<false, T, R, CH><<<(uint32_t)(S.C.n * tiles), SUM_THREADS, 0, st>>>(S, tiles);
}
// f(T(), R()) for the types of y and of the stream
template <typename F> void with_types(uint32_t type, uint32_t res, F f) {
    if (type == RK_F32) f(float(), float());
    else if (type == RK_BF16 && res == RK_F32) f(__bf16(), float());
    else if (type == RK_BF16) f(__bf16(), __bf16());
    else if (res == RK_F32) f(_Float16(), float());
    else f(_Float16(), _Float16());
}

bool aligned(const void *p, uint32_t type) { return ((uintptr_t)p & (type == RK_F32 ? 3u : 1u)) == 0; }

// what both directions ask of a block; mats: the matrices that have to be there
int32_t check_block(rk_ctx *ctx, const rk_norm_block *b, uint64_t n_rows, uint32_t width, const rk_matrix *x, const rk_matrix *y, const float *stats) {
    if (!b) return rk_fail(ctx, RK_ERR_INVALID_ARG, "block is null");
    if (b->post_kind > RK_NORM_LAYER || b->pre_kind > RK_NORM_LAYER) return rk_fail(ctx, RK_ERR_INVALID_ARG, "unknown kind of norm");
    if (b->param_type > RK_F16) return rk_fail(ctx, RK_ERR_INVALID_ARG, "unknown param_type");
    if (!(b->post_eps >= 0.f) || !(b->pre_eps >= 0.f) || !std::isfinite(b->post_eps) || !std::isfinite(b->pre_eps) || !std::isfinite(b->res_scale))
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "eps negative, or eps or res_scale not finite");
    if ((b->post_kind == RK_NORM_NONE && (b->post_weight || b->post_bias)) || (b->pre_kind == RK_NORM_NONE && (b->pre_weight || b->pre_bias)))
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "weight or bias of a norm that is not there");
    if (!y && (b->post_kind != RK_NORM_NONE || b->gate)) return rk_fail(ctx, RK_ERR_INVALID_ARG, "norm or gate of a block's output that is not there");
    if (!b->gate && b->gate_rows) return rk_fail(ctx, RK_ERR_INVALID_ARG, "gate_rows without a gate");
    if (b->gate_rows && n_rows > b->gate_rows && b->gate_stride < width) return rk_fail(ctx, RK_ERR_INVALID_ARG, "gate_stride below the width");
    for (const void *p : {b->post_weight, b->post_bias, b->pre_weight, b->pre_bias, b->gate})
        if (!aligned(p, b->param_type)) return rk_fail(ctx, RK_ERR_INVALID_ARG, "misaligned weight, bias or gate");
    if (width < 1) return rk_fail(ctx, RK_ERR_INVALID_ARG, "width below 1");
    if (width > RK_NORM_MAX_WIDTH) return rk_fail(ctx, RK_ERR_UNSUPPORTED, "rows of %u elements, %u at most", width, RK_NORM_MAX_WIDTH);
    if (n_rows > 0x7FFFFFFFull) return rk_fail(ctx, RK_ERR_UNSUPPORTED, "more than 2^31 - 1 rows");
    if (!rk_matrix_ok(x, n_rows, width) || (y && !rk_matrix_ok(y, n_rows, width)) || (n_rows && (!stats || ((uintptr_t)stats & 15u))))
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "x, y or stats null, misaligned or of a stride below the width");
    return RK_OK;
}
// the types go together: the stream's is y's and u's, or float32; the vectors' is y's and u's, or float32
int32_t check_types(rk_ctx *ctx, const rk_norm_block *b, uint32_t type, uint32_t res) {
    if (res != type && res != RK_F32) return rk_fail(ctx, RK_ERR_INVALID_ARG, "the stream's type is neither the block's nor RK_F32");
    const bool any = b->post_weight || b->post_bias || b->pre_weight || b->pre_bias || b->gate;
    if (any && b->param_type != type && b->param_type != RK_F32) return rk_fail(ctx, RK_ERR_INVALID_ARG, "param_type is neither the block's nor RK_F32");
    return RK_OK;
}
void fill_block(NormArgs &A, const rk_norm_block *b, uint64_t n_rows, uint32_t width) {
    A.vec[G_POST_W] = b->post_weight; A.vec[G_POST_B] = b->post_bias;
    A.vec[G_PRE_W] = b->pre_weight; A.vec[G_PRE_B] = b->pre_bias; A.vec[G_GATE] = b->gate;
    A.gate_rows = b->gate_rows < n_rows ? b->gate_rows : 0; A.gate_st = b->gate_stride;     // (a gate for all rows is one for all)
    A.n_rows = n_rows; A.width = width;
    A.post = b->post_kind; A.pre = b->pre_kind; A.p32 = b->param_type == RK_F32;
    A.post_eps = b->post_eps; A.pre_eps = b->pre_eps; A.scale = b->res_scale;
}

}  // namespace

extern "C" int32_t rk_norm_forward(rk_ctx *ctx, const rk_norm_block *block, uint64_t n_rows, uint32_t width, const rk_matrix *x,
                                   const rk_matrix *y, const rk_matrix *x_out, const rk_matrix *u, float *stats) {
    if (!ctx) return RK_ERR_INVALID_ARG;
    int32_t rc = check_block(ctx, block, n_rows, width, x, y, stats);
    if (rc != RK_OK) return rc;
    if ((u == nullptr) != (block->pre_kind == RK_NORM_NONE)) return rk_fail(ctx, RK_ERR_INVALID_ARG, "u goes with the norm before the next block");
    if (!u && !x_out) return rk_fail(ctx, RK_ERR_INVALID_ARG, "neither x_out nor u");
    if ((x_out && !rk_matrix_ok(x_out, n_rows, width)) || (u && !rk_matrix_ok(u, n_rows, width)))
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "x_out or u null, misaligned or of a stride below the width");
    const uint32_t type = u ? u->type : y ? y->type : x->type;
    if ((y && y->type != type) || (x_out && x_out->type != x->type)) return rk_fail(ctx, RK_ERR_INVALID_ARG, "y and u, or x and x_out, are of different types");
    if ((rc = check_types(ctx, block, type, x->type)) != RK_OK) return rc;
    if (n_rows == 0) return RK_OK;
    RK_HIP(ctx, hipSetDevice(ctx->device));
    NormArgs A{};
    fill_block(A, block, n_rows, width);
    A.x = x->data; A.x_st = x->stride;
    if (y) { A.y = y->data; A.y_st = y->stride; }
    if (x_out) { A.xo = x_out->data; A.xo_st = x_out->stride; }
    if (u) { A.u = u->data; A.u_st = u->stride; }
    A.stats = stats;
    with_types(type, x->type, [&](auto t, auto r) { launch_rows<decltype(t), decltype(r)>(ctx->stream, A, false); });
    RK_CHECK_LAUNCH(ctx, "k_norm_forward");
    return RK_OK;
}

extern "C" int32_t rk_norm_backward(rk_ctx *ctx, const rk_norm_block *block, uint64_t n_rows, uint32_t width, const rk_matrix *x_out,
                                    const rk_matrix *y, const float *stats, const rk_matrix *dx_out, const rk_matrix *du,
                                    const rk_matrix *dx, const rk_matrix *dy, const rk_norm_grads *grads) {
    if (!ctx) return RK_ERR_INVALID_ARG;
    int32_t rc = check_block(ctx, block, n_rows, width, x_out, y, stats);
    if (rc != RK_OK) return rc;
    if ((du == nullptr) != (block->pre_kind == RK_NORM_NONE)) return rk_fail(ctx, RK_ERR_INVALID_ARG, "du goes with the norm before the next block");
    if ((dy == nullptr) != (y == nullptr)) return rk_fail(ctx, RK_ERR_INVALID_ARG, "dy goes with y");
    if (!du && !dx_out) return rk_fail(ctx, RK_ERR_INVALID_ARG, "neither dx_out nor du");
    if (!rk_matrix_ok(dx, n_rows, width) || (dy && !rk_matrix_ok(dy, n_rows, width)) || (dx_out && !rk_matrix_ok(dx_out, n_rows, width)) ||
        (du && !rk_matrix_ok(du, n_rows, width)))
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "a gradient null, misaligned or of a stride below the width");
    const uint32_t type = du ? du->type : y ? y->type : x_out->type;
    if ((y && (y->type != type || dy->type != type)) || dx->type != x_out->type || (dx_out && dx_out->type != x_out->type))
        return rk_fail(ctx, RK_ERR_INVALID_ARG, "a gradient's type differs from its tensor's");
    if ((rc = check_types(ctx, block, type, x_out->type)) != RK_OK) return rc;
    float *out[G_VECTORS] = {};
    if (grads) {
        out[G_POST_W] = grads->post_weight; out[G_POST_B] = grads->post_bias;
        out[G_PRE_W] = grads->pre_weight; out[G_PRE_B] = grads->pre_bias; out[G_GATE] = grads->gate;
    }
    const void *const have[G_VECTORS] = {block->post_weight, block->post_bias, block->pre_weight, block->pre_bias, block->gate};
    bool any = false;
    for (int s = 0; s < G_VECTORS; ++s) {
        if (out[s] && (!have[s] || ((uintptr_t)out[s] & 3u))) return rk_fail(ctx, RK_ERR_INVALID_ARG, "gradient of a vector that is not there, or misaligned");
    }
    // the gates that rows use, and those behind them whose gradients are asked for
    const uint64_t needed = !out[G_GATE] || !block->gate_rows ? 0 : n_rows / block->gate_rows + (n_rows % block->gate_rows != 0);
    const uint64_t all_gates = out[G_GATE] && block->gate_rows && grads->gates ? grads->gates : needed;
    if (all_gates < needed || all_gates > 0x7FFFFFFFull) return rk_fail(ctx, RK_ERR_INVALID_ARG, "fewer gates than the rows need, or more than 2^31 - 1");
    if (all_gates > 1 && grads->gate_stride < width) return rk_fail(ctx, RK_ERR_INVALID_ARG, "gate_stride of the gradients below the width");
    if (block->gate_rows && !all_gates) out[G_GATE] = nullptr;              // no row, no gate
    for (float *o : out) any = any || o;
    if (n_rows == 0 && !any) return RK_OK;
    RK_HIP(ctx, hipSetDevice(ctx->device));
    NormArgs A{};
    fill_block(A, block, n_rows, width);
    if (du) { A.x = x_out->data; A.x_st = x_out->stride; }
    if (y) { A.y = y->data; A.y_st = y->stride; A.u = dy->data; A.u_st = dy->stride; }
    if (dx_out) { A.dxo = dx_out->data; A.dxo_st = dx_out->stride; }
    if (du) { A.du = du->data; A.du_st = du->stride; }
    A.xo = dx->data; A.xo_st = dx->stride;
    A.stats = const_cast<float *>(stats);
    NormSums S{};
    Joined J{};
    uint64_t join_jobs = 0;
    const bool bias = block->post_bias || out[G_PRE_B];
    const Shape H = sums_shape_of(width, type == RK_F32 ? 4 : 8);
    if (any) {
        // a chunk for every workgroup (of rows with gates that a wavefront holds: every wavefront) that fits the chip at once, but of
        // several rows, where there are enough: chunks cost a start and sums that have to be joined.  Half as many chunks: 8192 x 8576 178 -> 206 us, 4096 x
        // 5248 in 32 bits 94 -> 121, but 1000 x 2048 22.8 -> 17.9; twice as many: 184, 97 and 22.8, 1024 x 8576 39 -> 48.  Half the least rows: 2048 x 896
        // 14.3 -> 17.2 us, 300 x 2048 12.3 -> 16.1; twice: 15.4 and 12.9, 1000 x 2048 17.8.  (In graphs of 4 to 16 calls.)
        const uint64_t at_once = H.per_wave && A.gate_rows ? 2048 : H.nc && H.threads <= 512 ? 512 : 256;
        const uint64_t least = n_rows <= 256 ? (H.per_wave && !A.gate_rows ? 4 : 1) : H.per_wave && !A.gate_rows ? 8 : 2;
        uint64_t rows = (n_rows + at_once - 1) / at_once;
        if (rows < least) rows = least;
        const bool gates = A.gate_rows != 0;
        if (!gates) {
            S.C = Chunks{rows, 0, (n_rows + rows - 1) / rows};
        } else if (A.gate_rows <= rows) {
            rows = rows / A.gate_rows * A.gate_rows;
            S.C = Chunks{rows, 0, (n_rows + rows - 1) / rows};
        } else {
            const uint64_t per = (A.gate_rows + rows - 1) / rows, n_gates = (n_rows + A.gate_rows - 1) / A.gate_rows;
            S.C = Chunks{(A.gate_rows + per - 1) / per, per, per * n_gates};
        }
        S.gate_direct = gates && S.C.per_gate == 0 && out[G_GATE];
        S.gate_out_st = gates ? grads->gate_stride : 0;
        int n_part = 0;
        for (int s = 0; s < G_VECTORS; ++s) n_part += out[s] && !(s == G_GATE && S.gate_direct);
        float *part = nullptr;
        rc = rk_scratch(ctx, SL_NORM_PARTS, (size_t)(n_part * S.C.n * width) * 4, (void **)&part);
        if (rc != RK_OK) return rc;
        if (!H.nc && (rc = rk_scratch(ctx, SL_NORM_ROWS, (size_t)n_rows * 16, (void **)&A.row_sums)) != RK_OK) return rc;
        for (int s = 0; s < G_VECTORS; ++s) {
            if (!out[s]) continue;
            if (s == G_GATE && S.gate_direct) { S.part[s] = out[s]; continue; }
            S.part[s] = part; part += S.C.n * width;
            if (s == G_GATE && S.C.per_gate) {
                J.from[J.n] = S.part[s]; J.to[J.n] = out[s]; J.gate_chunks = S.C.per_gate; J.gate_out_st = S.gate_out_st;
                join_jobs = S.C.n / S.C.per_gate;
            } else {
                J.from[J.n] = S.part[s]; J.to[J.n] = out[s]; J.count[J.n] = S.C.n;
                ++J.n;
            }
        }
        join_jobs += J.n;
        if (S.C.n * ((width + 1023) / 1024) > 0x7FFFFFFFull) return rk_fail(ctx, RK_ERR_UNSUPPORTED, "too many rows");
    }
    S.A = A;
    if (n_rows && any && H.nc) {
        with_types(type, x_out->type, [&](auto t, auto r) { rc = launch_fused<decltype(t), decltype(r)>(ctx, S, H, bias); });
        if (rc != RK_OK) return rc;
        RK_CHECK_LAUNCH(ctx, "k_norm_backward_sums");
    } else if (n_rows) {
        with_types(type, x_out->type, [&](auto t, auto r) { launch_rows<decltype(t), decltype(r)>(ctx->stream, A, true); });
        RK_CHECK_LAUNCH(ctx, "k_norm_backward");
        if (any) {
            with_types(type, x_out->type, [&](auto t, auto r) { launch_sums<decltype(t), decltype(r)>(ctx->stream, S); });
            RK_CHECK_LAUNCH(ctx, "k_norm_sums");
        }
    }
    if (join_jobs) {
        // 64 columns a workgroup, or 16 where that would leave half of the compute units without one
        const bool narrow = join_jobs * ((width + 63) / 64) < 128;
        const uint32_t tiles = narrow ? (width + 15) / 16 : (width + 63) / 64;
        if (narrow) k_norm_join<4><<<(uint32_t)(join_jobs * tiles), 1024, 0, ctx->stream>>>(J, width, tiles);
        else k_norm_join<16><<<(uint32_t)(join_jobs * tiles), 1024, 0, ctx->stream>>>(J, width, tiles);
        RK_CHECK_LAUNCH(ctx, "k_norm_join");
    }
    const uint64_t written = needed ? needed : 1;               // (without a row the join has the first)
    if (all_gates > written) {
        const uint64_t blocks = ((all_gates - written) * width + 255) / 256;
        k_norm_no_rows<<<(uint32_t)(blocks < 2048 ? blocks : 2048), 256, 0, ctx->stream>>>(out[G_GATE] + written * grads->gate_stride, grads->gate_stride, all_gates - written, width);
        RK_CHECK_LAUNCH(ctx, "k_norm_no_rows");
    }
    return RK_OK;
}
