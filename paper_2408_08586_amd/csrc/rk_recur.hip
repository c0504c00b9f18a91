// Gated linear recurrence over packed sequences, and its gradient (rk_recur in rubick.h).
//
// Both directions are chains v <- p v + q, forward over h, backward over what a row hands to the one before it.  The rows are cut into tiles of
// RC_WAVES x L rows and 128 columns, a workgroup each: a wavefront has L rows, a lane two columns, and reads them once.  It takes
// its rows as one step (the product of their p, and q from nothing), the workgroup joins its wavefronts' steps, tells the tiles behind
// it what it makes of a value that comes in, finds the value that comes in to itself from the tiles before it, and goes through its rows again,
// in registers, for the results.
//
// What a tile says is one 64-bit word a column (p and q), readable as soon as it is no longer all ones, so that words need no flags or fences beside them.
// A tile joins the words of at most RC_BLOCK - 1 tiles before it, in order, with the value behind the last block of RC_BLOCK tiles, which that block's
// last tile writes: always the same sums in the same order.  The tiles of a column are handed out by a counter of its own, earlier ones first: who
// waits, waits for workgroups that run already.  A tile whose first row begins a sequence waits for nobody, and nobody
// looks behind the beginning of a sequence, so that nothing of one sequence comes near another.
//
// The gates' exponentials and divisions, the chain and the two ways through the rows are about 20 vector instructions an element forward and 44 backward, two fifths of the
// kernels' cycles; the rest is the rows' trip from memory and then the wait for the tiles before, under which two workgroups a compute unit have too little else to do
// (forward's gates and inflows take 64 of a lane's 128 registers through the wait; backward spills up to 204 bytes a lane).  Finding rows' sequences by their offsets is
// log2 of their number loads, each behind the one before: 64 x 5,248 of one row each 7.8 us, by seq_rows 7.1; 20,000 x 1,000 of 2 or of 1,000 sequences 48.
// Measured in bfloat16, coupled, kernels alone: forward 8,192 x 8,576 of equal sequences 92 to 95 us (421 MB, 4.5 TB/s); backward 8,192 x 5,248 118 to 122 us
// (516 MB, 4.3 TB/s), k_recur_bias 4 to 5, k_recur_clear 3 to 6.  One sequence of 65,536 x 1,024, not coupled: 102 to 106 us (403 MB, 3.9 TB/s): its 32 blocks
// of tiles wait for each other, about 1 us a block beyond what memory takes.  Blocks of 8 tiles or of 32, wavefronts of 8 rows or four to a workgroup were slower in most
// (timed with sequences of 2,048 rows, which a block holds whole, ragged ones and one of all rows; as it is, 8,192 x 8,576 takes 90 to 94 us for sequences of 1,000 to 8,192 rows).
#include <type_traits>

#include "rk_vec.h"

namespace {

constexpr uint32_t RC_WAVES = 8, RC_THREADS = 64 * RC_WAVES, RC_COLS = 128, RC_BLOCK = 16, RC_TICKET = 16;
// How long who waits sleeps before it looks again, in 64 clocks: looking takes the memory's time from those that are waited for (one sequence of 65536 x 1024 forward, of 1,
// 4, 8, 16 and 30: 136, 114, 111, 110 and 107 us; ragged 9001 x 1111 backward 73, 70, 70, 70 and 71; 8192 x 8576 the same)
constexpr int RC_NAP = 16;
constexpr uint32_t RC_ROWS = 16;                               // of a wavefront, the most

struct RecurArgs {
    const void *x, *z, *h, *dh, *bias;
    void *out, *dx, *dz;
    uint64_t x_st, z_st, h_st, dh_st, o_st, dx_st, dz_st;
    const float *state_in, *d_state_out;
    float *state_out, *d_state_in, *d_bias;
    uint64_t si_st, so_st, dso_st, dsi_st;
    const int32_t *offsets;
    uint32_t seq_rows, n_rows;
    uint32_t n_seqs, width, coupled, bias_type;
    uint32_t n_tiles, n_cols;       // tiles of rows; of columns
    uint32_t *ticket;               // [n_cols] counters, RC_TICKET words apart; null: no tile goes on with another's sequence
    uint64_t *steps;                // [n_tiles][width]: p and q
    uint32_t *behind;               // [n_tiles / RC_BLOCK][width]: the value behind a block of tiles
    float *bias_parts;              // [n_tiles][width]
    uint32_t idle;                  // workgroups that look for sequences without rows
};

// ---- a lane's two columns
template <typename T> using Two = Words<T, 2>;
template <typename T> using LooseTwo = Loose<Two<T>, T>;
struct Columns {
    uint32_t at;                    // where it reads: both elements are inside the row
    bool two, one;                  // writes both; the first alone, which it has read as the second
    __device__ __forceinline__ Columns(uint32_t c, uint32_t width) {
        two = c + 1 < width; one = c + 1 == width;
        at = two ? c : one && width > 1 ? width - 2 : 0;
    }
};
// CUT: rows have an odd number of elements
template <bool CUT, typename T> __device__ __forceinline__ Two<T> read_two(const T *row, const Columns &c, uint32_t width) {
    if (CUT && width == 1) {
        Vec<T, 2> v = (T)0.f;
        v[1] = row[0];
        return __builtin_bit_cast(Two<T>, v);
    }
    return *(const LooseTwo<T> *)((const char *)row + c.at * (uint32_t)sizeof(T));     // (a place of 32 bits beside a row that all lanes share)
}
template <bool CUT, typename T> __device__ __forceinline__ Vec<float, 2> floats(Two<T> w, const Columns &c) {
    Vec<float, 2> v;
    v[0] = element<T>(w, 0); v[1] = element<T>(w, 1);
    if (CUT) v[0] = c.one ? v[1] : v[0];
    return v;
}
// ONE: of a lane that has one column
template <bool ONE, typename T> __device__ __forceinline__ void write_two(T *row, uint32_t column, Vec<float, 2> f) {
    T *const at = (T *)((char *)row + column * (uint32_t)sizeof(T));
    Vec<T, 2> v;
    v[0] = (T)f[0]; v[1] = (T)f[1];
    if (ONE) *at = v[0];
    else __builtin_nontemporal_store(__builtin_bit_cast(Two<T>, v), (LooseTwo<T> *)at);
}
// f(false) for lanes of two columns, f(true) for one of a single column: what they do is done under one mask
template <bool CUT, typename F> __device__ __forceinline__ void where_columns(const Columns &c, F f) {
    if (c.two) f(std::false_type());
    if constexpr (CUT) { if (c.one) f(std::true_type()); }
}
template <bool CUT> __device__ __forceinline__ Vec<float, 2> read_state(const float *states, uint64_t stride, uint32_t seq, const Columns &c, uint32_t width) {
    return floats<CUT, float>(read_two<CUT, float>(states + seq * stride, c, width), c);
}
// L rows as they lie, from row0 on; behind the last of n_rows that one again
template <bool CUT, int L, typename T> __device__ __forceinline__ void read_rows(Two<T> (&w)[L], const void *data, uint64_t stride, uint32_t row0, uint32_t n_rows, const Columns &c, uint32_t width) {
    const T *p = (const T *)data + (uint64_t)(row0 < n_rows ? row0 : n_rows - 1) * stride;
#pragma unroll
    for (int i = 0; i < L; ++i) {
        w[i] = read_two<CUT, T>(p, c, width);
        p += row0 + i + 1 < n_rows ? stride : 0;
    }
}
__device__ __forceinline__ float bias_at(const RecurArgs &A, uint32_t c) {
    if (!A.bias || c >= A.width) return 0.f;
    if (A.bias_type == RK_F32) return ((const float *)A.bias)[c];
    return A.bias_type == RK_BF16 ? (float)((const __bf16 *)A.bias)[c] : (float)((const _Float16 *)A.bias)[c];
}

// f = sigmoid(z + bias) and 1 - f, which is a difference from one only where f is below a half.  Of 16 bits, the bias comes as bias_of gives it: in
// the unit of the exponent to base 2.
struct Gate { float f, not_f; };
template <typename T> __device__ __forceinline__ float bias_of(float bias) { return sizeof(T) == 4 ? bias : bias * -1.4426950408889634f; }
template <typename T> __device__ __forceinline__ Gate gate_of(float z, float bias) {
    if constexpr (sizeof(T) == 4) {
        const float v = z + bias;
        const float e = exp_f32(-fabsf(v)), near = __builtin_amdgcn_rcpf(1.f + e), far = e * near;
        return v >= 0.f ? Gate{near, far} : Gate{far, near};
    } else {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(z, -1.4426950408889634f, bias)), f = __builtin_amdgcn_rcpf(1.f + e);
        return Gate{f, e > 1.f ? 1.f - f : e * f};
    }
}

// ---- which rows of a wavefront begin and end sequences
struct Marks {
    uint32_t live, first, last;     // a bit a row
    int32_t seq, begin, end;        // of lane i: of row i; of lane L: of the tile's first row
    bool plain;                     // no sequence begins or ends in the tile, and all its rows are one's
};
// L rows from row0 on; rows that no sequence has are not live.  Offsets that are no offsets lead nowhere outside the rows.
template <int L> __device__ __forceinline__ Marks marks_of(const RecurArgs &A, uint32_t tile0, uint32_t row0) {
    const uint32_t lane = threadIdx.x & 63u, row = lane == L ? tile0 : row0 + lane;
    Marks m{0, 0, 0, 0, 0, 0, false};
    bool live = lane <= L && row < A.n_rows;
    if (A.offsets) {
        if (live) {
            // the last sequence that begins at this row or before it (of the most sequences there are 2^31 numbers from lo to hi)
            int32_t lo = -1, hi = (int32_t)(A.n_seqs + 1u);
            while ((uint32_t)hi - (uint32_t)lo > 1u) {
                const int32_t mid = lo + (int32_t)(((uint32_t)hi - (uint32_t)lo) / 2u);
                if (A.offsets[mid] <= (int32_t)row) lo = mid; else hi = mid;
            }
            live = lo >= 0 && lo < (int32_t)A.n_seqs;
            if (live) {
                m.seq = lo;
                m.begin = max(A.offsets[lo], 0);
                m.end = min(A.offsets[lo + 1], (int32_t)A.n_rows);
            }
        }
    } else if (live) {
        m.seq = (int32_t)(row / A.seq_rows);
        m.begin = m.seq * (int32_t)A.seq_rows;
        m.end = (int32_t)(A.n_rows - (uint32_t)m.begin < A.seq_rows ? A.n_rows : (uint32_t)m.begin + A.seq_rows);
    }
    // (lanes' registers are read here alone, where all lanes are at work: elsewhere one may have been brought back from memory for some of them)
    constexpr uint32_t ROWS = (1u << L) - 1u;
    const uint32_t lives = (uint32_t)__builtin_amdgcn_ballot_w64(live);
    m.live = lives & ROWS;
    m.first = (uint32_t)__builtin_amdgcn_ballot_w64(live && (int32_t)row == m.begin) & ROWS;
    m.last = (uint32_t)__builtin_amdgcn_ballot_w64(live && (int32_t)row + 1 == m.end) & ROWS;
    m.plain = (lives >> L & 1u) && (uint32_t)__builtin_amdgcn_readlane(m.begin, L) < tile0 && (uint32_t)__builtin_amdgcn_readlane(m.end, L) > tile0 + RC_WAVES * L;
    return m;
}

// ---- chains
struct Link { Vec<float, 2> p, q; };            // v -> p v + q
__device__ __forceinline__ uint32_t not_all_ones(float v) {
    const uint32_t w = __float_as_uint(v);
    return w == 0xFFFFFFFFu ? 0x7FC00000u : w;  // (one NaN for another)
}
struct Lds {
    Vec<float, 2> p[RC_WAVES][64], q[RC_WAVES][64];         // the wavefronts' links; those of the tiles before, a run a wavefront
    Vec<float, 2> jp[RC_WAVES][64], jq[RC_WAVES][64];
    uint32_t cuts;                              // wavefronts in which a chain begins
    uint32_t ticket;
    int32_t seq[RC_WAVES][64];                  // a row's sequence, for code that not all lanes are in
    __device__ __forceinline__ void keep(uint32_t wave, int32_t of_lane) {
        seq[wave][threadIdx.x & 63u] = of_lane;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    __device__ __forceinline__ uint32_t seq_of(uint32_t wave, int i) const { return (uint32_t)__builtin_amdgcn_readfirstlane(seq[wave][i]); }
};
// what the first n wavefronts make of a value, in the direction of the chain
__device__ __forceinline__ Link link_of(const Lds &lds, uint32_t n, uint32_t cuts) {
    const uint32_t lane = threadIdx.x & 63u;
    Link l;
    l.p = 1.f; l.q = 0.f;
    for (uint32_t w = 0; w < n; ++w) {
        const Vec<float, 2> p = lds.p[w][lane], q = lds.q[w][lane];
        if (cuts >> w & 1u) { l.p = 0.f; l.q = q; }
        else { l.q = p * l.q + q; l.p = l.p * p; }
    }
    return l;
}
// The value that comes in to this wavefront's rows.  order: its place in the direction of the chain; cut: a chain begins in its rows; needs: its
// tile's first row goes on with a chain that began in tile `from` (tiles counted in the direction of the chain).  (Links are folded anew where they are
// wanted: the rows leave no registers to keep them in.)
__device__ __forceinline__ Vec<float, 2> join(const RecurArgs &A, Lds &lds, uint32_t order, const Link &own, bool cut, uint32_t tile, uint32_t column, bool needs, uint32_t from) {
    const uint32_t lane = threadIdx.x & 63u;
    lds.p[order][lane] = own.p;
    lds.q[order][lane] = own.q;
    if (lane == 0 && cut) atomicOr(&lds.cuts, 1u << order);
    __syncthreads();
    const uint32_t cuts = __builtin_amdgcn_readfirstlane(lds.cuts);
    if (!A.ticket) return link_of(lds, order, cuts).q;      // (nothing comes in to any tile)
    if (order == RC_WAVES - 1) {
        const Link all = link_of(lds, RC_WAVES, cuts);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (column + i < A.width)
                __hip_atomic_store(A.steps + (uint64_t)tile * A.width + column + i, (uint64_t)not_all_ones(all.q[i]) << 32 | not_all_ones(cuts ? 0.f : all.p[i]),
                                   __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    Vec<float, 2> in = 0.f;
    if (needs) {
        const uint32_t block = tile / RC_BLOCK * RC_BLOCK, begin = from > block ? from : block, n = tile - begin;
        // the tiles before this one, a run of them a wavefront, and the value behind the block before
        const uint32_t a = begin + n * order / RC_WAVES, b = begin + n * (order + 1) / RC_WAVES;
        // (lanes wait together, those behind the last column with it: were some of them to go on alone, what does not fit the registers might be written down for
        // them alone)
        const uint32_t c0 = column < A.width ? column : A.width - 1, c1 = column + 1 < A.width ? column + 1 : A.width - 1;
        Vec<float, 2> jp = 1.f, jq = 0.f;
        for (uint32_t t = a; t < b; ++t) {
            const uint64_t *const at = A.steps + (uint64_t)t * A.width;
            uint64_t word[2];
            while (word[0] = __hip_atomic_load(at + c0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), word[1] = __hip_atomic_load(at + c1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT),
                   __builtin_amdgcn_ballot_w64(word[0] == ~0ull || word[1] == ~0ull))
                __builtin_amdgcn_s_sleep(RC_NAP);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float tp = __uint_as_float((uint32_t)word[i]), tq = __uint_as_float((uint32_t)(word[i] >> 32));
                jq[i] = tp * jq[i] + tq;
                jp[i] *= tp;
            }
        }
        if (order == 0 && from < block) {       // (the first of the runs goes on from there)
            const uint32_t *const at = A.behind + (uint64_t)(tile / RC_BLOCK - 1) * A.width;
            uint32_t word[2];
            while (word[0] = __hip_atomic_load(at + c0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), word[1] = __hip_atomic_load(at + c1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT),
                   __builtin_amdgcn_ballot_w64(word[0] == ~0u || word[1] == ~0u))
                __builtin_amdgcn_s_sleep(RC_NAP);
            in[0] = __uint_as_float(word[0]); in[1] = __uint_as_float(word[1]);
            jq = jp * in + jq;
            in = 0.f;
        }
        lds.jp[order][lane] = jp;
        lds.jq[order][lane] = jq;
        __syncthreads();                        // (needs is the same for the whole workgroup)
#pragma unroll
        for (uint32_t w = 0; w < RC_WAVES; ++w) in = lds.jp[w][lane] * in + lds.jq[w][lane];
    }
    // the value behind the tile, if it is a block's last: the next block is waiting for it
    if (order == RC_WAVES - 1 && tile % RC_BLOCK == RC_BLOCK - 1) {
        const Link all = link_of(lds, RC_WAVES, cuts);
        const Vec<float, 2> behind = cuts ? all.q : all.p * in + all.q;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (column + i < A.width)
                __hip_atomic_store(A.behind + (uint64_t)(tile / RC_BLOCK) * A.width + column + i, not_all_ones(behind[i]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    const Link before = link_of(lds, order, cuts);
    return cuts & ((1u << order) - 1u) ? before.q : before.p * in + before.q;
}
// Which tile a workgroup has; false: none, it looked for sequences without rows instead, whose state goes from one end to the other.
__device__ __forceinline__ bool take(const RecurArgs &A, Lds &lds, const float *from, uint64_t from_st, float *to, uint64_t to_st, uint32_t &tile, uint32_t &column_tile) {
    const uint32_t tiles = A.n_tiles * A.n_cols;
    if (threadIdx.x == 0) {
        lds.cuts = 0;
        lds.ticket = A.ticket && blockIdx.x < tiles ? atomicAdd(A.ticket + blockIdx.x % A.n_cols * RC_TICKET, 1u) : 0u;
    }
    __syncthreads();
    if (blockIdx.x < tiles) {
        tile = A.ticket ? lds.ticket : blockIdx.x / A.n_cols;
        column_tile = blockIdx.x % A.n_cols;
        return true;
    }
    for (uint32_t s = (blockIdx.x - tiles) * RC_WAVES + (threadIdx.x >> 6); s < A.n_seqs; s += A.idle * RC_WAVES) {
        const bool none = A.offsets ? A.offsets[s + 1] <= A.offsets[s] : A.n_rows == 0;
        if (none)
            for (uint32_t c = threadIdx.x & 63u; c < A.width; c += 64) to[s * to_st + c] = from ? from[s * from_st + c] : 0.f;
    }
    return false;
}

// Rows of a wavefront: of 32 bits half as many, which is what the registers hold (8192 x 4096 forward 92 us, with sixteen 109).
template <typename T> constexpr int rows_of() { return sizeof(T) == 4 ? RC_ROWS / 2 : RC_ROWS; }
// The rows' steps stay in registers until what comes in to them is known.
template <typename T, bool COUPLED, bool CUT> __global__ __launch_bounds__(RC_THREADS, 4) void k_recur_forward(const RecurArgs A) {
    __shared__ Lds lds;
    constexpr int L = rows_of<T>();
    uint32_t tile, column_tile;
    if (!take(A, lds, A.state_in, A.si_st, A.state_out, A.so_st, tile, column_tile)) return;
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t column = column_tile * RC_COLS + 2 * lane, tile0 = tile * RC_WAVES * L, row0 = __builtin_amdgcn_readfirstlane(tile0 + wave * L);
    const Columns c(column, A.width);
    Two<T> z[L], x[L];
    read_rows<CUT, L, T>(z, A.z, A.z_st, row0, A.n_rows, c, A.width);
    read_rows<CUT, L, T>(x, A.x, A.x_st, row0, A.n_rows, c, A.width);
    const Marks m = marks_of<L>(A, tile0, row0);
    lds.keep(wave, m.seq);
    Vec<float, 2> bias;
    bias[0] = bias_of<T>(bias_at(A, column)); bias[1] = bias_of<T>(bias_at(A, column + 1));
    auto rows = [&](auto plain) {
        constexpr bool PLAIN = decltype(plain)::value;
        Vec<float, 2> f[L], q[L];
        Link own;
        own.p = 1.f; own.q = 0.f;
#pragma unroll
        for (int g = 0; g < L / 4; ++g) {
            Vec<float, 2> state[4];
            if (!PLAIN && A.state_in && (m.first >> 4 * g & 15u))
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (m.first >> (4 * g + k) & 1u) state[k] = read_state<CUT>(A.state_in, A.si_st, lds.seq_of(wave, 4 * g + k), c, A.width);
#pragma unroll
            for (int i = 4 * g; i < 4 * g + 4; ++i) {
                const Vec<float, 2> zi = floats<CUT, T>(z[i], c), xi = floats<CUT, T>(x[i], c);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const Gate gate = gate_of<T>(zi[k], bias[k]);
                    f[i][k] = gate.f;
                    q[i][k] = COUPLED ? gate.not_f * xi[k] : xi[k];
                }
                if (!PLAIN) {
                    if (!(m.live >> i & 1u)) { f[i] = 1.f; q[i] = 0.f; }
                    if (m.first >> i & 1u) {
                        if (A.state_in) q[i] += f[i] * state[i % 4];
                        own.p = 0.f; own.q = 0.f;
                    }
                }
                own.p *= f[i];
                own.q = f[i] * own.q + q[i];
            }
            __builtin_amdgcn_sched_barrier(0);              // (four rows at a time: more under way would not fit the registers)
        }
        // how the tile's first row goes on
        __shared__ uint32_t from;
        if (threadIdx.x == 0) from = PLAIN || ((m.live & 1u) && !(m.first & 1u)) ? (uint32_t)m.begin / (RC_WAVES * L) : ~0u;     // (its lane's row)
        __syncthreads();
        const Vec<float, 2> in = join(A, lds, wave, own, !PLAIN && m.first != 0, tile, column, from != ~0u, from);
        where_columns<CUT>(c, [&](auto one) {
            constexpr bool ONE = decltype(one)::value;
            T *to = (T *)A.out + (uint64_t)row0 * A.o_st;
            Vec<float, 2> h = in;
#pragma unroll
            for (int i = 0; i < L; ++i) {
                if (!PLAIN && (m.first >> i & 1u)) h = 0.f;
                h = f[i] * h + q[i];
                if (PLAIN || (m.live >> i & 1u)) write_two<ONE>(to, column, h);
                if (!PLAIN && A.state_out && (m.last >> i & 1u)) write_two<ONE>(A.state_out + lds.seq_of(wave, i) * A.so_st, column, h);
                to += A.o_st;
            }
        });
    };
    if (m.plain) rows(std::true_type()); else rows(std::false_type());
}

// The rows wait for what comes in to them as they were read, and their gates are made a second time behind it: so a wavefront holds as many
// of the four matrices as it does forward of two.
template <typename T, bool COUPLED, bool CUT> __global__ __launch_bounds__(RC_THREADS, 4) void k_recur_backward(const RecurArgs A) {
    __shared__ Lds lds;
    constexpr int L = rows_of<T>();
    uint32_t tile, column_tile;                     // (counted from the last rows)
    if (!take(A, lds, A.d_state_out, A.dso_st, A.d_state_in, A.dsi_st, tile, column_tile)) return;
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t column = column_tile * RC_COLS + 2 * lane, tile0 = (A.n_tiles - 1 - tile) * RC_WAVES * L, row0 = __builtin_amdgcn_readfirstlane(tile0 + wave * L);
    const Columns c(column, A.width);
    Two<T> z[L], x[L], h[L], dh[L];
    read_rows<CUT, L, T>(z, A.z, A.z_st, row0, A.n_rows, c, A.width);
    read_rows<CUT, L, T>(dh, A.dh, A.dh_st, row0, A.n_rows, c, A.width);
    if constexpr (COUPLED) read_rows<CUT, L, T>(x, A.x, A.x_st, row0, A.n_rows, c, A.width);
    // (the rows before; before the matrix's first stands that one, which is not used)
    {
        const T *p = (const T *)A.h + (uint64_t)(row0 == 0 ? 0 : row0 <= A.n_rows ? row0 - 1 : A.n_rows - 1) * A.h_st;
#pragma unroll
        for (int i = 0; i < L; ++i) {
            h[i] = read_two<CUT, T>(p, c, A.width);
            p += row0 + i > 0 && row0 + i < A.n_rows ? A.h_st : 0;
        }
    }
    const Marks m = marks_of<L>(A, tile0, row0);
    lds.keep(wave, m.seq);
    Vec<float, 2> bias, sum = 0.f;
    bias[0] = bias_of<T>(bias_at(A, column)); bias[1] = bias_of<T>(bias_at(A, column + 1));
    const uint32_t order = RC_WAVES - 1 - wave;
    auto rows = [&](auto plain) {
        constexpr bool PLAIN = decltype(plain)::value;
        // rows 4 g .. 4 g + 3, the last first: row(i, ..), with what behind the last row of a sequence comes in to it, and cut() before that one
        auto four = [&](int g, auto cut, auto row) {
            Vec<float, 2> d_state[4];
            if (!PLAIN && A.d_state_out && (m.last >> 4 * g & 15u))
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (m.last >> (4 * g + k) & 1u) d_state[k] = read_state<CUT>(A.d_state_out, A.dso_st, lds.seq_of(wave, 4 * g + k), c, A.width);
#pragma unroll
            for (int k = 3; k >= 0; --k) {
                const int i = 4 * g + k;
                const Vec<float, 2> zi = floats<CUT, T>(z[i], c);
                Vec<float, 2> e = floats<CUT, T>(dh[i], c), f, not_f;
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const Gate gate = gate_of<T>(zi[n], bias[n]);
                    f[n] = gate.f; not_f[n] = gate.not_f;
                }
                if (!PLAIN) {
                    if (!(m.live >> i & 1u)) { f = 1.f; e = 0.f; }
                    if (m.last >> i & 1u) {
                        if (A.d_state_out) e += d_state[k];
                        cut();
                    }
                }
                row(i, e, f, not_f);
            }
            __builtin_amdgcn_sched_barrier(0);              // (four rows at a time: more under way would not fit the registers)
        };
        Link own;
        own.p = 1.f; own.q = 0.f;
#pragma unroll
        for (int g = L / 4 - 1; g >= 0; --g)
            four(g, [&]() { own.p = 0.f; own.q = 0.f; }, [&](int, const Vec<float, 2> &e, const Vec<float, 2> &f, const Vec<float, 2> &) {
                own.p *= f;
                own.q = f * (e + own.q);
            });
        __shared__ uint32_t from;
        // how the tile's last row goes on; a tile of the matrix's end is cut short there, and nothing comes in to it
        if (threadIdx.x == RC_THREADS - 64 + L - 1)         // (its lane's row)
            from = PLAIN || ((m.live >> (L - 1) & 1u) && !(m.last >> (L - 1) & 1u)) ? A.n_tiles - 1 - (uint32_t)(m.end - 1) / (RC_WAVES * L) : ~0u;
        __syncthreads();
        const Vec<float, 2> in = join(A, lds, order, own, !PLAIN && m.last != 0, tile, column, from != ~0u, from);
        // (nothing that is made of the rows is to be kept for here, or made ahead)
#pragma unroll
        for (int i = 0; i < L; ++i)
#pragma unroll
            for (int k = 0; k < (int)sizeof(T) / 2; ++k) {
                uint32_t v[4] = {z[i][k], dh[i][k], COUPLED ? x[i][k] : 0u, h[i][k]};
                asm volatile("" : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3]));
                z[i][k] = v[0]; dh[i][k] = v[1]; x[i][k] = v[2]; h[i][k] = v[3];
            }
        where_columns<CUT>(c, [&](auto one) {
            constexpr bool ONE = decltype(one)::value;
            T *to_x = (T *)A.dx + (uint64_t)(row0 + L - 1) * A.dx_st, *to_z = (T *)A.dz + (uint64_t)(row0 + L - 1) * A.dz_st;
            Vec<float, 2> carry = in;
#pragma unroll
            for (int g = L / 4 - 1; g >= 0; --g) {
                Vec<float, 2> state[4];
                if (!PLAIN && A.state_in && (m.first >> 4 * g & 15u))
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (m.first >> (4 * g + k) & 1u) state[k] = read_state<CUT>(A.state_in, A.si_st, lds.seq_of(wave, 4 * g + k), c, A.width);
                four(g, [&]() { carry = 0.f; }, [&](int i, const Vec<float, 2> &e, const Vec<float, 2> &f, const Vec<float, 2> &not_f) {
                    const Vec<float, 2> now = e + carry;
                    carry = f * now;
                    if (PLAIN || (m.live >> i & 1u)) {
                        const bool first = !PLAIN && (m.first >> i & 1u);
                        Vec<float, 2> of = floats<CUT, T>(h[i], c);
                        if (first) of = A.state_in ? state[i % 4] : Vec<float, 2>(0.f);
                        if (COUPLED) of -= floats<CUT, T>(x[i], c);
                        const Vec<float, 2> dz = now * of * (f * not_f);
                        sum += dz;
                        write_two<ONE>(to_x, column, COUPLED ? not_f * now : now);
                        write_two<ONE>(to_z, column, dz);
                        if (A.d_state_in && first) write_two<ONE>(A.d_state_in + lds.seq_of(wave, i) * A.dsi_st, column, carry);
                    }
                    to_x -= A.dx_st; to_z -= A.dz_st;
                });
            }
        });
    };
    if (m.plain) rows(std::true_type()); else rows(std::false_type());
    if (!A.d_bias) return;
    __syncthreads();
    lds.p[wave][lane] = sum;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (uint32_t w = 1; w < RC_WAVES; ++w) sum += lds.p[w][lane];
    float *const to = A.n_tiles > 1 ? A.bias_parts + (uint64_t)tile * A.width : A.d_bias;
#pragma unroll
    for (int k = 0; k < 2; ++k) if (column + k < A.width) to[column + k] = sum[k];
}

// sixteen runs of tiles a column, joined in fixed order
__global__ __launch_bounds__(1024) void k_recur_bias(const float *parts, uint32_t n_tiles, uint32_t width, float *d_bias) {
    __shared__ float lds[16][64];
    const uint32_t lane = threadIdx.x & 63u, run = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    float sum = 0.f;
    if (c < width) {
        const uint32_t end = (uint32_t)((uint64_t)n_tiles * (run + 1) / 16);
        for (uint32_t t = (uint32_t)((uint64_t)n_tiles * run / 16); t < end; ++t) sum += parts[(uint64_t)t * width + c];
    }
    lds[run][lane] = sum;
    __syncthreads();
    if (run || c >= width) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) sum += lds[i][lane];
    d_bias[c] = sum;
}
__global__ __launch_bounds__(256) void k_recur_clear(uint64_t *words, uint64_t n, uint32_t *ticket, uint32_t n_tickets) {
    for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < n_tickets; i += gridDim.x * 256) ticket[i] = 0;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (uint64_t)gridDim.x * 256) words[i] = ~0ull;
}

// f(type, coupled, whether rows have an odd number of elements)
template <typename F> void with_kernel(const RecurArgs &A, uint32_t type, F f) {
    auto cut = [&](auto t, auto coupled) { if (A.width % 2) f(t, coupled, std::true_type()); else f(t, coupled, std::false_type()); };
    auto typed = [&](auto t) { if (A.coupled) cut(t, std::true_type()); else cut(t, std::false_type()); };
    if (type == RK_F32) typed(float()); else if (type == RK_BF16) typed(__bf16()); else typed(_Float16());
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
        return rk_fail(ctx, RK_ERR_UNSUPPORTED, "more than 2^31 - 1 rows, 2^31 - 2 sequences or %u columns", RK_RECUR_MAX_WIDTH);
    if (!rk_matrix_ok(z, n_rows, width)) return rk_fail(ctx, RK_ERR_INVALID_ARG, "z null, misaligned or of a stride below the width");
    n_seqs = r->offsets ? r->n_seqs : r->seq_rows ? n_rows / r->seq_rows + (n_rows % r->seq_rows != 0) : 1;
    return RK_OK;
}
bool alike(const rk_matrix *m, const rk_matrix *z, uint64_t n_rows, uint32_t width) { return rk_matrix_ok(m, n_rows, width) && m->type == z->type; }
bool state_ok(const rk_matrix *m, uint64_t n_seqs, uint32_t width) { return !m || (rk_matrix_ok(m, n_seqs, width) && m->type == RK_F32); }
void fill_recur(RecurArgs &A, const rk_recur *r, uint64_t n_rows, uint32_t width, uint64_t n_seqs, const rk_matrix *z) {
    A.z = z->data; A.z_st = z->stride;
    A.bias = r->bias; A.bias_type = r->param_type;
    A.offsets = r->offsets;
    A.seq_rows = (uint32_t)(r->seq_rows && r->seq_rows < n_rows ? r->seq_rows : n_rows);
    A.n_rows = (uint32_t)n_rows; A.n_seqs = (uint32_t)n_seqs; A.width = width; A.coupled = r->coupled;
}
uint32_t tile_rows(uint32_t type) { return RC_WAVES * (uint32_t)(type == RK_F32 ? rows_of<float>() : rows_of<__bf16>()); }
// tiles of tile_rows rows, and what their chains need; the number of workgroups
int32_t tiles_of(rk_ctx *ctx, RecurArgs &A, uint32_t rows, bool states, uint64_t &blocks) {
    A.n_tiles = (uint32_t)(((uint64_t)A.n_rows + rows - 1) / rows);
    A.n_cols = (A.width + RC_COLS - 1) / RC_COLS;
    // (of sequences without rows there is only the state to be taken along)
    A.idle = states && (A.offsets || A.n_rows == 0) ? (A.n_seqs / RC_WAVES < 1024 ? A.n_seqs / RC_WAVES + 1 : 1024) : 0;
    blocks = (uint64_t)A.n_tiles * A.n_cols + A.idle;
    if (blocks > RK_LAUNCH_THREADS / RC_THREADS) return rk_fail(ctx, RK_ERR_UNSUPPORTED, "2^22 tiles of %u rows and %u columns or more", rows, RC_COLS);
    if (A.n_tiles < 2) return RK_OK;
    int32_t rc;
    if (A.d_bias && (rc = rk_scratch(ctx, SL_RECUR_BIAS, (uint64_t)A.n_tiles * A.width * 4, (void **)&A.bias_parts)) != RK_OK) return rc;
    // whole sequences in every tile, as in a step of serving, have nothing to tell (1,024 x 2,048, one row each: 9.3 us a call, with a chain 13.9)
    if (!A.offsets && rows % A.seq_rows == 0) return RK_OK;
    const uint64_t words = (uint64_t)A.n_tiles * A.width, after = ((uint64_t)(A.n_tiles / RC_BLOCK) * A.width + 1) / 2;
    rc = rk_scratch(ctx, SL_RECUR_CHAIN, (words + after) * 8 + (uint64_t)A.n_cols * RC_TICKET * 4, (void **)&A.steps);
    if (rc != RK_OK) return rc;
    A.behind = (uint32_t *)(A.steps + words);
    A.ticket = (uint32_t *)(A.steps + words + after);
    const uint64_t clear = (words + after + 1023) / 1024;
    k_recur_clear<<<(uint32_t)(clear < 2048 ? clear : 2048), 256, 0, ctx->stream>>>(A.steps, words + after, A.ticket, A.n_cols * RC_TICKET);
    RK_CHECK_LAUNCH(ctx, "k_recur_clear");
    return RK_OK;
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
    uint64_t blocks;
    if ((rc = tiles_of(ctx, A, tile_rows(z->type), state_out != nullptr, blocks)) != RK_OK) return rc;
    with_kernel(A, z->type, [&](auto t, auto coupled, auto cut) {
        k_recur_forward<decltype(t), decltype(coupled)::value, decltype(cut)::value><<<(uint32_t)blocks, RC_THREADS, 0, ctx->stream>>>(A);
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
    uint64_t blocks;
    if ((rc = tiles_of(ctx, A, tile_rows(z->type), d_state_in != nullptr, blocks)) != RK_OK) return rc;
    if (blocks) {
        with_kernel(A, z->type, [&](auto t, auto coupled, auto cut) {
            k_recur_backward<decltype(t), decltype(coupled)::value, decltype(cut)::value><<<(uint32_t)blocks, RC_THREADS, 0, ctx->stream>>>(A);
        });
        RK_CHECK_LAUNCH(ctx, "k_recur_backward");
    }
    if (d_bias && A.n_tiles != 1) {
        k_recur_bias<<<(width + 63) / 64, 1024, 0, ctx->stream>>>(A.bias_parts, A.n_tiles, width, d_bias);
        RK_CHECK_LAUNCH(ctx, "k_recur_bias");
    }
    return RK_OK;
}
