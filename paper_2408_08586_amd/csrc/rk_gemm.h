// Matrix products of the operators: out[b][a] = sum over k of A(a, k) B(b, k), held in float32.
//
// A workgroup of eight wavefronts makes a tile of TA x TB.  64 bytes of k at a time, both tiles go from memory straight into one of
// four places in LDS; fragments are read from there one step ahead of the products that take them, between the products of the step before, so that the matrix
// units, the reads of LDS and the loads from memory of the three steps that follow run side by side, with one barrier a step.  A wavefront
// has 128 x 64 sums of the largest tile, which 128 registers hold beside the two steps' fragments: with four wavefronts of 128 x 128, LDS is read a quarter less
// and nothing else runs on a SIMD while its one wavefront waits at the barrier.
// A side lies with k along its rows (ALONG) or with k from row to row (ACROSS), and so it comes into LDS; nothing is turned around beforehand:
//   ALONG   64 bytes a row.  A lane's part of a fragment is a 16-byte piece of its row; pieces lie in the order piece ^ something that rows
//           which are read together do not share, so that they do not meet in the banks.
//   ACROSS  a row of TA (TB) elements for every k.  Of narrow elements, sixteen lanes read four k of sixteen elements and get them
//           turned around by the LDS unit; of 32-bit ones, a lane reads its element of each k.  Pieces lie in the order piece ^ something that
//           the k of the lanes that read together do not share.
// Memory gives pieces in that order, as LDS is written in the order of the lanes.  The matrix units take sixteen elements of 32 narrow k at once, or of four
// 32-bit ones: there, each of four products takes one k of every lane's four, the same of both sides.
//
// Measured with 1,843 rows, 128,000 words and a width of 5,248 in bfloat16 (2.48 TFLOP a product): logits 2.19 ms, dx 2.25, d_weight 2.40, that is 1,130, 1,100 and
// 1,030 TFLOP/s, where large products of a library reach 1,260 to 1,310; what the matrix units do (rows up to whole tiles with it) fills 0.63, 0.66 and
// 0.54 of the cycles, at the 1.9 GHz that the card then holds.  In 32 bits (1,024 x 32,000 x 2,048, 134 GFLOP): 0.96 ms, 0.93 and 1.02, 140, 145 and 131 of the 152
// TFLOP/s that a library reaches.  d_weight has the shortest sums: what a tile spends before its first product and on writing is not covered.
#pragma once
#include <type_traits>

#include "rk_vec.h"

namespace {

constexpr uint32_t GM_WAVES = 8, GM_THREADS = 64 * GM_WAVES, GM_STEP = 64;          // threads; bytes of k of a step
constexpr uint32_t GM_NOWHERE = 0x80000000u;                // a lane's place behind every buffer: zeros

// c += a b, the sums staying in their registers (as a builtin, whose result may go anywhere, they wander from step to step, and what does not
// fit then is spilled).  The instruction's hazards are the caller's: sums are taken again three products later at the earliest, and read
// by others behind settle().
// (instructions and builtins of this GPU alone: the host's pass over the source does not know them)
template <typename T> __device__ __forceinline__ void product(const Vec<uint32_t, 4> &a, const Vec<uint32_t, 4> &b, int q, Vec<float, 4> &c) {
#ifdef __HIP_DEVICE_COMPILE__
    if constexpr (sizeof(T) == 4) asm volatile("v_mfma_f32_16x16x4_f32 %0, %1, %2, %0" : "+v"(c) : "v"(a[q]), "v"(b[q]));
    else if constexpr (__is_same(T, __bf16)) asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(c) : "v"(a), "v"(b));
    else asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+v"(c) : "v"(a), "v"(b));
#endif
}
__device__ __forceinline__ void into_lds(__amdgpu_buffer_rsrc_t buf, char *lds, uint32_t at) {
#ifdef __HIP_DEVICE_COMPILE__
    __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (__attribute__((address_space(3))) void *)lds, 16, at, 0, 0, 0);
#endif
}
// sixteen lanes give 8 bytes each, four rows of sixteen narrow elements; a lane gets its element of the four rows
__device__ __forceinline__ Vec<uint32_t, 2> turned(const char *lds) {
#ifdef __HIP_DEVICE_COMPILE__
    return __builtin_bit_cast(Vec<uint32_t, 2>, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) Vec<short, 4> *)const_cast<char *>(lds)));
#else
    return Vec<uint32_t, 2>{0u, 0u};
#endif
}
// Until no more than N of the wavefront's loads are under way, then until all wavefronts are here.
template <int N> __device__ __forceinline__ void landed() {
    asm volatile("" ::: "memory");
#ifdef __HIP_DEVICE_COMPILE__
    __builtin_amdgcn_s_waitcnt((0xC07F & ~0xC00F) | (N & 0xF) | (N >> 4 << 14));   // vmcnt(N) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
#endif
    asm volatile("" ::: "memory");
}

enum { ALONG = 0, ACROSS = 1 };
// One side of a product, its first byte and stride multiples of 16.
struct Side {
    const char *data;
    uint64_t stride;            // bytes from row to row
    uint64_t count;             // ALONG: rows; ACROSS: bytes of a row
};
// ALONG: a piece of row r lies at piece ^ {0, 2, 3, 1}[r / 4 % 4].  LDS takes a read of 16 bytes a lane in four parts, lanes 0 to 3, 12 to 15 and 20 to 27 in
// the first; with {0, 1, 2, 3} half of these met in the banks (4 more cycles a read, counted, and the same time: the matrix units' covers them).
__device__ __forceinline__ uint32_t order_along(uint32_t r) { return 0x78u >> (r >> 1 & 6u) & 3u; }
// ACROSS: a piece of k's row lies at piece ^ order_of(k): pairs of pieces change places (of 32-bit elements fours), differently for all k that
// are read together
template <typename T, uint32_t PIECES> __device__ __forceinline__ uint32_t order_of(uint32_t k) {
    static_assert((PIECES & (PIECES - 1)) == 0, "");
    if constexpr (sizeof(T) == 4) return (k >> 2 & 3u) * 4u % PIECES;
    else return ((k & 3u) | (k >> 3 & 3u) << 2) * 2u % PIECES;
}
// What a wavefront asks for of a tile of R elements, which is R / 16 instructions of 1,024 bytes: an eighth of these, rounded up, some of them twice, so
// that every wavefront has as many under way.
template <typename T, int R, int WAY> struct Fetch {
    static constexpr int N = (R / 16 + (int)GM_WAVES - 1) / (int)GM_WAVES;
    static constexpr uint32_t KS = GM_STEP / sizeof(T), PIECES = R * sizeof(T) / 16;    // k of a step; ACROSS: pieces of a row of LDS
    const char *base;
    uint64_t hop;               // bytes from step to step
    uint32_t at[N], tail[N];    // of a lane, and in the last step
    static __device__ __forceinline__ uint32_t part(int i) { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * N % (R / 16) + i; }
    __device__ __forceinline__ Fetch(const Side &s, uint64_t first, uint64_t k0, uint32_t ks) {
        const uint32_t lane = threadIdx.x & 63u, left = ks % KS ? ks % KS : KS;
        if constexpr (WAY == ALONG) {
            base = s.data + first * s.stride + k0 * sizeof(T);
            hop = GM_STEP;
            const uint64_t rows = s.count - first;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                uint32_t r = part(i) * 16 + (lane >> 2);
                const uint32_t piece = (lane & 3u) ^ order_along(r);
                r = r < rows ? r : (uint32_t)(rows - 1);    // (rows behind the last repeat it: their results go nowhere)
                at[i] = r * (uint32_t)s.stride + piece * 16;
                tail[i] = piece * (16 / sizeof(T)) < left ? at[i] : GM_NOWHERE;
            }
        } else {
            base = s.data + k0 * s.stride + first * sizeof(T);
            hop = KS * s.stride;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t x = part(i) * 64 + lane, k = x / PIECES, piece = (x % PIECES) ^ order_of<T, PIECES>(k);
                at[i] = first * sizeof(T) + piece * 16 < s.count ? k * (uint32_t)s.stride + piece * 16 : GM_NOWHERE;
                tail[i] = k < left ? at[i] : GM_NOWHERE;
            }
        }
    }
    // step s of `steps` into LDS; LAST: of the last one what is left of k, zeros behind it and of steps that there are not
    template <bool LAST> __device__ __forceinline__ void into(char *lds, uint32_t s, uint32_t steps) const {
        const __amdgpu_buffer_rsrc_t buf = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base) + (!LAST || s < steps ? s : 0) * hop, 0, (int)GM_NOWHERE, 0x00027000);
#pragma unroll
        for (int i = 0; i < N; ++i) into_lds(buf, lds + part(i) * 1024, !LAST || s + 1 < steps ? at[i] : s < steps ? tail[i] : GM_NOWHERE);
    }
};
// A wavefront's fragments, sixteen elements each, from element `first` of the tile on (a multiple of what the wavefront has)
template <typename T, int R, int WAY> struct Reader {
    static constexpr uint32_t PITCH = R * sizeof(T), PIECES = PITCH / 16;
    uint32_t at;
    __device__ __forceinline__ Reader(uint32_t first) {
        const uint32_t lane = threadIdx.x & 63u, j = lane & 15u, g = lane >> 4;
        if constexpr (WAY == ALONG) {
            at = (first + j) * GM_STEP + (g ^ order_along(j)) * 16;
        } else if constexpr (sizeof(T) == 4) {
            const uint32_t k = 4 * g, piece = first / 4 + (j >> 2);
            at = k * PITCH + (piece ^ order_of<T, PIECES>(k)) * 16 + (j & 3u) * 4;
        } else {
            const uint32_t k = 8 * g + (j >> 2), piece = first / 8 + (j >> 1 & 1u);
            at = k * PITCH + (piece ^ order_of<T, PIECES>(k)) * 16 + (j & 1u) * 8;
        }
    }
    // fragment i (ACROSS: its pieces' numbers differ from the first one's in bits that these do not have, and so do their places)
    __device__ __forceinline__ Vec<uint32_t, 4> read(const char *lds, int i) const {
        if constexpr (WAY == ALONG) {
            return *(const Vec<uint32_t, 4> *)(lds + at + i * 16 * GM_STEP);
        } else {
            const char *const p = lds + (at ^ (uint32_t)(i * 16 * sizeof(T)));
            if constexpr (sizeof(T) == 4) {
                Vec<uint32_t, 4> w;
#pragma unroll
                for (int q = 0; q < 4; ++q) w[q] = *(const uint32_t *)(p + q * PITCH);
                return w;
            } else {
                const Vec<uint32_t, 2> lo = turned(p), hi = turned(p + 4 * PITCH);
                return Vec<uint32_t, 4>{lo[0], lo[1], hi[0], hi[1]};
            }
        }
    }
};

// The tile at (a0, b0) over ks of k from k0 on; WA x WB wavefronts share it.  acc[i][j]: lane l holds the elements
// a = a0 + wa TA/WA + 16 i + 4 (l / 16) + 0..3,  b = b0 + wb TB/WB + 16 j + l % 16.
template <typename T, int TA, int TB, int WA, int WAY_A, int WAY_B> struct Tile {
    static constexpr int WB = (int)GM_WAVES / WA, MA = TA / WA / 16, MB = TB / WB / 16;
    static constexpr uint32_t KS = GM_STEP / sizeof(T), GRAIN = 4 * KS;         // k of a step; of a turn of the loop, which is done whole
    typedef Fetch<T, TA, WAY_A> FetchA;
    typedef Fetch<T, TB, WAY_B> FetchB;
    typedef Reader<T, TA, WAY_A> ReadA;
    typedef Reader<T, TB, WAY_B> ReadB;
    static constexpr int EACH = FetchA::N + FetchB::N;                          // a wavefront's loads of a step
    Vec<float, 4> acc[MA][MB];
    struct Fragments { Vec<uint32_t, 4> a[MA], b[MB]; };
    // The lane's place in the tile for what is made of the sums: taken anew behind the loop, which has no registers for it.
    struct At { uint32_t a, b, lane; };
    static __device__ __forceinline__ At place() {
        uint32_t t = threadIdx.x;
        asm volatile("" : "+v"(t));
        const uint32_t wave = t >> 6, lane = t & 63u;
        return At{wave / WB * (TA / WA) + 4 * (lane >> 4), wave % WB * (TB / WB) + (lane & 15u), lane};
    }
    static __device__ __forceinline__ uint32_t wave_a() { return (threadIdx.x >> 6) / WB * (TA / WA); }
    static __device__ __forceinline__ uint32_t wave_b() { return (threadIdx.x >> 6) % WB * (TB / WB); }

    static __device__ __forceinline__ void read(Fragments &f, const char *a, const char *b, const ReadA &ra, const ReadB &rb) {
#pragma unroll
        for (int j = 0; j < MB; ++j) f.b[j] = rb.read(b, j);
#pragma unroll
        for (int i = 0; i < MA; ++i) f.a[i] = ra.read(a, i);
    }
    // The products of `now`, with the next step's reads among them, in the first three quarters: what stands between two lines of products stays there.
    __device__ __forceinline__ void multiply(const Fragments &now, Fragments &next, const char *a, const char *b, const ReadA &ra, const ReadB &rb) {
        constexpr int READS = MA + MB, LINES = MB >= 4 && MA * 3 / 4 > 0 ? MA * 3 / 4 : 1, PARTS = sizeof(T) == 4 ? 4 : 1;
        auto reads = [&](int line) {
#pragma unroll
            for (int r = 0; r < READS; ++r)
                if (r * LINES / READS == line) {
                    if (r < MB) next.b[r] = rb.read(b, r); else next.a[r - MB] = ra.read(a, r - MB);
                }
            asm volatile("" ::: "memory");
        };
        if constexpr (MB >= 4) {
#pragma unroll
            for (int i = 0; i < MA; ++i) {
                reads(i);
#pragma unroll
                for (int q = 0; q < PARTS; ++q)
#pragma unroll
                    for (int j = 0; j < MB; ++j) product<T>(now.a[i], now.b[j], q, acc[i][j]);
            }
        } else {
            static_assert(MA * MB >= 4, "");                // (three others between two products for the same sums)
            reads(0);
#pragma unroll
            for (int q = 0; q < PARTS; ++q)
#pragma unroll
                for (int i = 0; i < MA; ++i)
#pragma unroll
                    for (int j = 0; j < MB; ++j) product<T>(now.a[i], now.b[j], q, acc[i][j]);
        }
    }
    // the sums as others may read them: the last products have been through the matrix units
    __device__ __forceinline__ void settle() {
#ifdef __HIP_DEVICE_COMPILE__
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
        for (int i = 0; i < MA; ++i)
#pragma unroll
            for (int j = 0; j < MB; ++j) asm volatile("" : "+v"(acc[i][j]));
#endif
    }
    // a wavefront's part of LDS behind the loop: 16 rows of TA / WA elements
    static constexpr int PART = TA / WA * 16 * (int)sizeof(T);
    char *part;
    char *shared;               // ... one of all wavefronts, 8 bytes for every WA and TB (two kilobytes and more)
    char *step_a, *step_b;      // ... and a step's place in the sides' order (step_a lies among the wavefronts' parts)

    __device__ __forceinline__ void run(const Side &A, const Side &B, uint64_t a0, uint64_t b0, uint64_t k0, uint32_t ks) {
        __shared__ __attribute__((aligned(128))) char a_0[TA * GM_STEP], a_1[TA * GM_STEP], a_2[TA * GM_STEP], a_3[TA * GM_STEP];
        __shared__ __attribute__((aligned(128))) char b_0[TB * GM_STEP], b_1[TB * GM_STEP], b_2[TB * GM_STEP], b_3[TB * GM_STEP];
#pragma unroll
        for (int i = 0; i < MA; ++i)
#pragma unroll
            for (int j = 0; j < MB; ++j) acc[i][j] = 0.f;
        {
            constexpr uint32_t HERE = TA * GM_STEP / PART;  // wavefronts whose parts one of the places holds
            const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), run = wave / HERE;
            static_assert(WA * TB * 8 <= TB * GM_STEP, "");
            shared = b_1; step_a = a_0; step_b = b_0;
            part = (run == 0 ? a_0 : run == 1 ? a_1 : run == 2 ? a_2 : a_3) + wave % HERE * PART;
        }
        const uint32_t steps = (ks + KS - 1) / KS;
        if (steps == 0) return;
        const FetchA fa(A, a0, k0, ks);
        const FetchB fb(B, b0, k0, ks);
        const ReadA ra(wave_a());
        const ReadB rb(wave_b());
        Fragments even, odd;
        auto fetch = [&](auto last, char *a, char *b, uint32_t s) {
            fa.template into<decltype(last)::value>(a, s, steps);
            fb.template into<decltype(last)::value>(b, s, steps);
        };
        constexpr std::true_type LAST{};
        constexpr std::false_type NOT_LAST{};
        fetch(LAST, a_0, b_0, 0);
        fetch(LAST, a_1, b_1, 1);
        fetch(LAST, a_2, b_2, 2);
        fetch(LAST, a_3, b_3, 3);
        landed<3 * EACH>();
        read(even, a_0, b_0, ra, rb);
        // Step s: its fragments are in registers; the next one's have landed, and no wavefront reads this one's place any more.
        auto turn = [&](auto last, Fragments &now, Fragments &next, char *a, char *b, const char *next_a, const char *next_b, uint32_t s) {
            landed<2 * EACH>();
            fetch(last, a, b, s + 4);
            multiply(now, next, next_a, next_b, ra, rb);
        };
        auto four = [&](auto last, uint32_t s) {
            turn(last, even, odd, a_0, b_0, a_1, b_1, s);
            turn(last, odd, even, a_1, b_1, a_2, b_2, s + 1);
            turn(last, even, odd, a_2, b_2, a_3, b_3, s + 2);
            turn(last, odd, even, a_3, b_3, a_0, b_0, s + 3);
        };
        uint32_t s = 0;
        for (; s + 8 < steps; s += 4) four(NOT_LAST, s);        // (nothing that is asked for there is the last)
        for (; s < steps; s += 4) four(LAST, s);
        settle();
        landed<0>();            // (places of steps that there are not are being filled with zeros)
    }

    // One step more, which lies in step_a and step_b, by itself.
    __device__ __forceinline__ void step_alone() {
        Fragments f;
        read(f, step_a, step_b, ReadA(wave_a()), ReadB(wave_b()));
        // (what vector instructions wrote is there two cycles later at the earliest)
#pragma unroll
        for (int i = 0; i < MA; ++i) asm volatile("" : "+v"(f.a[i]));
#pragma unroll
        for (int j = 0; j < MB; ++j) asm volatile("" : "+v"(f.b[j]));
#pragma unroll
        for (int i = 0; i < MA; ++i)
#pragma unroll
            for (int j = 0; j < MB; ++j) asm volatile("" : "+v"(acc[i][j]));
        asm volatile("s_nop 7" ::: "memory");
#pragma unroll
        for (int q = 0; q < (sizeof(T) == 4 ? 4 : 1); ++q)
#pragma unroll
            for (int i = 0; i < MA; ++i)
#pragma unroll
                for (int j = 0; j < MB; ++j) product<T>(f.a[i], f.b[j], q, acc[i][j]);
        settle();
    }

    static __device__ __forceinline__ void wave_sync() {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_sched_barrier(0);
    }
    // The tile as rows: value(i, j) gives four elements of acc[i][j], sink(a, b, words) takes 16 bytes of row b from element a on (both
    // in the tile).  A row's pieces lie in the order piece ^ row.
    template <typename Value, typename Sink> __device__ __forceinline__ void rows(Value value, Sink sink) {
        constexpr uint32_t PIECES = TA / WA * sizeof(T) / 16, AT_ONCE = 64 / PIECES, EACH = 16 / sizeof(T);
        char *const lds = part;
        const At at = place();
        const uint32_t first_a = at.a - 4 * (at.lane >> 4), first_b = at.b - (at.lane & 15u);
#pragma unroll
        for (int j = 0; j < MB; ++j) {
#pragma unroll
            for (int i = 0; i < MA; ++i) {
                const Vec<float, 4> f = value(i, j);
                Vec<T, 4> v;
#pragma unroll
                for (int q = 0; q < 4; ++q) v[q] = (T)f[q];
                const uint32_t r = at.lane & 15u, byte = (16 * i + 4 * (at.lane >> 4)) * sizeof(T), piece = (byte / 16) ^ (r % PIECES);
                *(Vec<T, 4> *)(lds + r * (PIECES * 16) + piece * 16 + byte % 16) = v;
            }
            wave_sync();
#pragma unroll
            for (uint32_t r0 = 0; r0 < 16; r0 += AT_ONCE) {
                const uint32_t r = r0 + at.lane / PIECES, piece = at.lane % PIECES;
                const Vec<uint32_t, 4> w = *(const Vec<uint32_t, 4> *)(lds + r * (PIECES * 16) + ((piece ^ (r % PIECES)) * 16));
                sink(first_a + piece * EACH, first_b + 16 * j + r, w);
            }
            wave_sync();
        }
    }
};

// Which tile a workgroup has.  Workgroups go to the eight dies in turn, each with its own L2: a die gets a run of the tiles, and in a
// run eight tiles of b are done for one of a before the next, so that what works at the same time shares both sides.
constexpr uint32_t GM_DIES = 8, GM_GROUP = 8;
struct Turn { uint32_t a, b; };
__device__ __forceinline__ uint32_t in_runs(uint32_t block, uint32_t blocks) {
    const uint32_t die = block % GM_DIES, each = blocks / GM_DIES, more = blocks % GM_DIES;
    return die * each + (die < more ? die : more) + block / GM_DIES;
}
__device__ __forceinline__ Turn turn_of(uint32_t i, uint32_t tiles_a, uint32_t tiles_b) {
    const uint32_t group = i / (tiles_a * GM_GROUP), rest = i - group * tiles_a * GM_GROUP;
    const uint32_t wide = tiles_b - group * GM_GROUP < GM_GROUP ? tiles_b - group * GM_GROUP : GM_GROUP;
    return Turn{rest / wide, group * GM_GROUP + rest % wide};
}

}  // namespace
