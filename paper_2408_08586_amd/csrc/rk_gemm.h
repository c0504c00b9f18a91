// Matrix products of the operators: out[b][a] = sum over k of A(a, k) B(b, k), held in float32.
//
// A workgroup of eight wavefronts makes a tile of TA x TB, 128 bytes of k at a time: both tiles go from memory straight into LDS
// while the ones before them are multiplied.  A side lies with k along its rows (ALONG) or with k from row to row (ACROSS), and so it
// comes into LDS; nothing is turned around beforehand:
//   ALONG   128 bytes a row.  A lane's part of a fragment is a 16-byte piece of its row; pieces lie in the order piece ^ (row % 8), so that the
//           sixteen rows of a fragment do not meet in the banks.
//   ACROSS  a row of TA (TB) elements for every k.  Of narrow elements, sixteen lanes read four k of sixteen elements and get them
//           turned around by the LDS unit; of 32-bit ones, a lane reads its element of each k.  Pieces lie in the order piece ^ something that
//           the k of the lanes that read together do not share.
// Memory gives pieces in that order, as LDS is written in the order of the lanes.  The matrix units take sixteen elements of 32 narrow k at once, or of four
// 32-bit ones: there, each of four products takes one k of every lane's four, the same of both sides.
#pragma once
#include "rk_vec.h"

namespace {

constexpr uint32_t GM_THREADS = 512, GM_ROW = 128;          // threads; bytes of k in LDS
constexpr uint32_t GM_NOWHERE = 0x80000000u;                // a lane's place behind every buffer: zeros

// (builtins of this GPU alone: the host's pass over the source does not know them)
template <typename T> __device__ __forceinline__ Vec<float, 4> products(const Vec<uint32_t, 4> &a, const Vec<uint32_t, 4> &b, Vec<float, 4> c) {
#ifdef __HIP_DEVICE_COMPILE__
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0, 0, 0);
    } else if constexpr (__is_same(T, __bf16)) {
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Vec<__bf16, 8>, a), __builtin_bit_cast(Vec<__bf16, 8>, b), c, 0, 0, 0);
    } else {
        c = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(Vec<_Float16, 8>, a), __builtin_bit_cast(Vec<_Float16, 8>, b), c, 0, 0, 0);
    }
#endif
    return c;
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

enum { ALONG = 0, ACROSS = 1 };
// One side of a product, its first byte and stride multiples of 16.
struct Side {
    const char *data;
    uint64_t stride;            // bytes from row to row
    uint64_t count;             // ALONG: rows; ACROSS: bytes of a row
};
// order of the pieces of a row of LDS for one k
template <typename T> __device__ __forceinline__ uint32_t order_of(uint32_t k) {
    if constexpr (sizeof(T) == 4) return (k >> 2 & 3u) * 4u;
    else return ((k & 3u) | (k >> 3 & 3u) << 2) * 2u;
}
// What a wavefront asks for of a tile of R elements: R / 64 instructions of 1,024 bytes.
template <typename T, int R, int WAY> struct Fetch {
    static constexpr int N = R >= 64 ? R / 64 : 1;
    static constexpr uint32_t KS = GM_ROW / sizeof(T), PIECES = R * sizeof(T) / 16;     // k of a step; ACROSS: pieces of a row of LDS
    const char *base;
    uint64_t hop;               // bytes from step to step
    uint32_t at[N], tail[N];    // of a lane, and in the last step
    __device__ __forceinline__ Fetch(const Side &s, uint64_t first, uint64_t k0, uint32_t ks) {
        const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63u, left = ks % KS ? ks % KS : KS;
        if constexpr (WAY == ALONG) {
            base = s.data + first * s.stride + k0 * sizeof(T);
            hop = GM_ROW;
            const uint64_t rows = s.count - first;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                uint32_t r = (wave * N + i) * 8 + (lane >> 3);
                const uint32_t piece = (lane & 7u) ^ (r & 7u);
                r = r < rows ? r : (uint32_t)(rows - 1);    // (rows behind the last repeat it: their results go nowhere)
                at[i] = r * (uint32_t)s.stride + piece * 16;
                tail[i] = piece * (16 / sizeof(T)) < left ? at[i] : GM_NOWHERE;
            }
        } else {
            base = s.data + k0 * s.stride + first * sizeof(T);
            hop = KS * s.stride;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t x = (wave * N + i) * 64 + lane, k = x / PIECES, piece = (x % PIECES) ^ (order_of<T>(k) % PIECES);
                at[i] = first * sizeof(T) + piece * 16 < s.count ? k * (uint32_t)s.stride + piece * 16 : GM_NOWHERE;
                tail[i] = k < left ? at[i] : GM_NOWHERE;
            }
        }
    }
    // step s into LDS; `last`: the rest of k alone, zeros behind it
    __device__ __forceinline__ void into(char *lds, uint32_t s, bool last) const {
        const uint32_t wave = threadIdx.x >> 6;
        if (R < 64 && wave * 8 >= R) return;
        const __amdgpu_buffer_rsrc_t buf = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base) + s * hop, 0, (int)GM_NOWHERE, 0x00027000);
#pragma unroll
        for (int i = 0; i < N; ++i) into_lds(buf, lds + (wave * N + i) * 1024, last ? tail[i] : at[i]);
    }
};
// A wavefront's fragments of M times sixteen elements, from element `first` of the tile on
template <typename T, int R, int WAY, int M> struct Reader {
    static constexpr uint32_t PITCH = R * sizeof(T), PIECES = PITCH / 16;
    uint32_t at[WAY == ALONG ? 2 : M];
    __device__ __forceinline__ Reader(uint32_t first) {
        const uint32_t lane = threadIdx.x & 63u, j = lane & 15u, g = lane >> 4;
        if constexpr (WAY == ALONG) {
#pragma unroll
            for (uint32_t h = 0; h < 2; ++h) at[h] = (first + j) * GM_ROW + ((h * 4 + g) ^ (j & 7u)) * 16;
        } else {
#pragma unroll
            for (int i = 0; i < M; ++i) {
                if constexpr (sizeof(T) == 4) {
                    const uint32_t k = 4 * g, piece = (first + 16 * i) / 4 + (j >> 2);
                    at[i] = k * PITCH + (piece ^ (order_of<T>(k) % PIECES)) * 16 + (j & 3u) * 4;
                } else {
                    const uint32_t k = 8 * g + (j >> 2), piece = (first + 16 * i) / 8 + (j >> 1 & 1u);
                    at[i] = k * PITCH + (piece ^ (order_of<T>(k) % PIECES)) * 16 + (j & 1u) * 8;
                }
            }
        }
    }
    // half h of the step's k
    __device__ __forceinline__ Vec<uint32_t, 4> read(const char *lds, int i, uint32_t h) const {
        if constexpr (WAY == ALONG) {
            return *(const Vec<uint32_t, 4> *)(lds + at[h] + i * 16 * GM_ROW);
        } else if constexpr (sizeof(T) == 4) {
            Vec<uint32_t, 4> w;
#pragma unroll
            for (int q = 0; q < 4; ++q) w[q] = *(const uint32_t *)(lds + at[i] + (16 * h + q) * PITCH);
            return w;
        } else {
            const Vec<uint32_t, 2> lo = turned(lds + at[i] + 32 * h * PITCH), hi = turned(lds + at[i] + (32 * h + 4) * PITCH);
            return Vec<uint32_t, 4>{lo[0], lo[1], hi[0], hi[1]};
        }
    }
};

// The tile at (a0, b0) over ks of k from k0 on; WA x WB wavefronts share it.  acc[i][j]: lane l holds the elements
// a = a0 + wa TA/WA + 16 i + 4 (l / 16) + 0..3,  b = b0 + wb TB/WB + 16 j + l % 16.
template <typename T, int TA, int TB, int WA, int WAY_A, int WAY_B> struct Tile {
    static constexpr int WB = 8 / WA, MA = TA / WA / 16, MB = TB / WB / 16;
    static constexpr uint32_t KS = GM_ROW / sizeof(T);
    typedef Reader<T, TA, WAY_A, MA> ReadA;
    typedef Reader<T, TB, WAY_B, MB> ReadB;
    Vec<float, 4> acc[MA][MB];
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

    __device__ __forceinline__ void step(const char *a, const char *b, const ReadA &ra, const ReadB &rb) {
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h) {
            Vec<uint32_t, 4> fa[MA], fb[MB];
#pragma unroll
            for (int j = 0; j < MB; ++j) fb[j] = rb.read(b, j, h);
#pragma unroll
            for (int i = 0; i < MA; ++i) fa[i] = ra.read(a, i, h);
#pragma unroll
            for (int i = 0; i < MA; ++i)
#pragma unroll
                for (int j = 0; j < MB; ++j) acc[i][j] = products<T>(fa[i], fb[j], acc[i][j]);
        }
    }
    char *room[2];              // two runs of TA * GM_ROW bytes of LDS, free behind the loop

    __device__ __forceinline__ void run(const Side &A, const Side &B, uint64_t a0, uint64_t b0, uint64_t k0, uint32_t ks) {
        __shared__ __attribute__((aligned(128))) char a_even[TA * GM_ROW], b_even[TB * GM_ROW];
        __shared__ __attribute__((aligned(128))) char a_odd[TA * GM_ROW], b_odd[TB * GM_ROW];
#pragma unroll
        for (int i = 0; i < MA; ++i)
#pragma unroll
            for (int j = 0; j < MB; ++j) acc[i][j] = 0.f;
        room[0] = a_even; room[1] = a_odd;
        const uint32_t steps = (ks + KS - 1) / KS;
        if (steps == 0) return;
        const Fetch<T, TA, WAY_A> fa(A, a0, k0, ks);
        const Fetch<T, TB, WAY_B> fb(B, b0, k0, ks);
        const ReadA ra(wave_a());
        const ReadB rb(wave_b());
        // an odd step goes first, and there is one way out of the loop: the sums stay in their registers
        uint32_t s = 0;
        if (steps & 1u) {
            fa.into(a_odd, 0, steps == 1);
            fb.into(b_odd, 0, steps == 1);
            __syncthreads();
            if (steps > 1) {
                fa.into(a_even, 1, false);
                fb.into(b_even, 1, false);
            }
            step(a_odd, b_odd, ra, rb);
            s = 1;
        } else {
            fa.into(a_even, 0, false);
            fb.into(b_even, 0, false);
        }
        __syncthreads();
        for (; s < steps; s += 2) {
            fa.into(a_odd, s + 1, s + 2 == steps);
            fb.into(b_odd, s + 1, s + 2 == steps);
            step(a_even, b_even, ra, rb);
            __syncthreads();
            if (s + 2 < steps) {
                fa.into(a_even, s + 2, false);
                fb.into(b_even, s + 2, false);
            }
            step(a_odd, b_odd, ra, rb);
            __syncthreads();
        }
    }

    // A wavefront's part of LDS behind the loop: 16 rows of TA / WA elements, or TA / WA rows of 16
    static constexpr int PART = TA / WA * 16 * (int)sizeof(T);
    __device__ __forceinline__ char *part() const {
        constexpr uint32_t HERE = TA * GM_ROW / PART;       // wavefronts whose parts the first run holds
        const uint32_t wave = threadIdx.x >> 6;
        return HERE >= 8 || wave < HERE ? room[0] + wave * PART : room[1] + (wave - HERE) * PART;
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
        char *const lds = part();
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

}  // namespace
