// Matrix products of the operators: out[b][a] = sum over k of A[a][k] B[b][k], both with k along their rows, held in float32.
//
// A workgroup of eight wavefronts makes a tile of TA x TB, 128 bytes of k at a time: both tiles' rows go from memory straight into LDS
// while the ones before them are multiplied.  A row's eight 16-byte pieces lie in the order piece ^ (row % 8), so that the lanes of a
// fragment, which read the same piece of sixteen rows, do not meet in the banks; memory gives them in that order, as LDS is written in the order of the
// lanes.  32-bit elements take the same pieces: four k a lane, one for each of four products, the same for both sides.
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
__device__ __forceinline__ void into_lds(__amdgpu_buffer_rsrc_t buf, char *lds, uint32_t at, uint32_t k) {
#ifdef __HIP_DEVICE_COMPILE__
    __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (__attribute__((address_space(3))) void *)lds, 16, at, k, 0, 0);
#endif
}

// One side of a product: rows whose first bytes and stride are multiples of 16, and how many bytes of each count.
struct Side {
    const char *data;
    uint64_t stride;            // bytes
    uint64_t rows;
};
// What a wavefront asks for of a tile of R rows: R / 64 instructions of eight rows each.
template <int R> struct Fetch {
    static constexpr int N = R >= 64 ? R / 64 : 1;
    __amdgpu_buffer_rsrc_t buf;
    uint32_t at[N], tail[N];    // of a lane, also where the last bytes of k end within a row of LDS
    __device__ __forceinline__ Fetch(const Side &s, uint64_t row0, uint32_t bytes_k) {
        buf = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(s.data) + row0 * s.stride, 0, (int)GM_NOWHERE, 0x00027000);
        const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63u;
        const uint64_t left = s.rows - row0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            uint32_t r = (wave * N + i) * 8 + (lane >> 3);
            const uint32_t piece = ((lane & 7u) ^ (r & 7u)) * 16u;
            r = r < left ? r : (uint32_t)(left - 1);        // (rows behind the last repeat it: their results go nowhere)
            at[i] = r * (uint32_t)s.stride + piece;
            tail[i] = piece < bytes_k % GM_ROW || bytes_k % GM_ROW == 0 ? at[i] : GM_NOWHERE;
        }
    }
    __device__ __forceinline__ void into(char *lds, uint32_t k, bool last) const {
        const uint32_t wave = threadIdx.x >> 6;
        if (R < 64 && wave * 8 >= R) return;
#pragma unroll
        for (int i = 0; i < N; ++i)
            into_lds(buf, lds + (wave * N + i) * 1024, last ? tail[i] : at[i], k);
    }
};

// The tile at (a0, b0) over bytes_k of k from k0 on; WA x WB wavefronts share it.  acc[i][j]: lane l holds the elements
// a = a0 + wa TA/WA + 16 i + 4 (l / 16) + 0..3,  b = b0 + wb TB/WB + 16 j + l % 16.
template <typename T, int TA, int TB, int WA> struct Tile {
    static constexpr int WB = 8 / WA, MA = TA / WA / 16, MB = TB / WB / 16;
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

    __device__ __forceinline__ void step(const char *a, const char *b) {
        const uint32_t lane = threadIdx.x & 63u, r = lane & 15u;
        const char *const pa = a + (wave_a() + r) * GM_ROW, *const pb = b + (wave_b() + r) * GM_ROW;
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h) {
            const uint32_t piece = ((h * 4 + (lane >> 4)) ^ (r & 7u)) * 16u;
            Vec<uint32_t, 4> fa[MA], fb[MB];
#pragma unroll
            for (int j = 0; j < MB; ++j) fb[j] = *(const Vec<uint32_t, 4> *)(pb + j * 16 * GM_ROW + piece);
#pragma unroll
            for (int i = 0; i < MA; ++i) fa[i] = *(const Vec<uint32_t, 4> *)(pa + i * 16 * GM_ROW + piece);
#pragma unroll
            for (int i = 0; i < MA; ++i)
#pragma unroll
                for (int j = 0; j < MB; ++j) acc[i][j] = products<T>(fa[i], fb[j], acc[i][j]);
        }
    }
    char *room[2];              // two runs of TA * GM_ROW bytes of LDS, free behind the loop

    __device__ __forceinline__ void run(const Side &A, const Side &B, uint64_t a0, uint64_t b0, uint64_t k0, uint32_t bytes_k) {
        __shared__ __attribute__((aligned(128))) char a_even[TA * GM_ROW], b_even[TB * GM_ROW];
        __shared__ __attribute__((aligned(128))) char a_odd[TA * GM_ROW], b_odd[TB * GM_ROW];
#pragma unroll
        for (int i = 0; i < MA; ++i)
#pragma unroll
            for (int j = 0; j < MB; ++j) acc[i][j] = 0.f;
        room[0] = a_even; room[1] = a_odd;
        const uint32_t steps = (bytes_k + GM_ROW - 1) / GM_ROW;
        if (steps == 0) return;
        const Side a = {A.data + k0, A.stride, A.rows}, b = {B.data + k0, B.stride, B.rows};
        const Fetch<TA> fa(a, a0, bytes_k);
        const Fetch<TB> fb(b, b0, bytes_k);
        // an odd step goes first, and there is one way out of the loop: the sums stay in their registers
        uint32_t s = 0;
        if (steps & 1u) {
            fa.into(a_odd, 0, steps == 1);
            fb.into(b_odd, 0, steps == 1);
            __syncthreads();
            if (steps > 1) {
                fa.into(a_even, GM_ROW, false);
                fb.into(b_even, GM_ROW, false);
            }
            step(a_odd, b_odd);
            s = 1;
        } else {
            fa.into(a_even, 0, false);
            fb.into(b_even, 0, false);
        }
        __syncthreads();
        for (; s < steps; s += 2) {
            fa.into(a_odd, (s + 1) * GM_ROW, s + 2 == steps);
            fb.into(b_odd, (s + 1) * GM_ROW, s + 2 == steps);
            step(a_even, b_even);
            __syncthreads();
            if (s + 2 < steps) {
                fa.into(a_even, (s + 2) * GM_ROW, false);
                fb.into(b_even, (s + 2) * GM_ROW, false);
            }
            step(a_odd, b_odd);
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
    // ... and turned around: sink(a, b, words) takes 16 bytes of what belongs to element a, from row b on
    template <typename Value, typename Sink> __device__ __forceinline__ void columns(Value value, Sink sink) {
        constexpr uint32_t ROW = 16 * sizeof(T), PIECES = ROW / 16, EACH = 16 / sizeof(T), TALL = TA / WA;
        char *const lds = part();
        const At at = place();
        const uint32_t first_a = at.a - 4 * (at.lane >> 4), first_b = at.b - (at.lane & 15u);
#pragma unroll
        for (int j = 0; j < MB; ++j) {
#pragma unroll
            for (int i = 0; i < MA; ++i) {
                const Vec<float, 4> f = value(i, j);
#pragma unroll
                for (int q = 0; q < 4; ++q) *(T *)(lds + (16 * i + 4 * (at.lane >> 4) + q) * ROW + (at.lane & 15u) * sizeof(T)) = (T)f[q];
            }
            wave_sync();
#pragma unroll
            for (uint32_t x = 0; x < TALL * PIECES; x += 64) {
                const uint32_t r = (x + at.lane) / PIECES, piece = at.lane % PIECES;
                if (TALL * PIECES >= 64 || r < TALL) sink(first_a + r, first_b + 16 * j + piece * EACH, *(const Vec<uint32_t, 4> *)(lds + r * ROW + piece * 16));
            }
            wave_sync();
        }
    }
};

}  // namespace
