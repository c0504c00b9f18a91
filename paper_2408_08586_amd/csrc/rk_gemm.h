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
    __device__ __forceinline__ void run(const Side &A, const Side &B, uint64_t a0, uint64_t b0, uint64_t k0, uint32_t bytes_k) {
        __shared__ __attribute__((aligned(128))) char a_even[TA * GM_ROW], b_even[TB * GM_ROW];
        __shared__ __attribute__((aligned(128))) char a_odd[TA * GM_ROW], b_odd[TB * GM_ROW];
#pragma unroll
        for (int i = 0; i < MA; ++i)
#pragma unroll
            for (int j = 0; j < MB; ++j) acc[i][j] = 0.f;
        const uint32_t steps = (bytes_k + GM_ROW - 1) / GM_ROW;
        if (steps == 0) return;
        const Side a = {A.data + k0, A.stride, A.rows}, b = {B.data + k0, B.stride, B.rows};
        const Fetch<TA> fa(a, a0, bytes_k);
        const Fetch<TB> fb(b, b0, bytes_k);
        fa.into(a_even, 0, steps == 1);
        fb.into(b_even, 0, steps == 1);
        __syncthreads();
        for (uint32_t s = 0; s < steps; s += 2) {
            if (s + 1 < steps) {
                fa.into(a_odd, (s + 1) * GM_ROW, s + 2 == steps);
                fb.into(b_odd, (s + 1) * GM_ROW, s + 2 == steps);
            }
            step(a_even, b_even);
            __syncthreads();
            if (s + 1 == steps) break;
            if (s + 2 < steps) {
                fa.into(a_even, (s + 2) * GM_ROW, s + 3 == steps);
                fb.into(b_even, (s + 2) * GM_ROW, s + 3 == steps);
            }
            step(a_odd, b_odd);
            __syncthreads();
        }
    }
};

}  // namespace
