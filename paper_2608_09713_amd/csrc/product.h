// Products of tiles on the matrix cores: out[n][m] = sum over k of A[m][k] B[n][k],
// both operands in rows of k, 32-bit sums.
//
// A workgroup of WM x WN wavefronts takes a tile of BM rows of A and BN rows of
// B and walks k in steps of 128 bytes.  The step's rows go from memory into LDS
// without passing through registers, one step ahead of the products, in two
// buffers.  A row's eight chunks of 16 bytes stand in LDS at chunk ^ (row % 8),
// so that the lanes that read one chunk of eight rows touch all banks once; the
// order is made by the addresses that the lanes load from, as the loads
// themselves write LDS in lane order.  Rows past an operand's end are read from
// its last row and their products not stored.
//
// A is the operand whose rows become the contiguous dimension of the output: a
// lane holds four consecutive m of one n.
#pragma once

#include "rows.h"

namespace spsyrk {

typedef float F4 __attribute__((ext_vector_type(4)));

// a 16-byte chunk of k per lane: 16 rows of A by 16 rows of B, four chunks of k
template <typename T>
struct Chunk;
template <>
struct Chunk<__bf16> {
    typedef __bf16 V __attribute__((ext_vector_type(8)));
    __device__ static F4 mul(V a, V b, F4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Chunk<_Float16> {
    typedef _Float16 V __attribute__((ext_vector_type(8)));
    __device__ static F4 mul(V a, V b, F4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <>
struct Chunk<float> {
    typedef float V __attribute__((ext_vector_type(4)));
    // (k's order within a chunk is the same for both operands, which is all that counts)
    __device__ static F4 mul(V a, V b, F4 c) {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
        return c;
    }
};

constexpr int kStepBytes = 128;  // of k, per row and step
inline int step_elements(int dt) { return kStepBytes / dtype_bytes(dt); }

// rows of k, on 16-byte boundaries, k a whole number of steps (zeros past its end)
struct Operand {
    const void* p = nullptr;
    int64_t ld = 0;
    int64_t rows = 0;
};

// A tile's place among tm x tn: XCDs take the workgroups in turn, so each gets
// a contiguous part of an order in which bands of eight n walk over m; the
// workgroups of an XCD then share their rows in its L2.
struct TileAt {
    int m, n;
};
__device__ inline TileAt tile_at(int64_t id, int64_t tm, int64_t tn) {
    const int64_t total = tm * tn, per = total / kXcds, rest = total % kXcds;
    const int64_t x = id % kXcds, j = id / kXcds;
    const int64_t t = x * per + min(x, rest) + j;
    constexpr int64_t BAND = 8;
    const int64_t band = t / (BAND * tm), in = t % (BAND * tm);
    const int64_t wide = min(BAND, tn - band * BAND);
    return {int(in / wide), int(band * BAND + in % wide)};
}

template <typename T, int FM, int FN, int WM, int WN>
struct TileProduct {
    static constexpr int BM = FM * WM * 16, BN = FN * WN * 16, WAVES = WM * WN, THREADS = WAVES * kWave;
    static constexpr int BUFFER = (BM + BN) * kStepBytes;
    static constexpr int CHUNK = 16 / int(sizeof(T));
    static constexpr int LA = BM / 8 / WAVES, LB = BN / 8 / WAVES;  // loads of a wavefront per step
    static_assert(LA * 8 * WAVES == BM && LB * 8 * WAVES == BN, "whole loads");
    using V = typename Chunk<T>::V;

    __device__ static void load_rows(const char* const* from, unsigned char* lds, int count, int64_t at) {
        typedef const __attribute__((address_space(1))) void* Global;
        typedef __attribute__((address_space(3))) void* Local;
        for (int i = 0; i < count; ++i)
            __builtin_amdgcn_global_load_lds((Global)(from[i] + at), (Local)(lds + i * 1024), 16, 0, 0);
    }

    // acc[i][j]: rows 16 i + 4 (lane / 16) + r of the wavefront's part of A, row
    // 16 j + lane % 16 of its part of B
    __device__ static void run(const Operand& A, const Operand& B, int64_t m0, int64_t n0, int64_t steps, int64_t step0,
                               unsigned char* buf0, unsigned char* buf1, F4 (&acc)[FM][FN]) {
        const int lane = lane_id(), w = int(uniform(threadIdx.x / kWave));
        const char *fa[LA], *fb[LB];
        const int chunk = ((lane & 7) ^ (lane >> 3)) * 16;
#pragma unroll
        for (int i = 0; i < LA; ++i)
            fa[i] = static_cast<const char*>(A.p) +
                    min(m0 + (w * LA + i) * 8 + (lane >> 3), A.rows - 1) * A.ld * int64_t(sizeof(T)) + chunk;
#pragma unroll
        for (int i = 0; i < LB; ++i)
            fb[i] = static_cast<const char*>(B.p) +
                    min(n0 + (w * LB + i) * 8 + (lane >> 3), B.rows - 1) * B.ld * int64_t(sizeof(T)) + chunk;
        auto fetch = [&](int64_t step, unsigned char* buf) {
            const int64_t at = (step0 + step) * kStepBytes;
#pragma unroll
            for (int i = 0; i < LA; ++i) load_rows(fa + i, buf + (w * LA + i) * 1024, 1, at);
#pragma unroll
            for (int i = 0; i < LB; ++i) load_rows(fb + i, buf + BM * kStepBytes + (w * LB + i) * 1024, 1, at);
        };
        const int ra = ((w / WN) * FM * 16 + (lane & 15)) * kStepBytes;
        const int rb = BM * kStepBytes + ((w % WN) * FN * 16 + (lane & 15)) * kStepBytes;
        auto multiply = [&](const unsigned char* buf) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                __builtin_amdgcn_sched_barrier(0);
                const int c = ((s * 4 + (lane >> 4)) ^ (lane & 7)) * 16;
                V a[FM], b[FN];
#pragma unroll
                for (int j = 0; j < FN; ++j) b[j] = *reinterpret_cast<const V*>(buf + rb + j * 16 * kStepBytes + c);
#pragma unroll
                for (int i = 0; i < FM; ++i) a[i] = *reinterpret_cast<const V*>(buf + ra + i * 16 * kStepBytes + c);
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j) acc[i][j] = Chunk<T>::mul(a[i], b[j], acc[i][j]);
            }
        };
        // (each barrier waits for the loads into the buffer that is read next, and
        // for the readers of the one that is loaded next)
        if (steps > 0) fetch(0, buf0);
        int64_t k = 0;
        for (; k + 1 < steps; k += 2) {
            __syncthreads();
            fetch(k + 1, buf1);
            multiply(buf0);
            __syncthreads();
            if (k + 2 < steps) fetch(k + 2, buf0);
            multiply(buf1);
        }
        if (k < steps) {
            __syncthreads();
            multiply(buf0);
        }
    }
};

}  // namespace spsyrk
