// How rows of dense elements are spread over lanes and workgroups, and sums over
// a row's threads: shared by the layer norm and the norms around a block.
#pragma once

#include <algorithm>

#include "rows.h"

namespace spsyrk {
namespace {

constexpr int kRowBlock = 1024;  // threads per row, at most
constexpr int kCus = 256;        // compute units of the chip

// Sum over groups of L lanes, in every lane.
template <int L>
__device__ inline float group_total(float v) {
    if constexpr (L == kWave) return wave_total(v);
    auto add = [&](auto ctrl) {
        v += __int_as_float(
            __builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, false));
    };
    using std::integral_constant;
    add(integral_constant<int, 0xb1>());   // lane ^ 1
    add(integral_constant<int, 0x4e>());   // lane ^ 2
    if constexpr (L >= 8) add(integral_constant<int, 0x141>());   // mirrored within 8
    if constexpr (L >= 16) add(integral_constant<int, 0x140>());  // within 16
    if constexpr (L >= 32) v += __shfl_xor(v, 16, kWave);
    return v;
}

// Sum over a row's threads: L lanes, or (L 0) the workgroup's wavefronts with
// buf of kMostWaves words, not used again before the next sum's barrier.
constexpr int kMostWaves = kRowBlock / kWave;
template <int L>
__device__ inline float row_sum(float v, float* buf) {
    v = group_total<L ? L : kWave>(v);
    if constexpr (L == 0) {
        if (lane_id() == 0) buf[threadIdx.x / kWave] = v;
        lds_barrier();
        v = 0.f;
        for (int i = 0; i < int(blockDim.x) / kWave; ++i) v += buf[i];
    }
    return v;
}

// The places of a thread's packs, `threads` per row.  Only the last one can
// pass the row's end (row_shape).
template <int N, int NP>
__device__ inline void row_places(int l, int threads, int64_t d, Place (&at)[NP]) {
#pragma unroll
    for (int k = 0; k < NP; ++k) at[k] = place<N>((int64_t(k) * threads + l) * N, d);
}
// whether element i of pack k belongs to this thread alone
template <int NP>
__device__ inline bool own(const Place (&at)[NP], int k, int i) {
    return k < NP - 1 || i >= at[k].shift;
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline int64_t packs_of(int64_t d, int dt) {
    const int64_t n = 16 / dtype_bytes(dt);
    return d >= n ? ceil_div(d, n) : d;
}

// How a row is spread over threads: `lanes` of a wavefront, or (0) a workgroup
// of `threads`, and packs per thread.  Of the packs per thread that leave no
// pack but the last past the row's end (64 np (np - 1) packs or more) those
// that leave the fewest threads' packs empty are taken, and of these the most;
// with `few`, the fewest that a workgroup's threads can hold.  np 0: the row is
// too long for registers (more than `most` packs per thread).
struct RowShape {
    int lanes, threads, np;
};
inline RowShape row_shape(int64_t packs, int most, bool few) {
    if (packs <= 2 * kWave) {
        int lanes = 4;
        while (lanes < kWave && lanes < packs) lanes *= 2;
        return {lanes, lanes, packs <= kWave ? 1 : 2};
    }
    RowShape best{0, 0, 0};
    for (int np = 2; np <= most; ++np) {
        const int64_t threads = ceil_div(ceil_div(packs, np), kWave) * kWave;
        if (threads > kRowBlock || packs < 64 * np * (np - 1)) continue;
        if (!best.np || (!few && threads * np <= int64_t(best.threads) * best.np)) best = {0, int(threads), np};
    }
    return best;
}

inline unsigned row_grid(int64_t blocks) { return unsigned(std::min<int64_t>(blocks, int64_t(1) << 20)); }

// f(lanes, packs per thread) of a shape, as constants
template <int N, typename F>
inline void by_shape(const RowShape& s, F f) {
    using std::integral_constant;
    const integral_constant<int, 1> one;
    if (s.lanes == 4) return f(integral_constant<int, 4>(), one);
    if (s.lanes == 8) return f(integral_constant<int, 8>(), one);
    if constexpr (N > 1) {
        if (s.lanes == 16) return f(integral_constant<int, 16>(), one);
        if (s.lanes == 32) return f(integral_constant<int, 32>(), one);
        if (s.lanes && s.np == 1) return f(integral_constant<int, kWave>(), one);
        if (s.lanes) return f(integral_constant<int, kWave>(), integral_constant<int, 2>());
        if (s.np == 2) return f(integral_constant<int, 0>(), integral_constant<int, 2>());
        if (s.np == 3) return f(integral_constant<int, 0>(), integral_constant<int, 3>());
        return f(integral_constant<int, 0>(), integral_constant<int, 4>());
    }
}

}  // namespace
}  // namespace spsyrk
