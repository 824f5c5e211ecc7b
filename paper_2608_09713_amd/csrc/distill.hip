// Distillation of a teacher's top entries into logits over all columns.
//
// Row r has logits s over V columns and teacher entries (c_e, t_e):
//     z = (s - max s) / T,  L = log sum exp z,  q = exp(z - L),
//     p_e = softmax over the row's entries of t_e / T,
//     loss = T^2 sum_e p_e (log p_e - (z_{c_e} - L)),
//     dS_j = weight T (q_j - sum of p_e over the entries with c_e = j).
// Entries whose column lies outside [0, V) are padding.  A row without
// entries, with teacher values of -inf only, or with logits of -inf only has
// no distribution to match: its loss and its gradient are 0.
//
// Bound by the bytes of the logits.  Logits are read 16 bytes a lane with a
// running maximum and sum of exponentials per thread; an element past the row
// counts as -inf.  Exponentials are powers of two of (s - max) log2(e) / T,
// all sums 32-bit floats.
#include <algorithm>

#include "internal.h"
#include "rows.h"

namespace spsyrk {
namespace {

constexpr int kRowBlock = 1024;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct RowStat {
    float m, l2;   // maximum of the logits, log2 of their sum of exponentials
    float tm, tl2; // the same of the teacher's entries
    float scale;   // weight T, 0 for a row without a gradient
};

// running maximum and sum of 2^((s - m) c)
struct MaxSum {
    float m, s;
};
constexpr MaxSum kNothing{-INFINITY, 0.f};

__device__ inline float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// (an operand of maximum -inf holds nothing; NaN is carried by its sum)
__device__ inline MaxSum merge(MaxSum a, MaxSum b, float c) {
    MaxSum r;
    r.m = fmaxf(a.m, b.m);
    const float sa = a.m == -INFINITY ? a.s : a.s * exp2_of((a.m - r.m) * c);
    const float sb = b.m == -INFINITY ? b.s : b.s * exp2_of((b.m - r.m) * c);
    r.s = sa + sb;
    return r;
}

template <int NT>
__device__ inline MaxSum block_merge(MaxSum v, float c, MaxSum* buf) {
#pragma unroll
    for (int d = kWave / 2; d > 0; d >>= 1) {
        MaxSum o;
        o.m = __shfl_xor(v.m, d, kWave);
        o.s = __shfl_xor(v.s, d, kWave);
        // (the lower lane's operand first: both lanes get the same bits)
        v = lane_id() & d ? merge(o, v, c) : merge(v, o, c);
    }
    if (lane_id() == 0) buf[threadIdx.x / kWave] = v;
    __syncthreads();
    v = buf[0];
#pragma unroll
    for (int i = 1; i < NT / kWave; ++i) v = merge(v, buf[i], c);
    __syncthreads();
    return v;
}

template <int NT>
__device__ inline float block_sum(float v, float* buf) {
    v = wave_reduce_sum(v);
    if (lane_id() == 0) buf[threadIdx.x / kWave] = v;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NT / kWave; ++i) s += buf[i];
    __syncthreads();
    return s;
}

template <typename T>
__device__ inline void add_pack(MaxSum& a, PackV<T> v, float c) {
    constexpr int N = Pack<T>::N;
    float x[N], m = a.m;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = float(v[i]);
        m = fmaxf(m, x[i]);
    }
    // (all -inf so far: 0 stands in for the maximum, so that -inf - m stays -inf)
    const float base = m == -INFINITY ? 0.f : m;
    float s = a.m == -INFINITY ? a.s : a.s * exp2_of((a.m - base) * c);
#pragma unroll
    for (int i = 0; i < N; ++i) s += exp2_of((x[i] - base) * c);
    a.m = m;
    a.s = s;
}

// entries [a, b) of row r of the teacher, by their positions in idx and val
struct RowEntries {
    int64_t n, i0, v0;
};
__device__ inline RowEntries row_entries(const Entries& t, int64_t r) {
    if (!t.rp) return {t.per_row, r * t.istride, r * t.vstride};
    const int64_t a = min(max(t.rp[r], int64_t(0)), t.nnz), b = min(max(t.rp[r + 1], a), t.nnz);
    return {b - a, a, a};
}

// Loss of a row and what its gradient needs.
template <typename T, int NT>
__global__ __launch_bounds__(NT) void distill_rows(const T* __restrict__ S, int64_t lds, int64_t m, int64_t V,
                                                   Entries t, float temp, const float* __restrict__ weight,
                                                   float* __restrict__ loss, RowStat* __restrict__ stat) {
    constexpr int N = Pack<T>::N;
    __shared__ MaxSum ms[NT / kWave];
    __shared__ float fs[NT / kWave];
    const float c = kLog2e / temp;
    for (int64_t r = blockIdx.x; r < m; r += gridDim.x) {
        const T* row = S + r * lds;
        MaxSum a = kNothing;
        for (int64_t j = int64_t(threadIdx.x) * N; j < V; j += int64_t(NT) * N)
            add_pack<T>(a, load_pack_nt(row + j, V - j, -INFINITY), c);
        a = block_merge<NT>(a, c, ms);
        const RowEntries e = row_entries(t, r);
        MaxSum b = kNothing;
        for (int64_t k = threadIdx.x; k < e.n; k += NT) {
            const int64_t col = load_column(t.idx, t.ib, e.i0 + k);
            if (col < 0 || col >= V) continue;
            MaxSum one;
            one.m = load_value(t.val, t.vt, e.v0 + k);
            one.s = one.m == -INFINITY ? 0.f : 1.f;
            if (one.m != one.m) one.s = one.m;  // (NaN, which a maximum drops)
            b = merge(b, one, c);
        }
        b = block_merge<NT>(b, c, ms);
        // NaN sums are kept: only rows of nothing but -inf have none
        const bool none = (a.m == -INFINITY && a.s == 0.f) || (b.m == -INFINITY && b.s == 0.f);
        const float l2 = log2f(a.s), tl2 = log2f(b.s);
        float x = 0.f;
        for (int64_t k = threadIdx.x; k < e.n && !none; k += NT) {
            const int64_t col = load_column(t.idx, t.ib, e.i0 + k);
            if (col < 0 || col >= V) continue;
            const float lp = (load_value(t.val, t.vt, e.v0 + k) - b.m) * c - tl2;
            const float p = exp2_of(lp);
            const float lq = (float(row[col]) - a.m) * c - l2;
            if (!(p == 0.f)) x += p * (lp - lq);
        }
        x = block_sum<NT>(x, fs);
        if (threadIdx.x == 0) {
            loss[r] = none ? 0.f : x * kLn2 * temp * temp;
            if (stat) {
                const float w = weight ? weight[r] : 1.f;
                stat[r] = {a.m, l2, b.m, tl2, none ? 0.f : w * temp};
            }
        }
    }
}

// Gradient of a chunk of a row: the teacher's part of the chunk is gathered in
// LDS (entries of one column add up), the logits are read again.
constexpr int kGradPacks = 4;
template <typename T>
__global__ __launch_bounds__(kBlock) void distill_grad_chunks(const T* __restrict__ S, int64_t lds, int64_t m,
                                                              int64_t V, Entries t, float temp,
                                                              const RowStat* __restrict__ stat, T* __restrict__ dS,
                                                              int64_t ldd, int64_t chunks) {
    constexpr int N = Pack<T>::N, COLS = kBlock * kGradPacks * N;
    __shared__ float p[COLS];
    const float c = kLog2e / temp;
    for (int64_t u = blockIdx.x; u < m * chunks; u += gridDim.x) {
        const int64_t r = u / chunks, c0 = u % chunks * COLS;
        const RowStat st = stat[r];
        const bool zero = st.scale == 0.f;  // (whatever the logits hold)
        PackV<T> v[kGradPacks];
        if (!zero) {
#pragma unroll
            for (int k = 0; k < kGradPacks; ++k) {
                const int64_t j = c0 + (int64_t(k) * kBlock + threadIdx.x) * N;
                v[k] = load_pack_nt(S + r * lds + j, V - j);
            }
            for (int x = threadIdx.x; x < COLS; x += kBlock) p[x] = 0.f;
            __syncthreads();
            const RowEntries e = row_entries(t, r);
            for (int64_t k = threadIdx.x; k < e.n; k += kBlock) {
                const int64_t col = load_column(t.idx, t.ib, e.i0 + k);
                if (col < 0 || col >= V || col < c0 || col >= c0 + COLS) continue;
                atomicAdd(&p[col - c0], exp2_of((load_value(t.val, t.vt, e.v0 + k) - st.tm) * c - st.tl2));
            }
            __syncthreads();
        }
#pragma unroll
        for (int k = 0; k < kGradPacks; ++k) {
            const int x = (k * kBlock + int(threadIdx.x)) * N;
            if (c0 + x >= V) break;
            PackV<T> o;
#pragma unroll
            for (int i = 0; i < N; ++i)
                o[i] = T(zero ? 0.f : (exp2_of((float(v[k][i]) - st.m) * c - st.l2) - p[x + i]) * st.scale);
            store_pack_nt(dS + r * ldd + c0 + x, o, V - c0 - x);
        }
        __syncthreads();
    }
}

}  // namespace

size_t distill_tmp_bytes(int64_t m, int64_t v, int dt, bool grad) {
    (void)v;
    (void)dt;
    return grad ? size_t(m) * sizeof(RowStat) : 0;
}

void distill(const DenseRows& S, const Entries& t, float temperature, const float* weight, float* loss,
             const DenseRows& dS, void* tmp, hipStream_t s) {
    by_dtype(S.dt, [&](auto e) {
        using T = decltype(e);
        const int64_t m = S.m, V = S.n;
        const T* x = static_cast<const T*>(S.p);
        RowStat* stat = dS.p ? static_cast<RowStat*>(tmp) : nullptr;
        const unsigned rows = unsigned(std::min<int64_t>(m, int64_t(1) << 20));
        if (V <= int64_t(kBlock) * Pack<T>::N * 4)
            distill_rows<T, kBlock><<<rows, kBlock, 0, s>>>(x, S.ld, m, V, t, temperature, weight, loss, stat);
        else
            distill_rows<T, kRowBlock><<<rows, kRowBlock, 0, s>>>(x, S.ld, m, V, t, temperature, weight, loss, stat);
        if (!stat) return;
        constexpr int64_t COLS = int64_t(kBlock) * kGradPacks * Pack<T>::N;
        const int64_t chunks = (V + COLS - 1) / COLS;
        distill_grad_chunks<T><<<unsigned(std::min<int64_t>(m * chunks, int64_t(1) << 20)), kBlock, 0, s>>>(
            x, S.ld, m, V, t, temperature, stat, static_cast<T*>(dS.p), dS.ld, chunks);
    });
}

}  // namespace spsyrk
