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
// running maximum and sum of exponentials per thread.  Exponentials are powers
// of two of (s - max) log2(e) / T, the difference first, so that large logits
// lose nothing; all sums are 32-bit floats.
//
// The gradient of a row of up to 256 KB is computed with the whole row in one
// workgroup's registers, so that it is read once; the workgroup goes on to
// further rows, and a pack's registers take the next row's pack as soon as its
// gradient is stored, which keeps loads in flight all the time.  Longer rows
// are read twice, first for their sums, then by chunks.
#include <algorithm>

#include "internal.h"
#include "rows.h"

namespace spsyrk {
namespace {

constexpr int kRowBlock = 1024;
constexpr int kCus = 256;  // compute units of the chip
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

// a.s relative to the maximum m >= a.m (of maximum -inf there is nothing to
// scale, but NaN, which a maximum passes over, is carried by the sum)
__device__ inline float scaled(MaxSum a, float m, float c) {
    return a.m == -INFINITY ? a.s : a.s * exp2_of((a.m - m) * c);
}
__device__ inline MaxSum wave_merge(MaxSum a, float c) {
    const float m = wave_max(a.m);
    return {m, wave_total(scaled(a, m, c))};
}
// of the first n <= kWave elements of buf, by every wavefront for itself
__device__ inline MaxSum merge_of(const MaxSum* buf, int n, float c) {
    return wave_merge(lane_id() < n ? buf[lane_id()] : kNothing, c);
}

// the pack's elements from `skip` on
template <typename T, int N>
__device__ inline void add_pack(MaxSum& a, Vec<T, N> v, int skip, float c) {
    float x[N], m = a.m;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = float(v[i]);
    if (skip > 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = i < skip ? -INFINITY : x[i];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, x[i]);
    // (all -inf so far: 0 stands in for the maximum, so that -inf - m stays -inf)
    const float base = m == -INFINITY ? 0.f : m;
    float s = a.s;
    if (m > a.m) s = scaled(a, base, c);
#pragma unroll
    for (int i = 0; i < N; ++i) s += exp2_of((x[i] - base) * c);
    a.m = m;
    a.s = s;
}

__device__ inline void add_value(MaxSum& a, float x, float c) {
    const float m = fmaxf(a.m, x);
    a.s = scaled(a, m, c) + (x == -INFINITY ? 0.f : exp2_of((x - m) * c));
    a.m = m;
}

// (NaN sums are something: only rows of nothing but -inf are empty)
__device__ inline bool is_empty(MaxSum a) { return a.m == -INFINITY && a.s == 0.f; }

// positions of the row's n entries in idx and val
struct RowEntries {
    int64_t n, i0, v0;
};
__device__ inline RowEntries row_entries(const Entries& t, int64_t r) {
    if (!t.rp) return {t.per_row, r * t.istride, r * t.vstride};
    const int64_t a = min(max(t.rp[r], int64_t(0)), t.nnz), b = min(max(t.rp[r + 1], a), t.nnz);
    return {b - a, a, a};
}

// One term of the loss, in units of log 2.
__device__ inline float loss_term(float p, float lp, float lq) { return p == 0.f ? 0.f : p * (lp - lq); }

// The block's sums over the teacher's entries: all of them, strided.
template <int NT>
__device__ inline MaxSum teacher_sums(const Entries& t, const RowEntries& e, int64_t V, float c) {
    MaxSum b = kNothing;
    for (int64_t k = threadIdx.x; k < e.n; k += NT) {
        const int64_t col = load_column(t.idx, t.ib, e.i0 + k);
        if (col >= 0 && col < V) add_value(b, load_value(t.val, t.vt, e.v0 + k), c);
    }
    return b;
}
template <typename T, int NT>
__device__ inline float teacher_loss(const Entries& t, const RowEntries& e, const T* row, int64_t V, float c,
                                     const RowStat& st) {
    float x = 0.f;
    for (int64_t k = threadIdx.x; k < e.n; k += NT) {
        const int64_t col = load_column(t.idx, t.ib, e.i0 + k);
        if (col < 0 || col >= V) continue;
        const float lp = (load_value(t.val, t.vt, e.v0 + k) - st.tm) * c - st.tl2;
        x += loss_term(exp2_of(lp), lp, (float(row[col]) - st.m) * c - st.l2);
    }
    return x;
}

// Loss of a row and what its gradient needs.
constexpr int kAhead = 4;  // packs per thread in flight
template <typename T, int N, int NT>
__global__ __launch_bounds__(NT) void distill_rows(const T* __restrict__ S, int64_t lds, int64_t m, int64_t V,
                                                   Entries t, float temp, const float* __restrict__ weight,
                                                   float* __restrict__ loss, RowStat* __restrict__ stat) {
    constexpr int W = NT / kWave;
    constexpr int64_t STEP = int64_t(NT) * N;
    __shared__ MaxSum ms[2][W];
    __shared__ float fs[W];
    const float c = kLog2e / temp;
    const int w = threadIdx.x / kWave;
    for (int64_t r = blockIdx.x; r < m; r += gridDim.x) {
        const T* row = S + r * lds;
        const RowEntries e = row_entries(t, r);
        MaxSum a = kNothing;
        int64_t j = int64_t(threadIdx.x) * N;
        for (; j + (kAhead - 1) * STEP <= V - N; j += kAhead * STEP) {
            Vec<T, N> v[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) v[k] = load_vec_nt<T, N>(row + j + k * STEP);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) add_pack<T, N>(a, v[k], 0, c);
        }
        for (; j < V; j += STEP) {
            const Place at = place<N>(j, V);
            add_pack<T, N>(a, load_vec_nt<T, N>(row + at.c), at.skip, c);
        }
        a = wave_merge(a, c);
        MaxSum b = wave_merge(teacher_sums<NT>(t, e, V, c), c);
        if (lane_id() == 0) {
            ms[0][w] = a;
            ms[1][w] = b;
        }
        __syncthreads();
        a = merge_of(ms[0], W, c);
        b = merge_of(ms[1], W, c);
        const bool none = is_empty(a) || is_empty(b);
        const RowStat st = {a.m, log2f(a.s), b.m, log2f(b.s), none ? 0.f : (weight ? weight[r] : 1.f) * temp};
        const float x = wave_total(none ? 0.f : teacher_loss<T, NT>(t, e, row, V, c, st));
        if (lane_id() == 0) fs[w] = x;
        __syncthreads();
        if (threadIdx.x == 0) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < W; ++i) sum += fs[i];
            loss[r] = sum * kLn2 * temp * temp;
            if (stat) stat[r] = st;
        }
    }
}

// p over a stretch of columns [c0, c0 + n), gathered in LDS (entries of one
// column add up).
template <int NT>
__device__ inline void gather_teacher(const Entries& t, const RowEntries& e, float tm, float tl2, int64_t V, float c,
                                      int64_t c0, int n, float* p) {
    for (int x = threadIdx.x; x < n; x += NT) p[x] = 0.f;
    __syncthreads();
    for (int64_t k = threadIdx.x; k < e.n; k += NT) {
        const int64_t col = load_column(t.idx, t.ib, e.i0 + k);
        if (col < 0 || col >= V || col < c0 || col >= c0 + n) continue;
        atomicAdd(&p[col - c0], exp2_of((load_value(t.val, t.vt, e.v0 + k) - tm) * c - tl2));
    }
    __syncthreads();
}

// the last pack of a row is stored without the elements of the pack before it
template <typename T, int N>
__device__ inline void store_from(T* p, Vec<T, N> v, int skip) {
    if (skip <= 0) {
        store_vec_nt<T, N>(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i >= skip) p[i] = v[i];
}

// Gradient of a chunk of a row; the logits are read again.
constexpr int kGradPacks = 4;
template <typename T, int N>
__global__ __launch_bounds__(kBlock) void distill_grad_chunks(const T* __restrict__ S, int64_t lds, int64_t m,
                                                              int64_t V, Entries t, float temp,
                                                              const RowStat* __restrict__ stat, T* __restrict__ dS,
                                                              int64_t ldd, int64_t chunks) {
    constexpr int COLS = kBlock * kGradPacks * N;
    __shared__ float p[COLS];
    const float c = kLog2e / temp;
    for (int64_t u = blockIdx.x; u < m * chunks; u += gridDim.x) {
        const int64_t r = u / chunks, c0 = u % chunks * COLS;
        const RowStat st = stat[r];
        const bool zero = st.scale == 0.f;  // (whatever the logits hold)
        Vec<T, N> v[kGradPacks];
        Place at[kGradPacks];
#pragma unroll
        for (int k = 0; k < kGradPacks; ++k) at[k] = place<N>(c0 + (int64_t(k) * kBlock + threadIdx.x) * N, V);
        if (!zero) {
#pragma unroll
            for (int k = 0; k < kGradPacks; ++k) v[k] = load_vec_nt<T, N>(S + r * lds + at[k].c);
            gather_teacher<kBlock>(t, row_entries(t, r), st.tm, st.tl2, V, c, c0, COLS, p);
        }
#pragma unroll
        for (int k = 0; k < kGradPacks; ++k) {
            if (at[k].skip >= N) break;
            Vec<T, N> o;
#pragma unroll
            for (int i = 0; i < N; ++i)
                o[i] = T(zero || i < at[k].skip
                             ? 0.f
                             : (exp2_of((float(v[k][i]) - st.m) * c - st.l2) - p[at[k].c + i - c0]) * st.scale);
            store_from<T, N>(dS + r * ldd + at[k].c, o, at[k].skip);
        }
        __syncthreads();
    }
}

// Loss and gradient with the row in registers: NP packs per thread.
//
// Up to one entry per thread the entries go to the threads that hold their
// columns by lists in LDS; those threads also hand back the logit that the
// loss needs, so that nothing is gathered from memory.  With more entries the
// row is stored without the teacher's part first, and the columns that have
// one are stored again, a stretch of columns at a time.
template <typename T, int N, int NT, int NP>
__global__ __launch_bounds__(NT) void distill_fused(const T* __restrict__ S, int64_t lds, int64_t m, int V,
                                                    Entries t, float temp, const float* __restrict__ weight,
                                                    float* __restrict__ loss, T* dS, int64_t ldd) {
    constexpr int W = NT / kWave;
    __shared__ MaxSum ms[2][W];
    __shared__ float lsum[W];
    __shared__ int head[NT], next_s[NT], col_s[NT];
    __shared__ float p_s[NT], lq_s[NT];
    __shared__ float dense[NT * N];
    const float c = kLog2e / temp;
    const int tid = threadIdx.x, w = tid / kWave;
    const int64_t step = gridDim.x;
    Vec<T, N> v[NP];
    // Pack k: its first column, moved back onto the row's end, and the elements
    // before its own.  (Both are formed where they are used: kept for all packs
    // they would take the registers of the row.)
    int c0 = tid * N;
    auto fresh = [&]() { asm volatile("" : "+v"(c0)); };
    auto column = [&](int k) { return min(c0 + k * NT * N, V - N); };
    auto skip = [&](int k) { return c0 + k * NT * N - (V - N); };
    auto load = [&](const T* row, int k) {
        const uint32_t bytes = uint32_t(column(k)) * uint32_t(sizeof(T));
        return load_vec_nt<T, N>(reinterpret_cast<const T*>(reinterpret_cast<const char*>(row) + bytes));
    };
    // the thread's entry of a row (-1: none)
    auto entry = [&](const RowEntries& e, int& col, float& val) {
        col = -1;
        val = 0.f;
        if (e.n > NT || tid >= e.n) return;
        const int64_t x = load_column(t.idx, t.ib, e.i0 + tid);
        val = load_value(t.val, t.vt, e.v0 + tid);
        if (x >= 0 && x < V) col = int(x);
    };
    int64_t r = blockIdx.x;
    if (r >= m) return;
    RowEntries e = row_entries(t, r);
    int col;
    float val;
    entry(e, col, val);
#pragma unroll
    for (int k = 0; k < NP; ++k) v[k] = load(S + r * lds, k);
    for (int64_t last = -1;; last = r, r += step) {
        const bool more = r + step < m;
        const RowEntries enext = more ? row_entries(t, r + step) : RowEntries{0, 0, 0};
        const float wr = weight ? weight[r] : 1.f;
        MaxSum a = kNothing;
        fresh();
#pragma unroll
        for (int k = 0; k < NP; ++k)
            if (skip(k) < N) add_pack<T, N>(a, v[k], skip(k), c);
        MaxSum b = kNothing;
        if (e.n > NT)
            b = teacher_sums<NT>(t, e, V, c);
        else if (col >= 0)
            add_value(b, val, c);
        a = wave_merge(a, c);
        b = wave_merge(b, c);
        if (lane_id() == 0) {
            ms[0][w] = a;
            ms[1][w] = b;
        }
        head[tid] = -1;
        lds_barrier();
        if (tid == 0 && last >= 0) {  // (the sums of the row before)
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < W; ++i) sum += lsum[i];
            loss[last] = sum * kLn2 * temp * temp;
        }
        a = merge_of(ms[0], W, c);
        b = merge_of(ms[1], W, c);
        const bool none = is_empty(a) || is_empty(b);
        const RowStat st = {a.m, log2f(a.s), b.m, log2f(b.s), none ? 0.f : wr * temp};
        const bool zero = st.scale == 0.f;  // (whatever the logits hold)
        const bool listed = e.n <= NT;
        float lp = 0.f, p = 0.f;
        if (col >= 0) {
            lp = (val - st.tm) * c - st.tl2;
            p = exp2_of(lp);
            col_s[tid] = col;
            p_s[tid] = p;
            next_s[tid] = atomicExch(&head[col / N % NT], tid);
        }
        lds_barrier();
        const int had = col;
        entry(enext, col, val);
        // the packs of this thread that have entries
        uint32_t packs = 0;
        const int first = head[tid];
        for (int x = first; x >= 0; x = next_s[x]) packs |= 1u << (col_s[x] / (N * NT));
        const T* const ahead = S + (more ? r + step : r) * lds;
        T* const out = dS + r * ldd;
        fresh();
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            if (skip(k) < N) {
                float g[N];
#pragma unroll
                for (int i = 0; i < N; ++i) g[i] = exp2_of((float(v[k][i]) - st.m) * c - st.l2);
                if (packs >> k & 1) {
                    for (int x = first; x >= 0; x = next_s[x]) {
                        if (col_s[x] / (N * NT) != k) continue;
                        const int j = col_s[x] - column(k);
                        const float px = p_s[x];
#pragma unroll
                        for (int i = 0; i < N; ++i)
                            if (i == j) {
                                g[i] -= px;
                                lq_s[x] = (float(v[k][i]) - st.m) * c - st.l2;
                            }
                    }
                }
                Vec<T, N> o;
#pragma unroll
                for (int i = 0; i < N; ++i) o[i] = T(zero ? 0.f : g[i] * st.scale);
                const uint32_t bytes = uint32_t(column(k)) * uint32_t(sizeof(T));
                store_from<T, N>(reinterpret_cast<T*>(reinterpret_cast<char*>(out) + bytes), o, skip(k));
            }
            if (more) v[k] = load(ahead, k);
        }
        if (!listed && !zero) {
            __threadfence();  // (stores to one address, by different threads)
            for (int x0 = 0; x0 < V; x0 += NT * N) {
                __syncthreads();
                gather_teacher<NT>(t, e, st.tm, st.tl2, V, c, x0, NT * N, dense);
                for (int x = tid; x < min(NT * N, V - x0); x += NT)
                    if (dense[x] != 0.f)
                        out[x0 + x] = T((exp2_of((float(S[r * lds + x0 + x]) - st.m) * c - st.l2) - dense[x]) * st.scale);
            }
        }
        lds_barrier();
        float x = 0.f;
        if (!none) x = !listed ? teacher_loss<T, NT>(t, e, S + r * lds, V, c, st)
                               : had >= 0 ? loss_term(p, lp, lq_s[tid]) : 0.f;
        x = wave_total(x);
        if (lane_id() == 0) lsum[w] = x;
        e = enext;
        if (!more) break;
    }
    lds_barrier();
    if (tid == 0) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) sum += lsum[i];
        loss[r] = sum * kLn2 * temp * temp;
    }
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int kFusedPacks = 16;  // packs per thread of a row in registers, at most
inline bool fused(int64_t v, int dt) { return ceil_div(v * dtype_bytes(dt), 16) <= int64_t(kFusedPacks) * kRowBlock; }

}  // namespace

size_t distill_tmp_bytes(int64_t m, int64_t v, int dt, bool grad) {
    return grad && !fused(v, dt) ? size_t(m) * sizeof(RowStat) : 0;
}

void distill(const DenseRows& S, const Entries& t, float temperature, const float* weight, float* loss,
             const DenseRows& dS, void* tmp, hipStream_t s) {
    by_width(S.dt, S.n, [&](auto e, auto width) {
        using T = decltype(e);
        constexpr int N = decltype(width)::value;
        const int64_t m = S.m, V = S.n, packs = ceil_div(V, N);
        const T* x = static_cast<const T*>(S.p);
        T* g = static_cast<T*>(dS.p);
        if (g && fused(V, S.dt)) {
            auto launch = [&](auto nt, auto np, int per_cu) {
                constexpr int NT = decltype(nt)::value, NP = decltype(np)::value;
                distill_fused<T, N, NT, NP><<<unsigned(std::min<int64_t>(m, int64_t(per_cu) * kCus)), NT, 0, s>>>(
                    x, S.ld, m, int(V), t, temperature, weight, loss, g, dS.ld);
            };
            using std::integral_constant;
            const integral_constant<int, kBlock> small;
            const integral_constant<int, kRowBlock> large;
            if (packs <= kBlock)
                return launch(small, integral_constant<int, 1>(), 8);
            if constexpr (N > 1) {
                if (packs <= 4 * kBlock) return launch(small, integral_constant<int, 4>(), 6);
                if (packs <= 4 * kRowBlock) return launch(large, integral_constant<int, 4>(), 2);
                if (packs <= 8 * kRowBlock) return launch(large, integral_constant<int, 8>(), 1);
                if (packs <= 12 * kRowBlock) return launch(large, integral_constant<int, 12>(), 1);
                return launch(large, integral_constant<int, kFusedPacks>(), 1);
            }
        }
        RowStat* stat = g ? static_cast<RowStat*>(tmp) : nullptr;
        const unsigned rows = unsigned(std::min<int64_t>(m, int64_t(1) << 20));
        if (N == 1 || packs <= 4 * kBlock)
            distill_rows<T, N, kBlock><<<rows, kBlock, 0, s>>>(x, S.ld, m, V, t, temperature, weight, loss, stat);
        else if constexpr (N > 1)
            distill_rows<T, N, kRowBlock><<<rows, kRowBlock, 0, s>>>(x, S.ld, m, V, t, temperature, weight, loss, stat);
        if constexpr (N > 1) {
            if (!stat) return;
            constexpr int64_t COLS = int64_t(kBlock) * kGradPacks * N;
            const int64_t chunks = ceil_div(V, COLS);
            distill_grad_chunks<T, N><<<unsigned(std::min<int64_t>(m * chunks, int64_t(1) << 20)), kBlock, 0, s>>>(
                x, S.ld, m, V, t, temperature, stat, g, dS.ld, chunks);
        }
    });
}

}  // namespace spsyrk
