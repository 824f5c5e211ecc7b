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
// of two of (s - max) c, c = log2(e) / T; all sums are 32-bit floats.
//
// The gradient of a row of up to 256 KB is computed with the whole row in one
// workgroup's registers, so that it is read once; the workgroup goes on to
// further rows, and a pack's registers take the next row's pack as soon as its
// gradient is stored, which keeps loads in flight all the time.  Longer rows
// are read twice, first for their sums, then by chunks.
#include <algorithm>

#include "internal.h"
#include "rows.h"

// Products and sums are fused where fmaf says so, and nowhere else: the loss
// has the same bits alone and with the gradient.
#pragma clang fp contract(off)

namespace spsyrk {
namespace {

constexpr int kRowBlock = 1024;  // threads per row, at most
constexpr int kMostWaves = kRowBlock / kWave;
constexpr int kCus = 256;  // compute units of the chip
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct RowStat {
    // log2 q = (s - m0) c - b0 - l2: b0 is the maximum's base, or m0 the
    // maximum; l2 is log2 of the sum of exponentials relative to it, `sum`
    float m0, b0, l2, sum;
    float tm, tl2;  // maximum and log2 of the sum of the teacher's entries
    float scale;    // weight T, 0 for a row without a gradient
    __device__ inline float log2q(float s, float c) const { return fmaf(s - m0, c, -b0) - l2; }
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

// the pack's own elements
template <typename T, int N>
__device__ inline void add_pack(MaxSum& a, Vec<T, N> v, int shift, float c) {
    float x[N], m = a.m;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = float(v[i]);
    if (shift != 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = mine<N>(shift, i) ? x[i] : -INFINITY;
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

// Sums over the logits are formed with s c - b, one operation, where the base b
// of a maximum is fl(max c): its rounding, a power of two 2^r with |r| up to half
// an ulp of max c, is a factor common to all exponentials and to their sum, and
// leaves q = 2^(s c - b) / sum as it is as long as 2^r is moderate.  So the
// bases end at 2^24, where r is a half.  Below -2^24 (logits masked by a large
// finite value) the base stays there: the exponents are then what they are,
// negative and exact, and go to 0 under a later, ordinary maximum.  Rows whose
// own maximum lies past 2^24 in either direction are done again from memory,
// differences first.  (A maximum of -inf has the lowest base too: 2^-inf is 0.)
constexpr float kMostBase = 16777216.f;
__device__ inline float base_of(float m, float c) { return fmaxf(m * c, -kMostBase); }
__device__ inline float scaled_base(MaxSum a, float m, float c) {
    return a.s * exp2_of(base_of(a.m, c) - base_of(m, c));
}
__device__ inline MaxSum wave_merge_base(MaxSum a, float c) {
    const float m = wave_max(a.m);
    return {m, wave_total(scaled_base(a, m, c))};
}
__device__ inline bool out_of_range(float m, float c) {
    return fabsf(m) < INFINITY && !(fabsf(m * c) < kMostBase);
}
template <typename T, int N>
__device__ inline void add_pack_base(MaxSum& a, Vec<T, N> v, int shift, float c) {
    float x[N], m = a.m;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = float(v[i]);
    if (shift != 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = mine<N>(shift, i) ? x[i] : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, x[i]);
    const float base = base_of(m, c);
    float s = a.s;
    if (m > a.m) s = scaled_base(a, m, c);
#pragma unroll
    for (int i = 0; i < N; ++i) s += exp2_of(fmaf(x[i], c, -base));
    a.m = m;
    a.s = s;
}

// The row's sums from each thread's, in every thread, and what follows from
// them; ms is written here.  b: the teacher's.
template <typename T, int N>
__device__ inline RowStat row_stat(MaxSum a, MaxSum b, const T* row, int64_t V, float c, float weight, float temp,
                                   MaxSum (*ms)[kMostWaves], bool* none, bool* far) {
    const int W = blockDim.x / kWave;
    const int w = threadIdx.x / kWave, l = lane_id();
    a = wave_merge_base(a, c);
    b = wave_merge(b, c);
    if (l == 0) {
        ms[0][w] = a;
        ms[1][w] = b;
    }
    // (the values are chosen between, not their addresses: those of LDS and of
    // a constant would make the loads flat ones, which wait for all others)
    auto part = [&](int k) {
        const MaxSum x = ms[k][min(l, W - 1)];
        return MaxSum{l < W ? x.m : -INFINITY, l < W ? x.s : 0.f};
    };
    lds_barrier();
    a = wave_merge_base(part(0), c);
    b = wave_merge(part(1), c);
    // (every thread of the workgroup has the same sums)
    *far = out_of_range(a.m, c);
    if (*far) {
        MaxSum x = kNothing;
        for (int64_t j = int64_t(threadIdx.x) * N; j < V; j += int64_t(blockDim.x) * N) {
            const Place at = place<N>(j, V);
            add_pack<T, N>(x, load_vec<T, N>(row + at.c), at.shift, c);
        }
        x = wave_merge(x, c);
        __syncthreads();
        if (l == 0) ms[0][w] = x;
        __syncthreads();
        a = wave_merge(part(0), c);
    }
    *none = is_empty(a) || is_empty(b);
    return {*far ? a.m : 0.f, *far ? 0.f : base_of(a.m, c), log2f(a.s), a.s, b.m, log2f(b.s), *none ? 0.f : weight * temp};
}

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

// The threads' parts of the sums over the teacher's entries, and of the loss:
// every blockDim.x-th entry from the k-th on.
__device__ inline void teacher_sums(MaxSum& b, const Entries& t, const RowEntries& e, int64_t k, int64_t V, float c) {
    for (; k < e.n; k += blockDim.x) {
        const int64_t col = load_column(t.idx, t.ib, e.i0 + k);
        if (col >= 0 && col < V) add_value(b, load_value(t.val, t.vt, e.v0 + k), c);
    }
}
template <typename T>
__device__ inline void teacher_loss(float& x, const Entries& t, const RowEntries& e, int64_t k, const T* row,
                                    int64_t V, float c, const RowStat& st) {
    for (; k < e.n; k += blockDim.x) {
        const int64_t col = load_column(t.idx, t.ib, e.i0 + k);
        if (col < 0 || col >= V) continue;
        const float lp = (load_value(t.val, t.vt, e.v0 + k) - st.tm) * c - st.tl2;
        x += loss_term(exp2_of(lp), lp, st.log2q(float(row[col]), c));
    }
}

// Loss of a row and what its gradient needs.
constexpr int kAhead = 4;  // packs per thread in flight
//
// MOST: the threads of a row, at most.  Rows of more than 512 keep to 64
// registers, so that two of them are on a compute unit (8192 x 65537 f32: 316
// us, 371 without); for the others that would only spill (16384 x 32768 bf16:
// 178 us, 191 so).
template <typename T, int N, int MOST>
__global__ __launch_bounds__(MOST, MOST > 512 ? 8 : 1) void distill_rows(const T* __restrict__ S, int64_t lds, int64_t m, int64_t V,
                                                          Entries t, float temp, const float* __restrict__ weight,
                                                          float* __restrict__ loss, RowStat* __restrict__ stat) {
    __shared__ MaxSum ms[2][kMostWaves];
    __shared__ float fs[kMostWaves];
    const int64_t STEP = int64_t(blockDim.x) * N;
    const float c = kLog2e / temp;
    const int w = threadIdx.x / kWave;
    for (int64_t r = blockIdx.x; r < m; r += gridDim.x) {
        const T* row = S + r * lds;
        const RowEntries e = row_entries(t, r);
        // the thread's first entry and its logit, on their way with the row
        const int64_t k0 = threadIdx.x;
        int64_t col = -1;
        float val = 0.f, logit = 0.f;
        if (k0 < e.n) {
            col = load_column(t.idx, t.ib, e.i0 + k0);
            val = load_value(t.val, t.vt, e.v0 + k0);
            if (col >= V) col = -1;
            if (col >= 0) logit = float(row[col]);
        }
        MaxSum a = kNothing;
        for (int64_t j = int64_t(threadIdx.x) * N - misaligned<T, N>(row); j < V; j += kAhead * STEP) {
            Vec<T, N> v[kAhead];
            // (only the row's very first pack can start before it)
            if (j >= 0 && j + (kAhead - 1) * STEP <= V - N) {
#pragma unroll
                for (int k = 0; k < kAhead; ++k) v[k] = load_vec_nt<T, N>(row + j + k * STEP);
#pragma unroll
                for (int k = 0; k < kAhead; ++k) add_pack_base<T, N>(a, v[k], 0, c);
            } else {
                Place at[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    at[k] = place<N>(j + k * STEP, V);
                    v[k] = load_vec_nt<T, N>(row + at[k].c);
                }
#pragma unroll
                for (int k = 0; k < kAhead; ++k)
                    if (at[k].shift < N) add_pack_base<T, N>(a, v[k], at[k].shift, c);
            }
        }
        MaxSum b = kNothing;
        if (col >= 0) add_value(b, val, c);
        teacher_sums(b, t, e, k0 + blockDim.x, V, c);
        bool none, far;
        const RowStat st = row_stat<T, N>(a, b, row, V, c, weight ? weight[r] : 1.f, temp, ms, &none, &far);
        float x = 0.f;
        if (!none) {
            const float lp = (val - st.tm) * c - st.tl2;
            if (col >= 0) x = loss_term(exp2_of(lp), lp, st.log2q(logit, c));
            teacher_loss<T>(x, t, e, k0 + blockDim.x, row, V, c, st);
        }
        x = wave_total(x);
        if (lane_id() == 0) fs[w] = x;
        __syncthreads();
        if (threadIdx.x == 0) {
            float sum = 0.f;
            for (int i = 0; i < int(blockDim.x / kWave); ++i) sum += fs[i];
            loss[r] = sum * kLn2 * temp * temp;
            if (stat) stat[r] = st;
        }
    }
}

// p over a stretch of columns [c0, c0 + n), gathered in LDS (entries of one
// column add up).
__device__ inline void gather_teacher(const Entries& t, const RowEntries& e, float tm, float tl2, int64_t V, float c,
                                      int64_t c0, int n, float* p) {
    for (int x = threadIdx.x; x < n; x += blockDim.x) p[x] = 0.f;
    __syncthreads();
    for (int64_t k = threadIdx.x; k < e.n; k += blockDim.x) {
        const int64_t col = load_column(t.idx, t.ib, e.i0 + k);
        if (col < 0 || col >= V || col < c0 || col >= c0 + n) continue;
        atomicAdd(&p[col - c0], exp2_of((load_value(t.val, t.vt, e.v0 + k) - tm) * c - tl2));
    }
    __syncthreads();
}

// the pack's own elements
template <typename T, int N>
__device__ inline void store_own(T* p, Vec<T, N> v, int shift) {
    if (shift == 0) {
        store_vec_nt<T, N>(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (mine<N>(shift, i)) p[i] = v[i];
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
        const int64_t r = u / chunks, c0 = u % chunks * COLS - misaligned<T, N>(S + r * lds);
        const RowStat st = stat[r];
        const bool zero = st.scale == 0.f;  // (whatever the logits hold)
        Vec<T, N> v[kGradPacks];
        Place at[kGradPacks];
#pragma unroll
        for (int k = 0; k < kGradPacks; ++k) at[k] = place<N>(c0 + (int64_t(k) * kBlock + threadIdx.x) * N, V);
        if (!zero) {
#pragma unroll
            for (int k = 0; k < kGradPacks; ++k) v[k] = load_vec_nt<T, N>(S + r * lds + at[k].c);
            gather_teacher(t, row_entries(t, r), st.tm, st.tl2, V, c, c0, COLS, p);
        }
#pragma unroll
        for (int k = 0; k < kGradPacks; ++k) {
            if (at[k].shift >= N) break;
            Vec<T, N> o;
#pragma unroll
            for (int i = 0; i < N; ++i)
                o[i] = T(zero || !mine<N>(at[k].shift, i)
                             ? 0.f
                             : (exp2_of(st.log2q(float(v[k][i]), c)) - p[at[k].c + i - c0]) * st.scale);
            store_own<T, N>(dS + r * ldd + at[k].c, o, at[k].shift);
        }
        __syncthreads();
    }
}

// An entry as it lies in memory: loaded a row ahead, and looked at only then.
struct RawEntry {
    uint32_t lo, hi;   // column
    uint32_t v0, v1;   // value: 16 bits each
    __device__ inline int column(int ib, int V) const {
        return (ib == 4 || hi == 0) && lo < uint32_t(V) ? int(lo) : -1;
    }
    __device__ inline float value(int vt) const {
        if (vt == kDtF32) return __uint_as_float(v0 | v1 << 16);
        return vt == kDtBF16 ? __uint_as_float(v0 << 16) : float(__builtin_bit_cast(_Float16, uint16_t(v0)));
    }
};
__device__ inline RawEntry raw_entry(const Entries& t, int64_t i, int64_t v) {
    const char *p = static_cast<const char*>(t.idx) + i * t.ib;
    const char *q = static_cast<const char*>(t.val) + v * (t.vt == kDtF32 ? 4 : 2);
    return {*reinterpret_cast<const uint32_t*>(p), *reinterpret_cast<const uint32_t*>(p + (t.ib == 8 ? 4 : 0)),
            *reinterpret_cast<const uint16_t*>(q), *reinterpret_cast<const uint16_t*>(q + (t.vt == kDtF32 ? 2 : 0))};
}

// Loss and gradient with the row in registers: NP packs per thread, of as many
// threads as that takes.
//
// Up to one entry per thread the entries go to the threads that hold their
// columns by lists in LDS; those threads also hand back the logit that the
// loss needs, so that nothing is gathered from memory.  With more entries the
// row is stored without the teacher's part first, and the columns that have
// one are stored again, a stretch of columns at a time.
template <typename T, int N, int NP, int THREADS>
__global__ __launch_bounds__(kRowBlock) void distill_fused(const T* S, int64_t lds, int64_t m, int V, Entries t, float temp,
                                                    const float* __restrict__ weight, float* __restrict__ loss,
                                                    T* dS, int64_t ldd) {
    const int NT = THREADS ? THREADS : blockDim.x;  // (known for the longest rows)
    __shared__ MaxSum ms[2][kMostWaves];
    __shared__ float lsum[kMostWaves];
    extern __shared__ int lists[];  // fused_lds_bytes(NT, N)
    int* const head = lists;               // first entry of a thread's columns (-1: none)
    int* const link = head + NT;           // of an entry: its pack in the thread << 16 | the next entry + 1
    int* const col_s = link + NT;          // or -1 - the entry that stands for it
    float* const p_s = reinterpret_cast<float*>(col_s + NT);
    float* const lq_s = p_s + NT;
    float* const dense = lq_s + NT;        // NT N
    const float c = kLog2e / temp;
    const int tid = threadIdx.x, w = tid / kWave;
    const int64_t step = gridDim.x;
    Vec<T, N> v[NP];
    // A thread's packs lie NT N columns apart from c0 on, the first thread's as
    // far before the row as that is off a boundary; packs that pass the row's
    // ends are moved back into it.  (Columns are formed where they are used: kept
    // for all packs they would take the registers of the row.)
    const int span = NT * N, end = V - N;
    int c0 = tid * N - misaligned<T, N>(S + int64_t(blockIdx.x) * lds);
    auto fresh = [&]() { asm volatile("" : "+v"(c0)); };
    auto inside = [&](int col) { return max(min(col, end), 0); };
    // (mask 0: the row's first pack, by every thread)
    auto load = [&](const T* row, int col, uint32_t mask) {
        const uint32_t bytes = (uint32_t(inside(col)) * uint32_t(sizeof(T))) & mask;
        return load_vec_nt<T, N>(reinterpret_cast<const T*>(reinterpret_cast<const char*>(row) + bytes));
    };
    // the thread's entry of a row
    auto entry = [&](const RowEntries& e) {
        RawEntry x = {~0u, ~0u, 0, 0};
        if (e.n <= NT && tid < e.n) x = raw_entry(t, e.i0 + tid, e.v0 + tid);
        return x;
    };
    // the waves' parts of the loss of the row before
    auto put_loss = [&](int64_t row) {
        float sum = 0.f;
        for (int i = 0; i < NT / kWave; ++i) sum += lsum[i];
        loss[row] = sum * kLn2 * temp * temp;
    };
    int64_t r = blockIdx.x;
    if (r >= m) return;
    RowEntries e = row_entries(t, r);
    RawEntry ahead = entry(e);
#pragma unroll
    for (int k = 0, at = c0; k < NP; ++k, at += span) v[k] = load(S + r * lds, at, ~0u);
    for (int64_t last = -1;; last = r, r += step) {
        const bool more = r + step < m;
        const T* const row = S + r * lds;
        MaxSum a = kNothing;
        fresh();
#pragma unroll
        for (int k = 0, at = c0; k < NP; ++k, at += span)
            if (at < V) add_pack_base<T, N>(a, v[k], at - inside(at), c);
        // (nothing else is waited for before the packs, which come last)
        const RowEntries enext = more ? row_entries(t, r + step) : RowEntries{0, 0, 0};
        const float wr = weight ? weight[r] : 1.f;
        const int col = ahead.column(t.ib, V);
        const float val = ahead.value(t.vt);
        MaxSum b = kNothing;
        if (e.n > NT)
            teacher_sums(b, t, e, tid, V, c);
        else if (col >= 0)
            add_value(b, val, c);
        head[tid] = -1;
        bool none, far;
        const RowStat st = row_stat<T, N>(a, b, row, V, c, wr, temp, ms, &none, &far);
        if (tid == 0 && last >= 0) put_loss(last);
        const bool zero = st.scale == 0.f;  // (whatever the logits hold)
        const bool listed = e.n <= NT;
        float lp = 0.f, p = 0.f;
        if (col >= 0) {
            lp = (val - st.tm) * c - st.tl2;
            p = exp2_of(lp);
            col_s[tid] = col;
            p_s[tid] = p;
            const int pack = (col + misaligned<T, N>(row)) / N, k = pack / NT;
            link[tid] = k << 16 | (atomicExch(&head[pack - k * NT], tid) + 1);
        }
        lds_barrier();
        ahead = entry(enext);
        // The packs of this thread that have entries.  Entries of one column are
        // added up at the one that the list has first (of two, the sum has one
        // value in either order, and the list may have either), and leave it: of
        // their column stays where its logit will be found.
        uint32_t packs = 0;
        const int first = head[tid];
        for (int x = first, before = -1; x >= 0;) {
            const int l = link[x], k = l >> 16;
            int y = x;
            if (packs >> k & 1)
                for (y = first; col_s[y] != col_s[x];) y = (link[y] & 0xffff) - 1;
            if (y == x) {
                packs |= 1u << k;
                before = x;
            } else {
                p_s[y] += p_s[x];
                col_s[x] = -1 - y;
                link[before] = (link[before] & ~0xffff) | (l & 0xffff);
            }
            x = (l & 0xffff) - 1;
        }
        // The next row's packs.  After the last row these are loads of nothing new:
        // under a condition they would have the sums wait for all packs at once.
        const T* const next = S + (more ? r + step : r) * lds;
        const uint32_t mask = more ? ~0u : 0u;
        const int shifted = misaligned<T, N>(row) - misaligned<T, N>(next);  // of the next row's packs against this one's
        T* const out = dS + r * ldd;
        const float qscale = st.scale / st.sum;
        fresh();
#pragma unroll
        for (int k = 0, at = c0; k < NP; ++k, at += span) {
            if (at < V) {
                float z[N], g[N];
                Vec<T, N> o;
#pragma unroll
                for (int i = 0; i < N; ++i) z[i] = fmaf(float(v[k][i]), c, -st.b0);
#pragma unroll
                for (int i = 0; i < N; ++i) g[i] = exp2_of(z[i]) * qscale;
                if (packs >> k & 1) {
                    for (int x = first; x >= 0; x = (link[x] & 0xffff) - 1) {
                        if (link[x] >> 16 != k) continue;
                        const int j = col_s[x] - inside(at);
                        const float px = p_s[x] * st.scale;
#pragma unroll
                        for (int i = 0; i < N; ++i)
                            if (i == j) {
                                g[i] -= px;
                                lq_s[x] = z[i] - st.l2;
                            }
                    }
                }
#pragma unroll
                for (int i = 0; i < N; ++i) o[i] = T(g[i]);
                if (zero) o = Vec<T, N>(T(0.f));
                const uint32_t bytes = uint32_t(inside(at)) * uint32_t(sizeof(T));
                store_own<T, N>(reinterpret_cast<T*>(reinterpret_cast<char*>(out) + bytes), o, at - inside(at));
            }
            v[k] = load(next, at + shifted, mask);
        }
        c0 += shifted;
        if ((!listed || far) && !zero) {
            // columns with a teacher's part (all columns of a row out of range), again
            __threadfence();  // (stores to one address, by different threads)
            for (int x0 = 0; x0 < V; x0 += NT * N) {
                __syncthreads();
                gather_teacher(t, e, st.tm, st.tl2, V, c, x0, NT * N, dense);
                for (int x = tid; x < min(NT * N, V - x0); x += NT)
                    if (far || dense[x] != 0.f)
                        out[x0 + x] = T((exp2_of(st.log2q(float(row[x0 + x]), c)) - dense[x]) * st.scale);
            }
        }
        lds_barrier();
        float x = 0.f;
        if (!none) {
            if (!listed || far)
                teacher_loss<T>(x, t, e, tid, row, V, c, st);
            else if (col >= 0)
                x = loss_term(p, lp, lq_s[col_s[tid] < 0 ? -1 - col_s[tid] : tid]);
        }
        x = wave_total(x);
        if (lane_id() == 0) lsum[w] = x;
        e = enext;
        if (!more) break;
    }
    lds_barrier();
    if (tid == 0) put_loss(r);
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int kFusedPacks = 16;  // packs per thread of a row in registers, at most
// packs of a row (one more may be needed where rows lie off the boundaries)
inline int64_t row_packs(const DenseRows& S) {
    const int64_t n = 16 / dtype_bytes(S.dt);
    return ceil_div(S.n + (on_boundaries(S.p, S.ld, S.dt) ? 0 : n - 1), n);
}
inline bool fused(const DenseRows& S) { return row_packs(S) <= int64_t(kFusedPacks) * kRowBlock; }
inline size_t fused_lds_bytes(int threads, int width) { return size_t(threads) * (5 + width) * sizeof(float); }

// Threads per row: eight packs each, so that many rows are on a compute unit
// (more than eight where that takes over kRowBlock threads), but one per entry
// of a typical row at least (and one wavefront where there is neither: rows of
// no columns have losses too).  Loss and gradient take the same number, so that
// they sum in one order.
inline int row_threads(int64_t packs, const Entries& t) {
    const int64_t entries = t.rp ? 2 * (t.nnz / std::max<int64_t>(t.m, 1)) : t.per_row;
    const int64_t n = std::max({ceil_div(packs, 8), std::min<int64_t>(entries, 256), int64_t(1)});
    // (whole rounds of the four SIMDs: loss over 8192 x 60000 bf16 with 15
    // wavefronts a row 251 us, with 16 190)
    const int64_t unit = n > 4 * kWave ? 4 * kWave : kWave;
    return int(std::min<int64_t>(ceil_div(n, unit) * unit, kRowBlock));
}

}  // namespace

size_t distill_tmp_bytes(const DenseRows& S, bool grad) {
    return grad && !fused(S) ? size_t(S.m) * sizeof(RowStat) : 0;
}

void distill(const DenseRows& S, const Entries& t, float temperature, const float* weight, float* loss,
             const DenseRows& dS, void* tmp, hipStream_t s) {
    by_width(S.dt, S.n, [&](auto e, auto width) {
        using T = decltype(e);
        constexpr int N = decltype(width)::value;
        const int64_t m = S.m, V = S.n;
        const int64_t packs = N > 1 ? row_packs(S) : V;
        const int nt = row_threads(packs, t);
        const T* x = static_cast<const T*>(S.p);
        T* g = static_cast<T*>(dS.p);
        if (g && fused(S)) {
            // rows in flight: 16 to 24 wavefronts per compute unit, by the registers
            auto launch = [&](auto np, auto threads, int waves) {
                constexpr int NP = decltype(np)::value, THREADS = decltype(threads)::value;
                const int64_t blocks = int64_t(std::max(waves * kWave / nt, 1)) * kCus;
                distill_fused<T, N, NP, THREADS><<<unsigned(std::min(m, blocks)), nt, fused_lds_bytes(nt, N), s>>>(
                    x, S.ld, m, int(V), t, temperature, weight, loss, g, dS.ld);
            };
            using std::integral_constant;
            const integral_constant<int, 0> any;
            const integral_constant<int, kRowBlock> most;
            if (packs <= nt) return launch(integral_constant<int, 1>(), any, 24);
            if constexpr (N > 1) {
                if (packs <= 2 * nt) return launch(integral_constant<int, 2>(), any, 24);
                if (packs <= 4 * nt) return launch(integral_constant<int, 4>(), any, 20);
                if (packs <= 8 * nt) {
                    if (nt < kRowBlock) return launch(integral_constant<int, 8>(), any, 16);
                    return launch(integral_constant<int, 8>(), most, 16);
                }
                // (a pack that no thread needs costs its place in the loops: 8192 x
                // 65537 bf16, 8193 packs, 490 us with ten a thread, 516 with twelve)
                if (packs <= 10 * nt) return launch(integral_constant<int, 10>(), most, 16);
                if (packs <= 12 * nt) return launch(integral_constant<int, 12>(), most, 16);
                if (packs <= 14 * nt) return launch(integral_constant<int, 14>(), most, 16);
                return launch(integral_constant<int, kFusedPacks>(), most, 16);
            }
        }
        RowStat* stat = g ? static_cast<RowStat*>(tmp) : nullptr;
        const unsigned rows = unsigned(std::min<int64_t>(m, int64_t(1) << 20));
        if (nt <= 512)
            distill_rows<T, N, 512><<<rows, nt, 0, s>>>(x, S.ld, m, V, t, temperature, weight, loss, stat);
        else if constexpr (N > 1)
            distill_rows<T, N, kRowBlock><<<rows, nt, 0, s>>>(x, S.ld, m, V, t, temperature, weight, loss, stat);
        if constexpr (N > 1) {
            if (!stat) return;
            constexpr int64_t COLS = int64_t(kBlock) * kGradPacks * N;
            const int64_t chunks = ceil_div(V + N - 1, COLS);
            distill_grad_chunks<T, N><<<unsigned(std::min<int64_t>(m * chunks, int64_t(1) << 20)), kBlock, 0, s>>>(
                x, S.ld, m, V, t, temperature, stat, g, dS.ld, chunks);
        }
    });
}

}  // namespace spsyrk
