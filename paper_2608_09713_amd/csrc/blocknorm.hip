// The norms before and after a block, with its gate and residual scale, and
// their gradient.
//
//     u = b r1 post,  r1 = 1 / sqrt(sum b^2 / d + eps)   (or u = b),
//     y = x + s gate u,  h = y r2 pre,  r2 = 1 / sqrt(sum y^2 / d + eps);
//     n2 = y r2,  a = dh pre,  Y = dy + r2 (a - n2 sum(a n2) / d),  dx = Y,
//     n1 = b r1,  c = s gate Y post,  db = r1 (c - n1 sum(c n1) / d)   (or s gate Y),
//     dpre = sum over rows of dh n2,  S = sum over rows of Y n1,
//     dgate = s post S,  dpost = s gate S.
//
// Bound by the bytes of the rows: x and b (the gradient: dy, dh, y, b) are read
// once, y and h (dx and db) written once, in one launch, a row in registers in
// between as in the layer norm.  The rows that share a row of the gate share S,
// so its gradient and that of post are one sum, told apart when the workgroups'
// parts are added up, in their order, by a second launch.  A gate of a row's own
// has its gradient written with the row.  Several rows of the gate: a workgroup
// keeps the sum of gate S over its groups, which is dpost's share.  y is rounded
// when it is stored; h and r2 come from the sum before that.
//
// 32768 x 4096 bf16, forward: 197 us, 5.4 TB/s; 16384 x 8192 with a gate of each
// row's own, gradient: 432 us, 5.0 TB/s; with one gate 8192 x 8192: 178 us, 4.5.  The
// gradient's loads of a row stand before its two sums and its stores behind them;
// loading a row ahead took the registers of other wavefronts (432 us: 564).
#include "internal.h"
#include "row_shape.h"
#include "training.h"

namespace spsyrk {
namespace {

// N elements from i on of an array of 32-bit floats or of T, as 32-bit floats; none where p is null
template <typename T, int N>
__device__ inline void load_any(const void* p, bool wide, int64_t i, float none, float (&out)[N]) {
    if (!p) {
#pragma unroll
        for (int k = 0; k < N; ++k) out[k] = none;
    } else if (wide) {
        const Vec<float, N> v = load_vec<float, N>(static_cast<const float*>(p) + i);
#pragma unroll
        for (int k = 0; k < N; ++k) out[k] = v[k];
    } else {
        const Vec<T, N> v = load_vec<T, N>(static_cast<const T*>(p) + i);
#pragma unroll
        for (int k = 0; k < N; ++k) out[k] = float(v[k]);
    }
}
template <typename T, int N>
__device__ inline void store_any(void* p, bool wide, int64_t i, const float (&v)[N]) {
    if (wide) {
        Vec<float, N> o;
#pragma unroll
        for (int k = 0; k < N; ++k) o[k] = v[k];
        store_vec<float, N>(static_cast<float*>(p) + i, o);
    } else {
        Vec<T, N> o;
#pragma unroll
        for (int k = 0; k < N; ++k) o[k] = T(v[k]);
        store_vec<T, N>(static_cast<T*>(p) + i, o);
    }
}

// Column c of a row in registers (fewer than 2^16 columns): an unsigned 32-bit
// offset, so that the row's address can stay in scalar registers.
template <typename T>
__device__ inline T* column(T* row, int c) {
    typedef typename std::conditional<std::is_const<T>::value, const char, char>::type B;
    return reinterpret_cast<T*>(reinterpret_cast<B*>(row) + uint32_t(c) * uint32_t(sizeof(T)));
}

// Keeps a pack of 16-bit elements as it is in its registers: what is made of it
// before cannot be held, converted, in twice as many until it is used after.
template <typename T>
__device__ inline void keep_packed(Vec<T, 16 / int(sizeof(T))>& v) {
    typedef unsigned U __attribute__((ext_vector_type(4)));
    U u = __builtin_bit_cast(U, v);
    asm volatile("" : "+v"(u));
    v = __builtin_bit_cast(Vec<T, 16 / int(sizeof(T))>, u);
}

// N elements that are loaded now and converted when they are used: of T, or (ANY)
// of T or 32-bit floats.
template <typename T, int N, bool ANY>
struct Held {
    Vec<T, N> v;
    __device__ void load(const void* p, bool, int64_t i, float none) {
        if (p) {
            v = load_vec<T, N>(static_cast<const T*>(p) + i);
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = T(none);
        }
    }
    __device__ float get(int k) const { return float(v[k]); }
    __device__ void keep() {
        if constexpr (sizeof(T) == 2 && N > 1) keep_packed<T>(v);
    }
};
template <typename T, int N>
struct Held<T, N, true> {
    float v[N];
    __device__ void load(const void* p, bool wide, int64_t i, float none) { load_any<T, N>(p, wide, i, none, v); }
    __device__ float get(int k) const { return v[k]; }
    __device__ void keep() {}
};

// a row's own gate, or one that `per` rows share
__device__ inline int64_t gate_row(const BlockGate& g, int64_t r) {
    return g.own ? r : int64_t(uint32_t(r) / uint32_t(g.per));
}

// f(own) for the elements of a pack: whether each belongs to this thread alone.
// Only the last wavefront of a row has a lane where some do not, so the others
// go without the comparisons.
template <int N, int NP, typename F>
__device__ inline void each_own(const Place (&at)[NP], int k, F f) {
    if (k < NP - 1 || at[k].shift == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) f(i, true);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) f(i, i >= at[k].shift);
    }
}

// OWN: a gate of each row's own; else post gate is held, for the rows that share it.
template <typename T, int N, int L, int MOST, int NP, bool ANY, bool OWN>
__global__ __launch_bounds__(MOST) void after_block(
    const T* __restrict__ x, int64_t ldx, const T* __restrict__ b, int64_t ldb, int64_t m, int64_t d, BlockGate gate,
    float scale, BlockParams par, bool normed, float eps, T* __restrict__ y, int64_t ldy, T* __restrict__ h,
    int64_t ldh, float* __restrict__ rstd_post, float* __restrict__ rstd_pre) {
    constexpr int ROWS = L ? MOST / (L ? L : 1) : 1;
    __shared__ float buf[2][2][kMostWaves];
    const int threads = L ? L : int(blockDim.x), l = L ? int(threadIdx.x) % (L ? L : 1) : int(threadIdx.x);
    int turn = 0;
    Place at[NP];
    row_places<N>(l, threads, d, at);
    using P = Held<T, N, ANY>;
    struct Row {
        Vec<T, N> x[NP], b[NP];
        P gate[OWN ? NP : 1];
    };
    auto load = [&](int64_t r) {
        Row q;
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            q.x[k] = load_vec_nt<T, N>(column(x + r * ldx, at[k].c));
            q.b[k] = load_vec_nt<T, N>(column(b + r * ldb, at[k].c));
            if constexpr (OWN) q.gate[k].load(gate.p, gate.wide, r * gate.ld + at[k].c, 1.f);
        }
        return q;
    };
    const int64_t step = int64_t(gridDim.x) * ROWS;
    int64_t r = int64_t(blockIdx.x) * ROWS + (L ? threadIdx.x / (L ? L : 1) : 0);
    Row next = load(min(r, m - 1));
    P post[NP], pre[NP];
    float mul[OWN ? 1 : NP][N];
#pragma unroll
    for (int k = 0; k < NP; ++k) {
        post[k].load(par.post, par.wide, at[k].c, 1.f);
        pre[k].load(par.pre, par.wide, at[k].c, 1.f);
    }
    int64_t held = -1;  // the row of the gate that mul has
    for (; r < m; r += step, turn ^= 1) {
        const Row q = next;
        next = load(min(r + step, m - 1));
        if constexpr (!OWN) {
            const int64_t want = gate_row(gate, r);
            if (want != held) {
                held = want;
#pragma unroll
                for (int k = 0; k < NP; ++k) {
                    load_any<T, N>(gate.p, gate.wide, want * gate.ld + at[k].c, 1.f, mul[k]);
#pragma unroll
                    for (int i = 0; i < N; ++i) mul[k][i] *= post[k].get(i);
                }
            }
        }
        float r1 = 1.f;
        if (normed) {
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < NP; ++k)
                each_own<N>(at, k, [&](int i, bool mine) {
                    const float z = mine ? float(q.b[k][i]) : 0.f;
                    s = fmaf(z, z, s);
                });
            r1 = 1.f / sqrtf(row_sum<L>(s, buf[turn][0]) / float(d) + eps);
            if (l == 0) rstd_post[r] = r1;
        }
        const float f = r1 * scale;
        float v[NP][N], s = 0.f;
#pragma unroll
        for (int k = 0; k < NP; ++k) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float w;
                if constexpr (OWN)
                    w = q.gate[k].get(i) * post[k].get(i);
                else
                    w = mul[k][i];
                v[k][i] = fmaf(float(q.b[k][i]) * f, w, float(q.x[k][i]));
            }
            each_own<N>(at, k, [&](int i, bool mine) {
                const float z = mine ? v[k][i] : 0.f;
                s = fmaf(z, z, s);
            });
        }
        const float r2 = 1.f / sqrtf(row_sum<L>(s, buf[turn][1]) / float(d) + eps);
        if (l == 0) rstd_pre[r] = r2;
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            if (at[k].shift >= N) break;
            Vec<T, N> oy, oh;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                oy[i] = T(v[k][i]);
                oh[i] = T(v[k][i] * r2 * pre[k].get(i));
            }
            store_vec_nt<T, N>(column(y + r * ldy, at[k].c), oy);
            store_vec_nt<T, N>(column(h + r * ldh, at[k].c), oh);
        }
    }
}

// rows too long for registers: three readings, the later ones from the caches
template <typename T>
__global__ __launch_bounds__(kRowBlock) void after_block_long(
    const T* __restrict__ x, int64_t ldx, const T* __restrict__ b, int64_t ldb, int64_t m, int64_t d, BlockGate gate,
    float scale, BlockParams par, bool normed, float eps, T* __restrict__ y, int64_t ldy, T* __restrict__ h,
    int64_t ldh, float* __restrict__ rstd_post, float* __restrict__ rstd_pre) {
    constexpr int N = 16 / int(sizeof(T));
    constexpr int64_t STEP = int64_t(kRowBlock) * N;
    __shared__ float buf[2][2][kMostWaves];
    int turn = 0;
    for (int64_t r = blockIdx.x; r < m; r += gridDim.x, turn ^= 1) {
        float r1 = 1.f;
        if (normed) {
            float s = 0.f;
            for (int64_t c = int64_t(threadIdx.x) * N; c < d; c += STEP) {
                const Place at = place<N>(c, d);
                const Vec<T, N> v = load_vec<T, N>(b + r * ldb + at.c);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float z = i >= at.shift ? float(v[i]) : 0.f;
                    s = fmaf(z, z, s);
                }
            }
            r1 = 1.f / sqrtf(row_sum<0>(s, buf[turn][0]) / float(d) + eps);
            if (threadIdx.x == 0) rstd_post[r] = r1;
        }
        const float f = r1 * scale;
        const int64_t at_gate = gate_row(gate, r) * gate.ld;
        auto sum_at = [&](int c, float (&out)[N]) {
            const Vec<T, N> vx = load_vec<T, N>(x + r * ldx + c), vb = load_vec<T, N>(b + r * ldb + c);
            float post[N], g[N];
            load_any<T, N>(par.post, par.wide, c, 1.f, post);
            load_any<T, N>(gate.p, gate.wide, at_gate + c, 1.f, g);
#pragma unroll
            for (int i = 0; i < N; ++i) out[i] = fmaf(float(vb[i]) * post[i], g[i] * f, float(vx[i]));
        };
        float s = 0.f;
        for (int64_t c = int64_t(threadIdx.x) * N; c < d; c += STEP) {
            const Place at = place<N>(c, d);
            float v[N];
            sum_at(at.c, v);
#pragma unroll
            for (int i = 0; i < N; ++i) s = i >= at.shift ? fmaf(v[i], v[i], s) : s;
        }
        const float r2 = 1.f / sqrtf(row_sum<0>(s, buf[turn][1]) / float(d) + eps);
        if (threadIdx.x == 0) rstd_pre[r] = r2;
        for (int64_t c = int64_t(threadIdx.x) * N; c < d; c += STEP) {
            const Place at = place<N>(c, d);
            float v[N], pre[N];
            sum_at(at.c, v);
            load_any<T, N>(par.pre, par.wide, at.c, 1.f, pre);
            Vec<T, N> oy, oh;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                oy[i] = T(v[i]);
                oh[i] = T(v[i] * r2 * pre[i]);
            }
            store_vec_nt<T, N>(y + r * ldy + at.c, oy);
            store_vec_nt<T, N>(h + r * ldh + at.c, oh);
        }
    }
}

// ---- gradient

constexpr int kGradBlock = 512;  // threads per workgroup where rows take lanes of a wavefront

// How the rows go over the workgroups.  Groups are the rows that share a row of
// the gate (one group of all rows where there is no gate, and where each row has
// its own).  A group is split into `parts`, taken by that many workgroups, and
// `slots` groups are under way at a time; with `whole` every row's threads take
// whole groups instead and write their gate's gradient themselves.
struct Spread {
    int64_t groups = 1, per = 1;
    int64_t slots = 1, parts = 1;
    bool whole = false;
    __host__ __device__ int64_t grid() const { return slots * parts; }
    // whether the workgroups finish the gate's gradient
    __host__ __device__ bool direct() const { return groups > 1 && parts == 1; }
};

// How the gate's rows go with the rows: one group, split over workgroups; several
// groups, each split; whole groups a row's threads; or a row each.
enum { kOne, kSplit, kWhole, kOwn };

// workspace: the workgroups' sums of dh n2, of several groups those of gate S, and
// S of the groups' parts that are still to be added up
struct Sums {
    float* pre = nullptr;
    float* post = nullptr;
    float* s = nullptr;
};
inline int64_t post_rows(const Spread& go) { return go.groups > 1 ? go.grid() : 0; }
inline int64_t s_rows(const Spread& go) { return go.direct() ? 0 : go.groups * go.parts; }

template <typename T>
struct GradArgs {
    const T *dy, *dh, *y, *b;
    int64_t ldy, ldh, ldo, ldb;
    int64_t m, d;
    int threads;  // of a row, where it takes more than a wavefront
    const float *rstd_post, *rstd_pre;
    BlockGate gate;
    BlockParams par;
    float scale;
    T *dx, *db;
    int64_t lddx, lddb;
    void* dgate;  // of the gate's type, rows of lddg
    int64_t lddg;
    Sums sums;
    Spread go;
};

// Sum over a row's threads: L lanes, or (L 0) `waves` wavefronts from `first` on
// with buf of kMostWaves words, not used again before the next sum's barrier.
template <int L>
__device__ inline float rows_sum(float v, float* buf, int first, int waves) {
    v = group_total<L ? L : kWave>(v);
    if constexpr (L == 0) {
        if (lane_id() == 0) buf[threadIdx.x / kWave] = v;
        lds_barrier();
        v = 0.f;
        for (int i = 0; i < waves; ++i) v += buf[first + i];
    }
    return v;
}

// The sums of the rows that a workgroup has under way, complete in the first
// row's threads.  L lanes: by lane distance in a wavefront, wavefronts pairwise
// through LDS; else the rows' threads one after another.
template <int L, int MOST, int N, int NP>
__device__ inline void add_rows(float (&v)[NP][N], float* lds, int threads, int subs) {
    if constexpr (L > 0) {
        constexpr int WAVES = MOST / kWave;
        const int w = threadIdx.x / kWave, lane = lane_id();
#pragma unroll
        for (int far = L; far < kWave; far *= 2)
#pragma unroll
            for (int k = 0; k < NP; ++k)
#pragma unroll
                for (int i = 0; i < N; ++i) v[k][i] += __shfl_xor(v[k][i], far, kWave);
#pragma unroll
        for (int half = WAVES / 2; half > 0; half /= 2) {
            if (w >= half && w < 2 * half)
#pragma unroll
                for (int k = 0; k < NP; ++k)
#pragma unroll
                    for (int i = 0; i < N; ++i) lds[(((w - half) * NP + k) * N + i) * kWave + lane] = v[k][i];
            __syncthreads();
            if (w < half)
#pragma unroll
                for (int k = 0; k < NP; ++k)
#pragma unroll
                    for (int i = 0; i < N; ++i) v[k][i] += lds[((w * NP + k) * N + i) * kWave + lane];
            __syncthreads();
        }
    } else if (subs > 1) {
        const int t = threadIdx.x;
        if (t >= threads)
#pragma unroll
            for (int k = 0; k < NP; ++k)
#pragma unroll
                for (int i = 0; i < N; ++i) lds[(k * N + i) * MOST + t] = v[k][i];
        __syncthreads();
        if (t < threads)
            for (int u = t + threads; u < threads * subs; u += threads)
#pragma unroll
                for (int k = 0; k < NP; ++k)
#pragma unroll
                    for (int i = 0; i < N; ++i) v[k][i] += lds[(k * N + i) * MOST + u];
        __syncthreads();
    }
}

// Four wavefronts a SIMD, two workgroups of 512 threads on a compute unit, even
// where sums are spilled for it (16384 x 4096, 64 groups: 162 us, 212 without the
// limit; 262144 x 128, 4096 groups: 75 and 92, 512 groups: 83 and 82), but for rows of
// a wavefront's lanes whose groups are not split (262144 x 128, a gate for each: 88,
// with it 93).
template <typename T, int N, int L, int MOST, int NP, bool ANY, int GATE>
__global__ __launch_bounds__(MOST) __attribute__((amdgpu_waves_per_eu(L && GATE != kSplit ? 2 : 4))) void
after_block_grad(GradArgs<T> a) {
    constexpr bool WHOLE = GATE == kWhole, OWN = GATE == kOwn, POST = GATE == kWhole || GATE == kSplit;
    __shared__ float buf[2][2][kMostWaves];
    __shared__ float lds[L ? MOST / 2 * NP * N : MOST < kRowBlock ? MOST * NP * N : 1];
    // rows under way in the workgroup (all of them take every step of the loops
    // together, for their sums' barriers; `active`: whether this one has a row)
    constexpr bool ONE = !L && MOST == kRowBlock;  // (one row)
    const int threads = L ? L : ONE ? int(blockDim.x) : a.threads;
    const int subs = L ? MOST / (L ? L : 1) : ONE ? 1 : int(blockDim.x) / threads;
    const int sub = ONE ? 0 : int(threadIdx.x) / threads, l = ONE ? int(threadIdx.x) : int(threadIdx.x) % threads;
    const int waves = threads / kWave, first = sub * waves;
    const int64_t d = a.d;
    const bool normed = a.rstd_post != nullptr;
    int turn = 0;
    Place at[NP];
    row_places<N>(l, threads, d, at);
    using P = Held<T, N, ANY>;
    struct Row {
        Vec<T, N> dy[NP], dh[NP], y[NP], b[NP];
        P gate[OWN ? NP : 1];
        float r1, r2;
    };
    // (without a gradient of y dh is read in its place, and not used; without a
    // norm of the block r2 in r1's)
    const T* dy = a.dy ? a.dy : a.dh;
    const int64_t ldy = a.dy ? a.ldy : a.ldh;
    const float* rstd_post = normed ? a.rstd_post : a.rstd_pre;
    auto load = [&](int64_t r) {
        Row q;
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            q.dh[k] = load_vec_nt<T, N>(column(a.dh + r * a.ldh, at[k].c));
            q.y[k] = load_vec_nt<T, N>(column(a.y + r * a.ldo, at[k].c));
            q.b[k] = load_vec_nt<T, N>(column(a.b + r * a.ldb, at[k].c));
            q.dy[k] = load_vec_nt<T, N>(column(dy + r * ldy, at[k].c));
            if constexpr (OWN) q.gate[k].load(a.gate.p, a.gate.wide, r * a.gate.ld + at[k].c, 1.f);
        }
        q.r1 = rstd_post[r];
        q.r2 = a.rstd_pre[r];
        return q;
    };
    // (whole: rows' threads take groups side by side; else the rows of one group)
    const int64_t walkers = WHOLE ? int64_t(gridDim.x) * subs : a.go.slots;
    const int64_t jstep = WHOLE ? 1 : a.go.parts * subs;
    const int64_t j0 = WHOLE ? 0 : blockIdx.x % a.go.parts * subs;
    const int64_t g0 = WHOLE ? int64_t(blockIdx.x) * subs : blockIdx.x / a.go.parts;
    // mul = scale post gate: of the group, or with a row's own gate of the row
    P post[NP], pre[NP];
    float mul[NP][N], sum_pre[NP][N] = {}, sum_s[NP][N] = {};
    float sum_post[POST ? NP : 1][N] = {};
#pragma unroll
    for (int k = 0; k < NP; ++k) {
        post[k].load(a.par.post, a.par.wide, at[k].c, 1.f);
        pre[k].load(a.par.pre, a.par.wide, at[k].c, 1.f);
    }
    for (int64_t g1 = g0; g1 < a.go.groups; g1 += walkers) {
        const int64_t gi = WHOLE && !ONE ? min(g1 + sub, a.go.groups - 1) : g1;
        const bool mine_too = !WHOLE || ONE || g1 + sub < a.go.groups;
        if constexpr (!OWN)
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                load_any<T, N>(a.gate.p, a.gate.wide, gi * a.gate.ld + at[k].c, 1.f, mul[k]);
#pragma unroll
                for (int i = 0; i < N; ++i) mul[k][i] *= a.scale * post[k].get(i);
            }
        for (int64_t j1 = j0; j1 < a.go.per; j1 += jstep, turn ^= 1) {
            const int64_t j = WHOLE || ONE ? j1 : j1 + sub;
            const bool active = ONE || (mine_too && j < a.go.per);
            const int64_t r = gi * a.go.per + (active ? j : a.go.per - 1);
            Row q = load(r);
            auto keep = [&] {
                if constexpr (sizeof(T) == 2 && N > 1)
#pragma unroll
                    for (int k = 0; k < NP; ++k) {
                        post[k].keep();
                        pre[k].keep();
                        keep_packed<T>(q.dh[k]);
                        keep_packed<T>(q.y[k]);
                        keep_packed<T>(q.b[k]);
                    }
            };
            const float r1 = normed ? q.r1 : 1.f;
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                if constexpr (OWN)
#pragma unroll
                    for (int i = 0; i < N; ++i) mul[k][i] = a.scale * q.gate[k].get(i) * post[k].get(i);
                if (active)
                    each_own<N>(at, k, [&](int i, bool mine) {
                        const float t = float(q.dh[k][i]) * float(q.y[k][i]);
                        sum_pre[k][i] = fmaf(t, q.r2, sum_pre[k][i]);
                        s = fmaf(mine ? t : 0.f, pre[k].get(i), s);
                    });
            }
            // Y = dy + r2 dh pre + y A, A = -r2^2 sum(a n2) / d
            const float A = -q.r2 * q.r2 * (q.r2 * rows_sum<L>(s, buf[turn][0], first, waves) / float(d));
            keep();
            float v[NP][N];
            s = 0.f;
#pragma unroll
            for (int k = 0; k < NP; ++k)
                each_own<N>(at, k, [&](int i, bool mine) {
                    const float Y = fmaf(float(q.dh[k][i]) * q.r2, pre[k].get(i),
                                         fmaf(float(q.y[k][i]), A, a.dy ? float(q.dy[k][i]) : 0.f));
                    v[k][i] = Y;
                    s = fmaf(mine ? Y * mul[k][i] : 0.f, float(q.b[k][i]), s);
                });
            // db = r1 c + b B, B = -r1^2 sum(c n1) / d
            const float B = normed ? -r1 * r1 * (r1 * rows_sum<L>(s, buf[turn][1], first, waves) / float(d)) : 0.f;
            keep();
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                if (!active) break;
                Vec<T, N> ox, ob;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float e = v[k][i] * r1, f = float(q.b[k][i]);
                    sum_s[k][i] = fmaf(OWN ? e * q.gate[OWN ? k : 0].get(i) : e, f, sum_s[k][i]);
                    ox[i] = T(v[k][i]);
                    ob[i] = T(fmaf(f, B, e * mul[k][i]));
                }
                if (at[k].shift >= N) break;
                store_vec_nt<T, N>(column(a.dx + r * a.lddx, at[k].c), ox);
                store_vec_nt<T, N>(column(a.db + r * a.lddb, at[k].c), ob);
                if constexpr (OWN) {
                    float dg[N];
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        dg[i] = v[k][i] * r1 * a.scale * float(q.b[k][i]) * post[k].get(i);
                    store_any<T, N>(a.dgate, a.gate.wide, r * a.lddg + at[k].c, dg);
                }
            }
        }
        if constexpr (!WHOLE) add_rows<L, MOST>(sum_s, lds, threads, subs);
        const bool write = WHOLE ? mine_too : sub == 0;
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            if (POST && write) {
                float g[N];
                load_any<T, N>(a.gate.p, a.gate.wide, gi * a.gate.ld + at[k].c, 1.f, g);
#pragma unroll
                for (int i = 0; i < N; ++i) sum_post[POST ? k : 0][i] = fmaf(sum_s[k][i], g[i], sum_post[POST ? k : 0][i]);
            }
            if (write && at[k].shift < N) {
                if (WHOLE || (POST && a.go.direct())) {
                    float dg[N];
#pragma unroll
                    for (int i = 0; i < N; ++i) dg[i] = a.scale * sum_s[k][i] * post[k].get(i);
                    store_any<T, N>(a.dgate, a.gate.wide, gi * a.lddg + at[k].c, dg);
                } else {
                    store_any<float, N>(a.sums.s + (gi * a.go.parts + blockIdx.x % a.go.parts) * d, true, at[k].c,
                                        sum_s[k]);
                }
            }
#pragma unroll
            for (int i = 0; i < N; ++i) sum_s[k][i] = 0.f;
        }
    }
    add_rows<L, MOST>(sum_pre, lds, threads, subs);
    if constexpr (WHOLE) add_rows<L, MOST>(sum_post, lds, threads, subs);
    if (sub > 0) return;
#pragma unroll
    for (int k = 0; k < NP; ++k) {
        if (at[k].shift >= N) break;
        store_any<float, N>(a.sums.pre + int64_t(blockIdx.x) * d, true, at[k].c, sum_pre[k]);
        if constexpr (POST) store_any<float, N>(a.sums.post + int64_t(blockIdx.x) * d, true, at[k].c, sum_post[k]);
    }
}

// rows too long for registers: dx and db by three readings; m2: the rows' sum(a n2) / d
template <typename T>
__global__ __launch_bounds__(kRowBlock) void after_block_grad_long(GradArgs<T> a, float* __restrict__ means) {
    constexpr int N = 16 / int(sizeof(T));
    constexpr int64_t STEP = int64_t(kRowBlock) * N;
    __shared__ float buf[2][2][kMostWaves];
    const bool normed = a.rstd_post != nullptr;
    int turn = 0;
    for (int64_t r = blockIdx.x; r < a.m; r += gridDim.x, turn ^= 1) {
        const float r1 = normed ? a.rstd_post[r] : 1.f, r2 = a.rstd_pre[r];
        const int64_t at_gate = gate_row(a.gate, r) * a.gate.ld;
        float s = 0.f;
        for (int64_t c = int64_t(threadIdx.x) * N; c < a.d; c += STEP) {
            const Place at = place<N>(c, a.d);
            const Vec<T, N> dh = load_vec<T, N>(a.dh + r * a.ldh + at.c), y = load_vec<T, N>(a.y + r * a.ldo + at.c);
            float pre[N];
            load_any<T, N>(a.par.pre, a.par.wide, at.c, 1.f, pre);
#pragma unroll
            for (int i = 0; i < N; ++i)
                s = i >= at.shift ? fmaf(float(dh[i]) * pre[i], float(y[i]) * r2, s) : s;
        }
        const float m2 = row_sum<0>(s, buf[turn][0]) / float(a.d);
        if (threadIdx.x == 0) means[r] = m2;
        auto grads_at = [&](int c, float (&Y)[N], float (&cc)[N], float (&n1)[N], float (&dg)[N]) {
            const Vec<T, N> dh = load_vec<T, N>(a.dh + r * a.ldh + c), y = load_vec<T, N>(a.y + r * a.ldo + c),
                            b = load_vec<T, N>(a.b + r * a.ldb + c);
            float pre[N], post[N], g[N], dy[N];
            load_any<T, N>(a.par.pre, a.par.wide, c, 1.f, pre);
            load_any<T, N>(a.par.post, a.par.wide, c, 1.f, post);
            load_any<T, N>(a.gate.p, a.gate.wide, at_gate + c, 1.f, g);
            load_any<T, N>(a.dy, false, r * a.ldy + c, 0.f, dy);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                Y[i] = fmaf(r2, fmaf(float(dh[i]), pre[i], -float(y[i]) * r2 * m2), dy[i]);
                n1[i] = float(b[i]) * r1;
                cc[i] = a.scale * Y[i] * g[i] * post[i];
                dg[i] = a.scale * Y[i] * n1[i] * post[i];
            }
        };
        s = 0.f;
        float Y[N], cc[N], n1[N], dg[N];
        if (normed)
            for (int64_t c = int64_t(threadIdx.x) * N; c < a.d; c += STEP) {
                const Place at = place<N>(c, a.d);
                grads_at(at.c, Y, cc, n1, dg);
#pragma unroll
                for (int i = 0; i < N; ++i) s = i >= at.shift ? fmaf(cc[i], n1[i], s) : s;
            }
        const float m1 = normed ? row_sum<0>(s, buf[turn][1]) / float(a.d) : 0.f;
        for (int64_t c = int64_t(threadIdx.x) * N; c < a.d; c += STEP) {
            const Place at = place<N>(c, a.d);
            grads_at(at.c, Y, cc, n1, dg);
            Vec<T, N> ox, ob;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                ox[i] = T(Y[i]);
                ob[i] = T(r1 * fmaf(-n1[i], m1, cc[i]));
            }
            if (a.gate.own) store_any<T, N>(a.dgate, a.gate.wide, r * a.lddg + at.c, dg);
            store_vec_nt<T, N>(a.dx + r * a.lddx + at.c, ox);
            store_vec_nt<T, N>(a.db + r * a.lddb + at.c, ob);
        }
    }
}

// The sums of long rows: workgroup (x, y) takes a pack of columns per lane of
// the groups and parts that y stands for, its wavefronts in turn.
template <typename T, bool SEVERAL>
__global__ __launch_bounds__(kBlock) void after_block_sums_long(GradArgs<T> a, const float* __restrict__ means) {
    constexpr int N = 16 / int(sizeof(T));
    __shared__ float lds[kWavesPerBlock][kWave][N];
    const int w = threadIdx.x / kWave, l = lane_id();
    const Place at = place<N>((int64_t(blockIdx.x) * kWave + l) * N, a.d);
    const bool normed = a.rstd_post != nullptr;
    float post[N], pre[N], sum_pre[N] = {}, sum_post[N] = {};
    load_any<T, N>(a.par.post, a.par.wide, at.c, 1.f, post);
    load_any<T, N>(a.par.pre, a.par.wide, at.c, 1.f, pre);
    // (the wavefronts' sums in their order; complete in the first one)
    auto add = [&](float (&v)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i) lds[w][l][i] = v[i];
        __syncthreads();
        if (w == 0)
            for (int q = 1; q < kWavesPerBlock; ++q)
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] += lds[q][l][i];
        __syncthreads();
    };
    const int64_t part = blockIdx.y % a.go.parts;
    for (int64_t gi = blockIdx.y / a.go.parts; gi < a.go.groups; gi += a.go.slots) {
        float sum_s[N] = {}, g[N];
        load_any<T, N>(a.gate.own ? nullptr : a.gate.p, a.gate.wide, gi * a.gate.ld + at.c, 1.f, g);
        for (int64_t j = part * kWavesPerBlock + w; j < a.go.per; j += a.go.parts * kWavesPerBlock) {
            const int64_t r = gi * a.go.per + j;
            const float r1 = normed ? a.rstd_post[r] : 1.f, r2 = a.rstd_pre[r], m2 = means[r];
            const Vec<T, N> dh = load_vec<T, N>(a.dh + r * a.ldh + at.c), y = load_vec<T, N>(a.y + r * a.ldo + at.c),
                            b = load_vec<T, N>(a.b + r * a.ldb + at.c);
            float dy[N], k[N];
            load_any<T, N>(a.dy, false, r * a.ldy + at.c, 0.f, dy);
            load_any<T, N>(a.gate.own ? a.gate.p : nullptr, a.gate.wide, r * a.gate.ld + at.c, 1.f, k);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float n2 = float(y[i]) * r2;
                const float Y = fmaf(r2, fmaf(float(dh[i]), pre[i], -n2 * m2), dy[i]);
                sum_pre[i] = fmaf(float(dh[i]), n2, sum_pre[i]);
                sum_s[i] = fmaf(Y * float(b[i]) * r1, k[i], sum_s[i]);
            }
        }
        add(sum_s);
        if (w == 0 && at.shift < N) {
            if constexpr (SEVERAL)
#pragma unroll
                for (int i = 0; i < N; ++i) sum_post[i] = fmaf(sum_s[i], g[i], sum_post[i]);
            if (SEVERAL && a.go.direct()) {
                float dg[N];
#pragma unroll
                for (int i = 0; i < N; ++i) dg[i] = a.scale * sum_s[i] * post[i];
                store_any<T, N>(a.dgate, a.gate.wide, gi * a.lddg + at.c, dg);
            } else {
                store_any<float, N>(a.sums.s + (gi * a.go.parts + part) * a.d, true, at.c, sum_s);
            }
        }
    }
    add(sum_pre);
    if (w > 0 || at.shift >= N) return;
    store_any<float, N>(a.sums.pre + int64_t(blockIdx.y) * a.d, true, at.c, sum_pre);
    if constexpr (SEVERAL) store_any<float, N>(a.sums.post + int64_t(blockIdx.y) * a.d, true, at.c, sum_post);
}

// The parts added up.  A workgroup takes some columns of dpre, of dpost (and of the
// gate, if that is one row) or of a row of the gate, many parts of them side by
// side: each in its order, then those sums pairwise.  16 columns instead of 64 where
// few would leave most of the chip idle (512 parts of 1001 columns: 4.4 us and 4.9; of
// 4096: 9.6 and 5.8); kGateColumns of a gate's row that has few parts (16384 x 4096, 64
// rows of the gate, 8 parts each: 161 us in all, 178 by 64 columns).
constexpr int kJoinBlock = 1024, kGateColumns = 256;
inline __host__ __device__ int gate_columns(int64_t parts, int columns) { return parts < 16 ? kGateColumns : columns; }

// the sum of `count` rows of d at column c0 + threadIdx.x % COLUMNS, for the first COLUMNS threads
template <int COLUMNS>
__device__ inline float join_columns(const float* from, int64_t count, int64_t d, int64_t c0, float* lds) {
    constexpr int W = kJoinBlock / COLUMNS;  // parts under way
    const int w = threadIdx.x / COLUMNS;
    const int64_t c = c0 + threadIdx.x % COLUMNS;
    float s = 0.f;
    if (c < d)
#pragma unroll 8
        for (int64_t q = w; q < count; q += W) s += from[q * d + c];
    lds[threadIdx.x] = s;
    __syncthreads();
#pragma unroll
    for (int half = W / 2; half > 0; half /= 2) {
        if (w < half) lds[threadIdx.x] += lds[threadIdx.x + half * COLUMNS];
        __syncthreads();
    }
    s = lds[threadIdx.x % COLUMNS];
    __syncthreads();
    return s;
}

template <typename T, int COLUMNS>
__global__ __launch_bounds__(kJoinBlock) void join_sums(Sums sums, Spread go, int64_t gate_rows, int64_t d,
                                                        BlockGate gate, BlockParams par, float scale, void* dpre,
                                                        void* dpost, void* dgate, int64_t lddg) {
    __shared__ float lds[kJoinBlock];
    const bool one = go.groups == 1;
    const int64_t across = (d + COLUMNS - 1) / COLUMNS, wide = gate_columns(go.parts, COLUMNS),
                  gate_across = (d + wide - 1) / wide;
    for (int64_t b = blockIdx.x; b < 2 * across + gate_rows * gate_across; b += gridDim.x) {
        float v[1], k[1];
        if (b < across) {
            if (!dpre) continue;
            const int64_t c0 = b * COLUMNS, c = c0 + threadIdx.x;
            v[0] = join_columns<COLUMNS>(sums.pre, go.grid(), d, c0, lds);
            if (threadIdx.x < COLUMNS && c < d) store_any<T, 1>(dpre, par.wide, c, v);
        } else if (b < 2 * across) {
            const bool gated = one && gate.p && !gate.own;
            if (!dpost && !gated) continue;
            const int64_t c0 = (b - across) * COLUMNS, c = c0 + threadIdx.x;
            const float S = scale * join_columns<COLUMNS>(one ? sums.s : sums.post, one ? go.parts : go.grid(), d, c0, lds);
            if (threadIdx.x < COLUMNS && c < d) {
                load_any<T, 1>(gated ? gate.p : nullptr, gate.wide, c, 1.f, k);
                v[0] = S * k[0];
                if (dpost) store_any<T, 1>(dpost, par.wide, c, v);
                load_any<T, 1>(par.post, par.wide, c, 1.f, k);
                v[0] = S * k[0];
                if (gated) store_any<T, 1>(dgate, gate.wide, c, v);
            }
        } else {
            const int64_t gi = (b - 2 * across) / gate_across;
            const int64_t c0 = (b - 2 * across) % gate_across * wide, c = c0 + threadIdx.x;
            const float* from = sums.s + gi * go.parts * d;
            v[0] = wide == COLUMNS ? join_columns<COLUMNS>(from, go.parts, d, c0, lds)
                                   : join_columns<kGateColumns>(from, go.parts, d, c0, lds);
            if (threadIdx.x < wide && c < d) {
                load_any<T, 1>(par.post, par.wide, c, 1.f, k);
                v[0] *= scale * k[0];
                store_any<T, 1>(dgate, gate.wide, gi * lddg + c, v);
            }
        }
    }
}

// Lanes of a wavefront for up to 64 packs, else a workgroup's threads, one pack
// each (two of four columns past 1024): the gradient's thread holds four inputs,
// three parameters and up to three sums for each of its columns, and has no
// registers for more.  Rows of more than 8192 columns are read again (np 0), by the
// forward pass too, which goes by the gradient's shapes (4096 x 16384 bf16, one gate:
// forward 128 us, 4.2 TB/s of what has to move, and gradient 341, 2.4; as many elements
// in rows of 8192: 96, 5.6 TB/s, and 176, 4.6).
inline RowShape block_shape(int64_t d, int dt) {
    const int64_t packs = packs_of(d, dt);
    if (packs <= kWave) {
        int lanes = 4;
        while (lanes < packs) lanes *= 2;
        return {lanes, lanes, 1};
    }
    const int np = packs <= kRowBlock ? 1 : 2;
    const int64_t threads = ceil_div(ceil_div(packs, np), kWave) * kWave;
    if (threads > kRowBlock || (np == 2 && dt != kDtF32)) return {0, 0, 0};
    return {0, int(threads), np};
}

// f(lanes, threads a workgroup can have, packs per thread) of a shape, as constants
template <typename T, int N, int LANES_BLOCK, typename F>
inline void by_block_shape(const RowShape& s, F f) {
    using std::integral_constant;
    const integral_constant<int, 1> one;
    auto lanes = [&](auto l) { f(l, integral_constant<int, LANES_BLOCK>(), one); };
    if (s.lanes == 4) return lanes(integral_constant<int, 4>());
    if (s.lanes == 8) return lanes(integral_constant<int, 8>());
    if constexpr (N > 1) {
        if (s.lanes == 16) return lanes(integral_constant<int, 16>());
        if (s.lanes == 32) return lanes(integral_constant<int, 32>());
        if (s.lanes) return lanes(integral_constant<int, kWave>());
        const integral_constant<int, 0> none;
        const integral_constant<int, kRowBlock> all;
        if (s.threads <= kGradBlock) return f(none, integral_constant<int, kGradBlock>(), one);
        if constexpr (sizeof(T) == 4)
            if (s.np == 2) return f(none, all, integral_constant<int, 2>());
        f(none, all, one);
    }
}

// Rows that a workgroup of the gradient has under way, and workgroups: 16
// wavefronts on a compute unit, as few workgroups as that takes, since each leaves
// sums of d floats (8191 x 1001: 29 us, with half as many workgroups 36, with twice
// as many 36; 8192 x 4096: 80, 103 and 87; but 262144 x 128: 83, 74 and 78).
inline int grad_rows(const RowShape& s) {
    return s.lanes ? kGradBlock / s.lanes : s.threads && s.threads <= kGradBlock ? kGradBlock / s.threads : 1;
}
constexpr int64_t kLongParts = 64;
Spread spread_of(int64_t m, int64_t groups, const RowShape& s) {
    Spread go;
    go.groups = groups;
    go.per = m / groups;
    const int rows = s.np ? grad_rows(s) : 1;
    const int64_t room = !s.np ? kLongParts : s.threads > kGradBlock ? kCus : 2 * kCus;
    // Groups of fewer rows than a workgroup takes side by side go whole to a row's
    // threads each, if they are so many that the workgroups would take longer by
    // turns (262144 x 128: of 16 rows 101 us, split 130; of 2 rows 81 and 728; of 32
    // rows, which fill a workgroup, 81 split and 105 whole).
    if (rows > 1 && m > 0 && go.per < rows && go.per * room < 2 * groups) {
        go.whole = true;
        go.slots = std::min(room, ceil_div(groups, rows));
        return go;
    }
    go.slots = std::min(groups, room);
    const int64_t most = std::max<int64_t>(1, ceil_div(go.per, s.np ? rows : kWavesPerBlock));
    go.parts = std::min(most, std::max<int64_t>(1, room / go.slots));
    return go;
}

// f(whether a parameter or the gate is of another type than the rows)
template <typename T, typename F>
inline void by_types(const BlockGate& gate, const BlockParams& par, F f) {
    if constexpr (sizeof(T) == 2)
        if (((par.post || par.pre) && par.wide) || (gate.p && gate.wide)) return f(std::integral_constant<bool, true>());
    f(std::integral_constant<bool, false>());
}

int64_t groups_of(const BlockGate& gate) { return gate.p && !gate.own ? gate.rows : 1; }

}  // namespace

void block_norm(const DenseRows& X, const DenseRows& B, const BlockGate& gate, float scale, const BlockParams& par,
                bool normed, float eps, const DenseRows& Y, const DenseRows& H, float* rstd_post, float* rstd_pre,
                hipStream_t s) {
    const RowShape shape = block_shape(X.n, X.dt);
    by_width(X.dt, X.n, [&](auto e, auto n) {
        using T = decltype(e);
        constexpr int N = decltype(n)::value;
        const int64_t m = X.m, d = X.n;
        const T *x = static_cast<const T*>(X.p), *b = static_cast<const T*>(B.p);
        T *y = static_cast<T*>(Y.p), *h = static_cast<T*>(H.p);
        if (!shape.np) {
            if constexpr (N > 1)
                after_block_long<T><<<row_grid(m), kRowBlock, 0, s>>>(x, X.ld, b, B.ld, m, d, gate, scale, par, normed,
                                                                     eps, y, Y.ld, h, H.ld, rstd_post, rstd_pre);
            return;
        }
        by_block_shape<T, N, kBlock>(shape, [&](auto lanes, auto most, auto np) {
            constexpr int L = decltype(lanes)::value, MOST = decltype(most)::value, NP = decltype(np)::value;
            const int threads = L ? MOST : shape.threads;
            const int64_t blocks = L ? ceil_div(m, MOST / (L ? L : 1)) : m;
            const unsigned grid = unsigned(std::min<int64_t>(blocks, kCus * std::max(1, 1024 / threads)));
            by_types<T>(gate, par, [&](auto any) {
                auto launch = [&](auto own_gate) {
                    after_block<T, N, L, MOST, NP, decltype(any)::value, decltype(own_gate)::value>
                        <<<grid, threads, 0, s>>>(x, X.ld, b, B.ld, m, d, gate, scale, par, normed, eps, y, Y.ld, h,
                                                  H.ld, rstd_post, rstd_pre);
                };
                if (gate.own)
                    launch(std::integral_constant<bool, true>());
                else
                    launch(std::integral_constant<bool, false>());
            });
        });
    });
}

size_t block_norm_grad_tmp_bytes(int64_t m, int64_t d, int dt, const BlockGate& gate) {
    const RowShape shape = block_shape(d, dt);
    const Spread go = spread_of(m, groups_of(gate), shape);
    return size_t((go.grid() + post_rows(go) + s_rows(go)) * d + (shape.np ? 0 : m)) * sizeof(float);
}

void block_norm_grad(const DenseRows& DY, const DenseRows& DH, const DenseRows& Y, const DenseRows& B,
                     const float* rstd_post, const float* rstd_pre, const BlockGate& gate, float scale,
                     const BlockParams& par, const DenseRows& DX, const DenseRows& DB, void* dgate, int64_t lddg,
                     void* dpost, void* dpre, void* tmp, hipStream_t s) {
    const RowShape shape = block_shape(Y.n, Y.dt);
    const int64_t m = Y.m, d = Y.n;
    const Spread go = spread_of(m, groups_of(gate), shape);
    Sums sums;
    sums.pre = static_cast<float*>(tmp);
    sums.post = sums.pre + go.grid() * d;
    sums.s = sums.post + post_rows(go) * d;
    float* means = sums.s + s_rows(go) * d;
    by_width(Y.dt, d, [&](auto e, auto n) {
        using T = decltype(e);
        constexpr int N = decltype(n)::value;
        auto in = [](const DenseRows& r) { return static_cast<const T*>(r.p); };
        GradArgs<T> a;
        a.dy = in(DY);
        a.dh = in(DH);
        a.y = in(Y);
        a.b = in(B);
        a.ldy = DY.ld;
        a.ldh = DH.ld;
        a.ldo = Y.ld;
        a.ldb = B.ld;
        a.m = m;
        a.d = d;
        a.threads = shape.threads;
        a.rstd_post = rstd_post;
        a.rstd_pre = rstd_pre;
        a.gate = gate;
        a.par = par;
        a.scale = scale;
        a.dx = static_cast<T*>(DX.p);
        a.db = static_cast<T*>(DB.p);
        a.lddx = DX.ld;
        a.lddb = DB.ld;
        a.dgate = dgate;
        a.lddg = lddg;
        a.sums = sums;
        a.go = go;
        using std::integral_constant;
        if (m > 0 && shape.np) {
            by_block_shape<T, N, kGradBlock>(shape, [&](auto lanes, auto most, auto np) {
                constexpr int L = decltype(lanes)::value, MOST = decltype(most)::value, NP = decltype(np)::value;
                by_types<T>(gate, par, [&](auto any) {
                    auto launch = [&](auto how) {
                        after_block_grad<T, N, L, MOST, NP, decltype(any)::value, decltype(how)::value>
                            <<<unsigned(go.grid()), L ? MOST : shape.threads * grad_rows(shape), 0, s>>>(a);
                    };
                    if constexpr (MOST == kGradBlock)  // (past it no rows side by side)
                        if (go.whole) return launch(integral_constant<int, kWhole>());
                    if (gate.p && gate.own)
                        launch(integral_constant<int, kOwn>());
                    else if (go.groups > 1)
                        launch(integral_constant<int, kSplit>());
                    else
                        launch(integral_constant<int, kOne>());
                });
            });
        } else if (m > 0) {
            if constexpr (N > 1) {
                after_block_grad_long<T><<<row_grid(m), kRowBlock, 0, s>>>(a, means);
                auto launch = [&](auto several) {
                    after_block_sums_long<T, decltype(several)::value>
                        <<<dim3(unsigned(ceil_div(packs_of(d, Y.dt), kWave)), unsigned(go.grid())), kBlock, 0, s>>>(
                            a, means);
                };
                if (go.groups > 1)
                    launch(integral_constant<bool, true>());
                else
                    launch(integral_constant<bool, false>());
            }
        }
        const int64_t gate_rows = go.groups > 1 && !(m > 0 && go.direct()) ? go.groups : 0;
        Spread add = go;
        if (m == 0) add.parts = 0;  // (of no rows: zeros)
        auto join = [&](auto columns) {
            constexpr int COLUMNS = decltype(columns)::value;
            const int64_t blocks = 2 * ceil_div(d, COLUMNS) + gate_rows * ceil_div(d, gate_columns(add.parts, COLUMNS));
            join_sums<T, COLUMNS><<<row_grid(blocks), kJoinBlock, 0, s>>>(sums, add, gate_rows, d, gate, par, scale, dpre,
                                                                         dpost, dgate, lddg);
        };
        if (ceil_div(d, 64) >= kCus / 4)
            join(integral_constant<int, 64>());
        else
            join(integral_constant<int, 16>());
    });
}

}  // namespace spsyrk
