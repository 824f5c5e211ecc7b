// The norms before and after a block, with its gate and residual scale, and
// their gradient.
//
//     u = b r1 post,  r1 = 1 / sqrt(sum b^2 / d + eps)   (or u = b),
//     y = x + s gate u,  h = y r2 pre,  r2 = 1 / sqrt(sum y^2 / d + eps);
//     n2 = y r2,  a = dh pre,  Y = dy + r2 (a - n2 sum(a n2) / d),  dx = Y,
//     n1 = b r1,  c = s gate Y post,  db = r1 (c - n1 sum(c n1) / d)   (or s gate Y),
//     dpre = sum over rows of dh n2,  S = sum over rows of s Y n1,
//     dgate = post S,  dpost = gate S.
//
// Bound by the bytes of the rows: x and b (the gradient: dy, dh, y, b) are read
// once, y and h (dx and db) written once, in one launch, a row in registers in
// between as in the layer norm.  The rows that share a row of the gate share S,
// so its gradient and that of post are one sum, told apart when the workgroups'
// parts are added up, in their order, by a second launch.  A gate of a row's own
// has its gradient written with the row.  y is rounded when it is stored; h and
// r2 come from the sum before that.
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

// N elements of either type that are loaded now and converted when they are used
template <typename T, int N>
struct Later {
    Vec<T, N> narrow;
    Vec<float, N> wide;
    __device__ void load(const void* p, bool f32, int64_t i) {
        if (f32)
            wide = load_vec<float, N>(static_cast<const float*>(p) + i);
        else
            narrow = load_vec<T, N>(static_cast<const T*>(p) + i);
    }
    __device__ void get(bool f32, float (&out)[N]) const {
#pragma unroll
        for (int k = 0; k < N; ++k) out[k] = f32 ? wide[k] : float(narrow[k]);
    }
};

// a row's own gate, or one that `per` rows share
__device__ inline int64_t gate_row(const BlockGate& g, int64_t r) {
    return g.own ? r : int64_t(uint32_t(r) / uint32_t(g.per));
}

template <typename T, int N, int L, int MOST, int NP>
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
    struct Row {
        Vec<T, N> x[NP], b[NP];
        Later<T, N> gate[NP];
    };
    auto load = [&](int64_t r) {
        Row q;
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            q.x[k] = load_vec_nt<T, N>(x + r * ldx + at[k].c);
            q.b[k] = load_vec_nt<T, N>(b + r * ldb + at[k].c);
        }
        if (gate.own)
#pragma unroll
            for (int k = 0; k < NP; ++k) q.gate[k].load(gate.p, gate.wide, r * gate.ld + at[k].c);
        return q;
    };
    const int64_t step = int64_t(gridDim.x) * ROWS;
    int64_t r = int64_t(blockIdx.x) * ROWS + (L ? threadIdx.x / (L ? L : 1) : 0);
    Row next;
    if (r < m) next = load(r);
    float post[NP][N], pre[NP][N], g[NP][N];
#pragma unroll
    for (int k = 0; k < NP; ++k) {
        load_any<T, N>(par.post, par.wide, at[k].c, 1.f, post[k]);
        load_any<T, N>(par.pre, par.wide, at[k].c, 1.f, pre[k]);
    }
    int64_t held = -1;  // the row of the gate that g has
    for (; r < m; r += step, turn ^= 1) {
        const Row q = next;
        if (r + step < m) next = load(r + step);
        if (!gate.own) {
            const int64_t want = gate_row(gate, r);
            if (want != held) {
                held = want;
#pragma unroll
                for (int k = 0; k < NP; ++k) load_any<T, N>(gate.p, gate.wide, want * gate.ld + at[k].c, 1.f, g[k]);
            }
        }
        float r1 = 1.f;
        if (normed) {
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < NP; ++k)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float z = own(at, k, i) ? float(q.b[k][i]) : 0.f;
                    s = fmaf(z, z, s);
                }
            r1 = 1.f / sqrtf(row_sum<L>(s, buf[turn][0]) / float(d) + eps);
            if (l == 0) rstd_post[r] = r1;
        }
        const float f = r1 * scale;
        float v[NP][N], s = 0.f;
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            if (gate.own) q.gate[k].get(gate.wide, g[k]);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[k][i] = fmaf(float(q.b[k][i]) * post[k][i], g[k][i] * f, float(q.x[k][i]));
                const float z = own(at, k, i) ? v[k][i] : 0.f;
                s = fmaf(z, z, s);
            }
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
                oh[i] = T(v[k][i] * r2 * pre[k][i]);
            }
            store_vec_nt<T, N>(y + r * ldy + at[k].c, oy);
            store_vec_nt<T, N>(h + r * ldh + at[k].c, oh);
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
};

// workspace: the workgroups' sums of dh n2, then of S (split groups: one of each
// part of a group; whole groups: a workgroup's sums of gate S)
struct Sums {
    float* pre = nullptr;
    float* s = nullptr;
};

template <typename T>
struct GradArgs {
    const T *dy, *dh, *y, *b;
    int64_t ldy, ldh, ldo, ldb;
    int64_t m, d;
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

// the sums of a workgroup's rows: lanes' groups by lane distance, wavefronts
// pairwise through LDS; complete in the first L lanes of the first wavefront
template <int L, int WAVES, int N, int NP>
__device__ inline void add_rows(float (&v)[NP][N], float* lds) {
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
}

template <typename T, int N, int L, int MOST, int NP, bool WHOLE>
__global__ __launch_bounds__(MOST) void after_block_grad(GradArgs<T> a) {
    constexpr int ROWS = L ? MOST / (L ? L : 1) : 1, WAVES = MOST / kWave;
    __shared__ float buf[2][2][kMostWaves];
    __shared__ float lds[ROWS > 1 ? WAVES / 2 * NP * N * kWave : 1];
    const int threads = L ? L : int(blockDim.x), l = L ? int(threadIdx.x) % (L ? L : 1) : int(threadIdx.x);
    const int sub = L ? int(threadIdx.x) / (L ? L : 1) : 0;
    const int64_t d = a.d;
    const bool normed = a.rstd_post != nullptr;
    int turn = 0;
    Place at[NP];
    row_places<N>(l, threads, d, at);
    struct Row {
        Vec<T, N> dy[NP], dh[NP], y[NP], b[NP];
        Later<T, N> gate[NP];
        float r1, r2;
    };
    auto load = [&](int64_t r) {
        Row q;
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            q.dh[k] = load_vec_nt<T, N>(a.dh + r * a.ldh + at[k].c);
            q.y[k] = load_vec_nt<T, N>(a.y + r * a.ldo + at[k].c);
            q.b[k] = load_vec_nt<T, N>(a.b + r * a.ldb + at[k].c);
        }
        if (a.dy)
#pragma unroll
            for (int k = 0; k < NP; ++k) q.dy[k] = load_vec_nt<T, N>(a.dy + r * a.ldy + at[k].c);
        if (a.gate.own)
#pragma unroll
            for (int k = 0; k < NP; ++k) q.gate[k].load(a.gate.p, a.gate.wide, r * a.gate.ld + at[k].c);
        q.r1 = normed ? a.rstd_post[r] : 1.f;
        q.r2 = a.rstd_pre[r];
        return q;
    };
    // the rows of this row's threads: j-th of group gi
    const int64_t walkers = WHOLE ? int64_t(gridDim.x) * ROWS : a.go.slots;
    const int64_t jstep = WHOLE ? 1 : a.go.parts * ROWS;
    const int64_t j0 = WHOLE ? 0 : blockIdx.x % a.go.parts * ROWS + sub;
    const int64_t g0 = WHOLE ? int64_t(blockIdx.x) * ROWS + sub : blockIdx.x / a.go.parts;
    auto row_of = [&](int64_t gi, int64_t j) { return gi * a.go.per + j; };
    constexpr bool AHEAD = MOST < kRowBlock;  // (a row ahead, but where its registers would spill)
    Row next;
    if (AHEAD && g0 < a.go.groups && j0 < a.go.per) next = load(row_of(g0, j0));

    float post[NP][N], pre[NP][N], g[NP][N], sum_pre[NP][N] = {}, sum_s[NP][N] = {};
    float sum_post[WHOLE ? NP : 1][N] = {};
#pragma unroll
    for (int k = 0; k < NP; ++k) {
        load_any<T, N>(a.par.post, a.par.wide, at[k].c, 1.f, post[k]);
        load_any<T, N>(a.par.pre, a.par.wide, at[k].c, 1.f, pre[k]);
    }
    for (int64_t gi = g0; gi < a.go.groups; gi += walkers) {
        if (!a.gate.own)
#pragma unroll
            for (int k = 0; k < NP; ++k)
                load_any<T, N>(a.gate.p, a.gate.wide, gi * a.gate.ld + at[k].c, 1.f, g[k]);
        for (int64_t j = j0; j < a.go.per; j += jstep, turn ^= 1) {
            const int64_t r = row_of(gi, j);
            const Row q = AHEAD ? next : load(r);
            if (AHEAD) {
                // (the next one of this group, or the first of the next group)
                if (j + jstep < a.go.per)
                    next = load(row_of(gi, j + jstep));
                else if (gi + walkers < a.go.groups)
                    next = load(row_of(gi + walkers, j0));
            }
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < NP; ++k)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float w = float(q.dh[k][i]), n2 = float(q.y[k][i]) * q.r2;
                    sum_pre[k][i] = fmaf(w, n2, sum_pre[k][i]);
                    s = fmaf(own(at, k, i) ? w * pre[k][i] : 0.f, n2, s);
                }
            const float m2 = row_sum<L>(s, buf[turn][0]) / float(d);
            float v[NP][N];
            s = 0.f;
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                if (a.gate.own) q.gate[k].get(a.gate.wide, g[k]);
                float dg[N];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float n2 = float(q.y[k][i]) * q.r2, n1 = float(q.b[k][i]) * q.r1;
                    const float Y = fmaf(q.r2, fmaf(float(q.dh[k][i]), pre[k][i], -n2 * m2),
                                         a.dy ? float(q.dy[k][i]) : 0.f);
                    const float sy = a.scale * Y, t = sy * n1;
                    dg[i] = t * post[k][i];
                    sum_s[k][i] = fmaf(t, a.gate.own ? g[k][i] : 1.f, sum_s[k][i]);
                    const float c = sy * g[k][i] * post[k][i];
                    s = fmaf(own(at, k, i) ? c : 0.f, n1, s);
                    v[k][i] = Y;
                }
                if (a.gate.own && at[k].shift < N)
                    store_any<T, N>(a.dgate, a.gate.wide, r * a.lddg + at[k].c, dg);
            }
            const float m1 = normed ? row_sum<L>(s, buf[turn][1]) / float(d) : 0.f;
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                if (at[k].shift >= N) break;
                Vec<T, N> ox, ob;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float c = a.scale * v[k][i] * g[k][i] * post[k][i], n1 = float(q.b[k][i]) * q.r1;
                    ox[i] = T(v[k][i]);
                    ob[i] = T(q.r1 * fmaf(-n1, m1, c));
                }
                store_vec_nt<T, N>(a.dx + r * a.lddx + at[k].c, ox);
                store_vec_nt<T, N>(a.db + r * a.lddb + at[k].c, ob);
            }
        }
        if constexpr (WHOLE) {
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                float dg[N];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    dg[i] = sum_s[k][i] * post[k][i];
                    sum_post[k][i] = fmaf(sum_s[k][i], g[k][i], sum_post[k][i]);
                    sum_s[k][i] = 0.f;
                }
                if (at[k].shift < N) store_any<T, N>(a.dgate, a.gate.wide, gi * a.lddg + at[k].c, dg);
            }
        } else {
            if constexpr (ROWS > 1) add_rows<L, WAVES>(sum_s, lds);
            if (ROWS == 1 || int(threadIdx.x) < L) {
                float* p = a.sums.s + (gi * a.go.parts + blockIdx.x % a.go.parts) * d;
#pragma unroll
                for (int k = 0; k < NP; ++k)
                    if (at[k].shift < N) store_any<float, N>(p, true, at[k].c, sum_s[k]);
            }
#pragma unroll
            for (int k = 0; k < NP; ++k)
#pragma unroll
                for (int i = 0; i < N; ++i) sum_s[k][i] = 0.f;
        }
    }
    if constexpr (ROWS > 1) {
        add_rows<L, WAVES>(sum_pre, lds);
        if constexpr (WHOLE) add_rows<L, WAVES>(sum_post, lds);
        if (int(threadIdx.x) >= L) return;
    }
#pragma unroll
    for (int k = 0; k < NP; ++k) {
        if (at[k].shift >= N) break;
        store_any<float, N>(a.sums.pre + int64_t(blockIdx.x) * d, true, at[k].c, sum_pre[k]);
        if constexpr (WHOLE) store_any<float, N>(a.sums.s + int64_t(blockIdx.x) * d, true, at[k].c, sum_post[k]);
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
template <typename T, bool WHOLE>
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
                sum_s[i] = fmaf(a.scale * Y * float(b[i]) * r1, k[i], sum_s[i]);
            }
        }
        add(sum_s);
        if (w == 0 && at.shift < N) {
            if constexpr (WHOLE) {
                float dg[N];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    dg[i] = sum_s[i] * post[i];
                    sum_post[i] = fmaf(sum_s[i], g[i], sum_post[i]);
                }
                store_any<T, N>(a.dgate, a.gate.wide, gi * a.lddg + at.c, dg);
            } else {
                store_any<float, N>(a.sums.s + (gi * a.go.parts + part) * a.d, true, at.c, sum_s);
            }
        }
    }
    add(sum_pre);
    if (w > 0 || at.shift >= N) return;
    store_any<float, N>(a.sums.pre + int64_t(blockIdx.y) * a.d, true, at.c, sum_pre);
    if constexpr (WHOLE) store_any<float, N>(a.sums.s + int64_t(blockIdx.y) * a.d, true, at.c, sum_post);
}

// The parts added up: dpre (item 0), dpost (1) and the gate's rows (2 and on),
// parts in their order within a wavefront, the wavefronts in theirs.
constexpr int kJoinBlock = 1024;
template <typename T>
__global__ __launch_bounds__(kJoinBlock) void join_sums(Sums sums, Spread go, int64_t items, int64_t d, BlockGate gate,
                                                        BlockParams par, void* dpre, void* dpost, void* dgate,
                                                        int64_t lddg) {
    constexpr int W = kJoinBlock / kWave;
    __shared__ float lds[W][kWave];
    const int w = threadIdx.x / kWave, l = lane_id();
    for (int64_t item = blockIdx.y; item < items; item += gridDim.y) {
        if (item == 0 ? !dpre : item == 1 && !dpost) continue;
        const int64_t gi = item - 2;
        const float* from = item == 0 ? sums.pre : item == 1 ? sums.s : sums.s + gi * go.parts * d;
        const int64_t count = item == 0 || (item == 1 && go.whole) ? go.grid()
                              : item == 1                          ? go.groups * go.parts
                                                                   : go.parts;
        // (S of a part of a group, times that group's gate, is its share of dpost)
        const bool weighted = item == 1 && !go.whole && gate.p && !gate.own;
        for (int64_t c0 = int64_t(blockIdx.x) * kWave; c0 < d; c0 += int64_t(gridDim.x) * kWave) {
            const int64_t c = c0 + l;
            float s = 0.f;
            if (c < d && weighted) {
                for (int64_t q = w; q < count; q += W) {
                    float k[1];
                    load_any<T, 1>(gate.p, gate.wide, q / go.parts * gate.ld + c, 1.f, k);
                    s = fmaf(from[q * d + c], k[0], s);
                }
            } else if (c < d) {
#pragma unroll 8
                for (int64_t q = w; q < count; q += W) s += from[q * d + c];
            }
            lds[w][l] = s;
            __syncthreads();
            if (w == 0 && c < d) {
                float v[1] = {0.f};
#pragma unroll
                for (int i = 0; i < W; ++i) v[0] += lds[i][l];
                if (item > 1) {
                    float k[1];
                    load_any<T, 1>(par.post, par.wide, c, 1.f, k);
                    v[0] *= k[0];
                    store_any<T, 1>(dgate, gate.wide, gi * lddg + c, v);
                } else {
                    store_any<T, 1>(item ? dpost : dpre, par.wide, c, v);
                }
            }
            __syncthreads();
        }
    }
}

// Lanes of a wavefront for up to 64 packs, else a workgroup's threads, one pack
// each (two of four columns past 1024): the gradient's thread holds four inputs
// and the next row's, three parameters and two sums for each of its columns, and
// has no registers for more.  Rows of more than 8192 columns are read again (np 0).
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

// Workgroups of the gradient: as many as a compute unit holds at two wavefronts
// a SIMD, over the groups.
constexpr int64_t kLongParts = 64;
Spread spread_of(int64_t m, int64_t groups, const RowShape& s) {
    Spread go;
    go.groups = groups;
    go.per = m / groups;
    const int rows = s.lanes ? kGradBlock / s.lanes : 1;
    const int64_t room = !s.np ? kLongParts : kCus * std::max(1, 512 / (s.lanes ? kGradBlock : s.threads));
    // (as many groups as walkers: each takes whole ones)
    if (m > 0 && groups > 1 && groups >= (s.np ? room * rows : room) / 2) {
        go.whole = true;
        go.slots = std::min(room, ceil_div(groups, s.np ? rows : 1));
        return go;
    }
    go.slots = std::min(groups, room);
    const int64_t most = std::max<int64_t>(1, ceil_div(go.per, s.np ? rows : kWavesPerBlock));
    go.parts = std::min(most, std::max<int64_t>(1, room / go.slots));
    return go;
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
            after_block<T, N, L, MOST, NP><<<grid, threads, 0, s>>>(x, X.ld, b, B.ld, m, d, gate, scale, par, normed,
                                                                    eps, y, Y.ld, h, H.ld, rstd_post, rstd_pre);
        });
    });
}

size_t block_norm_grad_tmp_bytes(int64_t m, int64_t d, int dt, const BlockGate& gate) {
    const RowShape shape = block_shape(d, dt);
    const Spread go = spread_of(m, groups_of(gate), shape);
    const int64_t rows = go.grid() + (go.whole ? go.grid() : go.groups * go.parts);
    return size_t(rows * d + (shape.np ? 0 : m)) * sizeof(float);
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
    sums.s = sums.pre + go.grid() * d;
    float* means = sums.s + (go.whole ? go.grid() : go.groups * go.parts) * d;
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
        auto by_whole = [&](auto f) {
            if (go.whole)
                f(integral_constant<bool, true>());
            else
                f(integral_constant<bool, false>());
        };
        if (m > 0 && shape.np) {
            by_block_shape<T, N, kGradBlock>(shape, [&](auto lanes, auto most, auto np) {
                constexpr int L = decltype(lanes)::value, MOST = decltype(most)::value, NP = decltype(np)::value;
                by_whole([&](auto whole) {
                    after_block_grad<T, N, L, MOST, NP, decltype(whole)::value>
                        <<<unsigned(go.grid()), L ? MOST : shape.threads, 0, s>>>(a);
                });
            });
        } else if (m > 0) {
            if constexpr (N > 1) {
                after_block_grad_long<T><<<row_grid(m), kRowBlock, 0, s>>>(a, means);
                by_whole([&](auto whole) {
                    after_block_sums_long<T, decltype(whole)::value>
                        <<<dim3(unsigned(ceil_div(packs_of(d, Y.dt), kWave)), unsigned(go.grid())), kBlock, 0, s>>>(
                            a, means);
                });
            }
        }
        const bool shared = gate.p && !gate.own && !go.whole;
        const int64_t items = shared ? 2 + go.groups : 2;
        Spread add = go;
        if (m == 0) add.parts = 0;  // (of no rows: zeros)
        join_sums<T><<<dim3(row_grid(ceil_div(d, kWave)), unsigned(std::min<int64_t>(items, 1 << 15))), kJoinBlock, 0,
                       s>>>(sums, add, items, d, gate, par, dpre, dpost, dgate, lddg);
    });
}

}  // namespace spsyrk
