// Layer norm of dense rows and its gradient.
//
//     mean = sum x / d,  var = sum (x - mean)^2 / d,  rstd = 1 / sqrt(var + eps),
//     h = (x - mean) rstd,  y = gamma h + beta;
//     a = gamma dy,  dx = rstd (a - sum a / d - h sum(a h) / d),
//     dgamma = sum over rows of dy h,  dbeta = sum over rows of dy.
//
// Bound by the bytes of the rows: every row is read once and held in
// registers (16 bytes per lane and pack) between its statistics and its
// output, by a group of 4 to 64 lanes or by a workgroup of as many wavefronts
// as it takes; the variance is a second pass
// over the registers, not a difference of sums.  Statistics and sums are
// 32-bit floats.  The parameters' gradients are summed by the threads that
// own the columns over the rows of a workgroup, written once per workgroup,
// and added in the workgroups' order by a second launch, so that results do
// not depend on timing; the gradient's workgroups load a row ahead.  Rows too
// long for registers are read again instead.
#include <algorithm>

#include "internal.h"
#include "row_shape.h"

namespace spsyrk {
namespace {

// N parameters of type PT at column c
template <int N, typename PT>
__device__ inline void load_params(const PT* p, int c, float none, float (&out)[N]) {
    constexpr int NP = N * int(sizeof(PT)) > 16 ? 16 / int(sizeof(PT)) : N;
    if (!p) {
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = none;
        return;
    }
#pragma unroll
    for (int q = 0; q < N / NP; ++q) {
        const Vec<PT, NP> v = load_vec<PT, NP>(p + c + q * NP);
#pragma unroll
        for (int i = 0; i < NP; ++i) out[q * NP + i] = float(v[i]);
    }
}

template <typename T, typename PT, int N, int L, int NP>
__global__ __launch_bounds__(L ? kBlock : kRowBlock) void norm_kernel(
    const T* __restrict__ x, int64_t ldx, int64_t m, int64_t d, const PT* __restrict__ gamma,
    const PT* __restrict__ beta, float eps, T* __restrict__ y, int64_t ldy, float* __restrict__ mean,
    float* __restrict__ rstd) {
    constexpr int ROWS = L ? kBlock / (L ? L : 1) : 1;
    constexpr bool KEEP = L && NP == 1;  // the parameters stay in registers over the rows
    __shared__ float buf[2][2][kMostWaves];
    const int threads = L ? L : int(blockDim.x), l = L ? int(threadIdx.x) % (L ? L : 1) : int(threadIdx.x);
    int turn = 0;
    Place at[NP];
    row_places<N>(l, threads, d, at);
    float g[N], b[N];
    if constexpr (KEEP) {
        load_params<N>(gamma, at[0].c, 1.f, g);
        load_params<N>(beta, at[0].c, 0.f, b);
    }
    for (int64_t r = int64_t(blockIdx.x) * ROWS + (L ? threadIdx.x / (L ? L : 1) : 0); r < m;
         r += int64_t(gridDim.x) * ROWS, turn ^= 1) {
        Vec<T, N> v[NP];
#pragma unroll
        for (int k = 0; k < NP; ++k) v[k] = load_vec_nt<T, N>(x + r * ldx + at[k].c);
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < NP; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) s += own(at, k, i) ? float(v[k][i]) : 0.f;
        const float mu = row_sum<L>(s, buf[turn][0]) / float(d);
        s = 0.f;
#pragma unroll
        for (int k = 0; k < NP; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float z = own(at, k, i) ? float(v[k][i]) - mu : 0.f;
                s = fmaf(z, z, s);
            }
        const float rs = 1.f / sqrtf(row_sum<L>(s, buf[turn][1]) / float(d) + eps);
        if (l == 0) {
            mean[r] = mu;
            rstd[r] = rs;
        }
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            if (at[k].shift >= N) break;
            if constexpr (!KEEP) {
                load_params<N>(gamma, at[k].c, 1.f, g);
                load_params<N>(beta, at[k].c, 0.f, b);
            }
            Vec<T, N> o;
#pragma unroll
            for (int i = 0; i < N; ++i) o[i] = T(fmaf((float(v[k][i]) - mu) * rs, g[i], b[i]));
            store_vec_nt<T, N>(y + r * ldy + at[k].c, o);
        }
    }
}

// rows too long for registers: three readings, the later ones from the caches
template <typename T, typename PT>
__global__ __launch_bounds__(kRowBlock) void norm_long(const T* __restrict__ x, int64_t ldx, int64_t m, int64_t d,
                                                       const PT* __restrict__ gamma, const PT* __restrict__ beta,
                                                       float eps, T* __restrict__ y, int64_t ldy,
                                                       float* __restrict__ mean, float* __restrict__ rstd) {
    constexpr int N = 16 / int(sizeof(T));
    constexpr int64_t STEP = int64_t(kRowBlock) * N;
    __shared__ float buf[2][2][kMostWaves];
    int turn = 0;
    for (int64_t r = blockIdx.x; r < m; r += gridDim.x, turn ^= 1) {
        const T* xr = x + r * ldx;
        float s = 0.f;
        for (int64_t c = int64_t(threadIdx.x) * N; c < d; c += STEP) {
            const Place at = place<N>(c, d);
            const Vec<T, N> v = load_vec<T, N>(xr + at.c);
#pragma unroll
            for (int i = 0; i < N; ++i) s += i >= at.shift ? float(v[i]) : 0.f;
        }
        const float mu = row_sum<0>(s, buf[turn][0]) / float(d);
        s = 0.f;
        for (int64_t c = int64_t(threadIdx.x) * N; c < d; c += STEP) {
            const Place at = place<N>(c, d);
            const Vec<T, N> v = load_vec<T, N>(xr + at.c);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float z = i >= at.shift ? float(v[i]) - mu : 0.f;
                s = fmaf(z, z, s);
            }
        }
        const float rs = 1.f / sqrtf(row_sum<0>(s, buf[turn][1]) / float(d) + eps);
        if (threadIdx.x == 0) {
            mean[r] = mu;
            rstd[r] = rs;
        }
        for (int64_t c = int64_t(threadIdx.x) * N; c < d; c += STEP) {
            const Place at = place<N>(c, d);
            const Vec<T, N> v = load_vec<T, N>(xr + at.c);
            float g[N], b[N];
            load_params<N>(gamma, at.c, 1.f, g);
            load_params<N>(beta, at.c, 0.f, b);
            Vec<T, N> o;
#pragma unroll
            for (int i = 0; i < N; ++i) o[i] = T(fmaf((float(v[i]) - mu) * rs, g[i], b[i]));
            store_vec_nt<T, N>(y + r * ldy + at.c, o);
        }
    }
}

// ---- gradient

// Threads per workgroup where rows take lanes of a wavefront.
constexpr int kGradBlock = 512;

// a row's packs of x and dy, and its statistics
template <typename T, int N, int NP>
struct GradRow {
    Vec<T, N> x[NP], dy[NP];
    float mu, rs;
};

// part: per workgroup the sums of dy h over its rows (d words), then of dy
// (null: no parameters).  L: lanes per row, or 0 and a workgroup of up to MOST
// threads per row.
template <typename T, typename PT, int N, int L, int MOST, int NP>
__global__ __launch_bounds__(MOST) void norm_grad_kernel(
    const T* __restrict__ dy, int64_t ldg, const T* __restrict__ x, int64_t ldx, int64_t m, int64_t d,
    const float* __restrict__ mean, const float* __restrict__ rstd, const PT* __restrict__ gamma, T* __restrict__ dx,
    int64_t ldd, float* __restrict__ part) {
    constexpr int ROWS = L ? MOST / (L ? L : 1) : 1;
    __shared__ float2 buf[2][kMostWaves];
    const int threads = L ? L : int(blockDim.x), l = L ? int(threadIdx.x) % (L ? L : 1) : int(threadIdx.x);
    int turn = 0;
    Place at[NP];
    row_places<N>(l, threads, d, at);
    float g[NP][N], dg[NP][N] = {}, db[NP][N] = {};
#pragma unroll
    for (int k = 0; k < NP; ++k) load_params<N>(gamma, at[k].c, 1.f, g[k]);
    auto load = [&](int64_t r) {
        GradRow<T, N, NP> q;
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            q.x[k] = load_vec_nt<T, N>(x + r * ldx + at[k].c);
            q.dy[k] = load_vec_nt<T, N>(dy + r * ldg + at[k].c);
        }
        q.mu = mean[r];
        q.rs = rstd[r];
        return q;
    };
    const int64_t step = int64_t(gridDim.x) * ROWS;
    int64_t r = int64_t(blockIdx.x) * ROWS + (L ? threadIdx.x / (L ? L : 1) : 0);
    // (a row ahead, but where its registers would spill)
    constexpr bool AHEAD = MOST < kRowBlock;
    GradRow<T, N, NP> next;
    if (AHEAD && r < m) next = load(r);
    for (; r < m; r += step, turn ^= 1) {
        const GradRow<T, N, NP> q = AHEAD ? next : load(r);
        if (AHEAD && r + step < m) next = load(r + step);
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < NP; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float w = float(q.dy[k][i]), h = (float(q.x[k][i]) - q.mu) * q.rs;
                const float a = own(at, k, i) ? w * g[k][i] : 0.f;
                s1 += a;
                s2 = fmaf(a, h, s2);
                dg[k][i] = fmaf(w, h, dg[k][i]);
                db[k][i] += w;
            }
        s1 = group_total<L ? L : kWave>(s1);
        s2 = group_total<L ? L : kWave>(s2);
        if constexpr (L == 0) {
            // (two buffers: a wavefront can be one row ahead of another)
            if (lane_id() == 0) buf[turn][l / kWave] = make_float2(s1, s2);
            lds_barrier();
            s1 = s2 = 0.f;
            for (int i = 0; i < threads / kWave; ++i) {
                s1 += buf[turn][i].x;
                s2 += buf[turn][i].y;
            }
        }
        s1 /= float(d);
        s2 /= float(d);
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            if (at[k].shift >= N) break;
            Vec<T, N> o;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float h = (float(q.x[k][i]) - q.mu) * q.rs;
                o[i] = T(q.rs * (float(q.dy[k][i]) * g[k][i] - s1 - h * s2));
            }
            store_vec_nt<T, N>(dx + r * ldd + at[k].c, o);
        }
    }
    if (!part) return;
    float* p = part + int64_t(blockIdx.x) * 2 * d;
    if constexpr (ROWS > 1) {
        // the sums of a wavefront's groups, by lane distance; then the
        // wavefronts', pairwise: the upper half's through LDS to the lower half
        constexpr int WAVES = MOST / kWave;
        __shared__ float sum[WAVES / 2][2][NP][N][kWave];
        const int w = threadIdx.x / kWave, lane = lane_id();
#pragma unroll
        for (int far = L; far < kWave; far *= 2)
#pragma unroll
            for (int k = 0; k < NP; ++k)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    dg[k][i] += __shfl_xor(dg[k][i], far, kWave);
                    db[k][i] += __shfl_xor(db[k][i], far, kWave);
                }
#pragma unroll
        for (int half = WAVES / 2; half > 0; half /= 2) {
            if (w >= half && w < 2 * half)
#pragma unroll
                for (int k = 0; k < NP; ++k)
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        sum[w - half][0][k][i][lane] = dg[k][i];
                        sum[w - half][1][k][i][lane] = db[k][i];
                    }
            __syncthreads();
            if (w < half)
#pragma unroll
                for (int k = 0; k < NP; ++k)
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        dg[k][i] += sum[w][0][k][i][lane];
                        db[k][i] += sum[w][1][k][i][lane];
                    }
            __syncthreads();
        }
        if (w > 0 || lane >= L) return;
    }
#pragma unroll
    for (int k = 0; k < NP; ++k) {
        if (at[k].shift >= N) break;
        Vec<float, N> a, b;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            a[i] = dg[k][i];
            b[i] = db[k][i];
        }
        store_vec<float, N>(p + at[k].c, a);
        store_vec<float, N>(p + d + at[k].c, b);
    }
}

// rows too long for registers: dx by two readings
template <typename T, typename PT>
__global__ __launch_bounds__(kRowBlock) void norm_grad_long(const T* __restrict__ dy, int64_t ldg,
                                                            const T* __restrict__ x, int64_t ldx, int64_t m,
                                                            int64_t d, const float* __restrict__ mean,
                                                            const float* __restrict__ rstd,
                                                            const PT* __restrict__ gamma, T* __restrict__ dx,
                                                            int64_t ldd) {
    constexpr int N = 16 / int(sizeof(T));
    constexpr int64_t STEP = int64_t(kRowBlock) * N;
    __shared__ float buf[2][2][kMostWaves];
    int turn = 0;
    for (int64_t r = blockIdx.x; r < m; r += gridDim.x, turn ^= 1) {
        const T *xr = x + r * ldx, *gr = dy + r * ldg;
        const float mu = mean[r], rs = rstd[r];
        float s1 = 0.f, s2 = 0.f;
        for (int64_t c = int64_t(threadIdx.x) * N; c < d; c += STEP) {
            const Place at = place<N>(c, d);
            const Vec<T, N> v = load_vec<T, N>(xr + at.c), w = load_vec<T, N>(gr + at.c);
            float g[N];
            load_params<N>(gamma, at.c, 1.f, g);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float a = i >= at.shift ? float(w[i]) * g[i] : 0.f;
                s1 += a;
                s2 = fmaf(a, (float(v[i]) - mu) * rs, s2);
            }
        }
        s1 = row_sum<0>(s1, buf[turn][0]) / float(d);
        s2 = row_sum<0>(s2, buf[turn][1]) / float(d);
        for (int64_t c = int64_t(threadIdx.x) * N; c < d; c += STEP) {
            const Place at = place<N>(c, d);
            const Vec<T, N> v = load_vec<T, N>(xr + at.c), w = load_vec<T, N>(gr + at.c);
            float g[N];
            load_params<N>(gamma, at.c, 1.f, g);
            Vec<T, N> o;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float h = (float(v[i]) - mu) * rs;
                o[i] = T(rs * (float(w[i]) * g[i] - s1 - h * s2));
            }
            store_vec_nt<T, N>(dx + r * ldd + at.c, o);
        }
    }
}

// The parameters' sums of long rows: workgroup (x, y) takes a pack of columns
// per lane and every gridDim.y-th row, its wavefronts in turn.
template <typename T>
__global__ __launch_bounds__(kBlock) void norm_params_long(const T* __restrict__ dy, int64_t ldg,
                                                           const T* __restrict__ x, int64_t ldx, int64_t m, int64_t d,
                                                           const float* __restrict__ mean,
                                                           const float* __restrict__ rstd, float* __restrict__ part) {
    constexpr int N = 16 / int(sizeof(T));
    __shared__ float sum[2][kWave * N];
    const int w = threadIdx.x / kWave, l = lane_id();
    const Place at = place<N>((int64_t(blockIdx.x) * kWave + l) * N, d);
    float dg[N] = {}, db[N] = {};
    for (int64_t r = int64_t(blockIdx.y) * kWavesPerBlock + w; r < m; r += int64_t(gridDim.y) * kWavesPerBlock) {
        const Vec<T, N> v = load_vec<T, N>(x + r * ldx + at.c), g = load_vec<T, N>(dy + r * ldg + at.c);
        const float mu = mean[r], rs = rstd[r];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            dg[i] = fmaf(float(g[i]), (float(v[i]) - mu) * rs, dg[i]);
            db[i] += float(g[i]);
        }
    }
    for (int q = 0; q < kWavesPerBlock; ++q) {
        if (w == q)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                sum[0][l * N + i] = dg[i] + (q ? sum[0][l * N + i] : 0.f);
                sum[1][l * N + i] = db[i] + (q ? sum[1][l * N + i] : 0.f);
            }
        __syncthreads();
    }
    if (w > 0 || at.shift >= N) return;
    float* p = part + int64_t(blockIdx.y) * 2 * d + at.c;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        p[i] = sum[0][l * N + i];
        p[d + i] = sum[1][l * N + i];
    }
}

// dgamma (blockIdx.y 0) and dbeta (1): the groups' sums in their order within
// a wavefront, the wavefronts' in theirs
constexpr int kJoinBlock = 1024;
template <typename PT>
__global__ __launch_bounds__(kJoinBlock) void norm_params_join(const float* __restrict__ part, int64_t groups,
                                                               int64_t d, PT* __restrict__ dgamma,
                                                               PT* __restrict__ dbeta) {
    constexpr int W = kJoinBlock / kWave;
    __shared__ float sum[W][kWave];
    PT* out = blockIdx.y ? dbeta : dgamma;
    if (!out) return;
    const int w = threadIdx.x / kWave, l = lane_id();
    for (int64_t c0 = int64_t(blockIdx.x) * kWave; c0 < d; c0 += int64_t(gridDim.x) * kWave) {
        const int64_t c = c0 + l;
        float s = 0.f;
        if (c < d) {
#pragma unroll 8
            for (int64_t q = w; q < groups; q += W) s += part[(2 * q + blockIdx.y) * d + c];
        }
        sum[w][l] = s;
        __syncthreads();
        if (w == 0 && c < d) {
            s = 0.f;
#pragma unroll
            for (int i = 0; i < W; ++i) s += sum[i][l];
            out[c] = PT(s);
        }
        __syncthreads();
    }
}

// The gradient's threads hold two rows' packs of x and dy, gamma and two sums
// per column: two packs of eight columns, or up to four of four.
inline RowShape grad_shape(int64_t d, int dt) { return row_shape(packs_of(d, dt), dt == kDtF32 ? 4 : 2, true); }

// Workgroups of the gradient (each writes 2 d sums): as many as the registers
// let a compute unit hold, 12 or 16 wavefronts (more would take a second turn).
constexpr int64_t kLongGroups = 64;
inline int64_t grad_groups(int64_t m, const RowShape& s, int dt) {
    if (!s.np) return kLongGroups;
    if (s.lanes) return std::min<int64_t>(ceil_div(m, kGradBlock / s.lanes), s.np == 1 ? 2 * kCus : kCus);
    const int waves = dt == kDtF32 && s.np == 2 ? 16 : 12;
    return std::min<int64_t>(m, int64_t(kCus) * std::max(waves * kWave / s.threads, 1));
}

template <typename F>
inline void by_params(int dt, int pt, int64_t d, F f) {
    by_width(dt, d, [&](auto e, auto n) {
        if (pt == kDtF32)
            f(e, float(), n);
        else
            f(e, e, n);
    });
}

}  // namespace

void layer_norm(const DenseRows& X, const void* gamma, const void* beta, int pt, float eps, const DenseRows& Y,
                float* mean, float* rstd, hipStream_t s) {
    by_params(X.dt, pt, X.n, [&](auto e, auto q, auto n) {
        using T = decltype(e);
        using PT = decltype(q);
        constexpr int N = decltype(n)::value;
        const int64_t m = X.m, d = X.n;
        const T* x = static_cast<const T*>(X.p);
        const PT *g = static_cast<const PT*>(gamma), *b = static_cast<const PT*>(beta);
        T* y = static_cast<T*>(Y.p);
        const RowShape shape = row_shape(packs_of(d, X.dt), 4, false);
        if (!shape.np) {
            if constexpr (N > 1)
                norm_long<T, PT><<<row_grid(m), kRowBlock, 0, s>>>(x, X.ld, m, d, g, b, eps, y, Y.ld, mean, rstd);
            return;
        }
        by_shape<N>(shape, [&](auto lanes, auto np) {
            constexpr int L = decltype(lanes)::value, NP = decltype(np)::value;
            // (parameters in registers: as many workgroups as the chip holds, over all rows)
            const int64_t blocks = L ? ceil_div(m, kBlock / (L ? L : 1)) : m;
            const unsigned grid = row_grid(L && NP == 1 ? std::min<int64_t>(blocks, 8 * kCus) : blocks);
            norm_kernel<T, PT, N, L, NP><<<grid, L ? kBlock : shape.threads, 0, s>>>(x, X.ld, m, d, g, b, eps, y, Y.ld,
                                                                                    mean, rstd);
        });
    });
}

size_t layer_norm_grad_tmp_bytes(int64_t m, int64_t d, int dt, bool params) {
    return params ? size_t(grad_groups(m, grad_shape(d, dt), dt)) * 2 * size_t(d) * sizeof(float) : 0;
}

void layer_norm_grad(const DenseRows& G, const DenseRows& X, const float* mean, const float* rstd, const void* gamma,
                     int pt, const DenseRows& dX, void* dgamma, void* dbeta, void* tmp, hipStream_t s) {
    const RowShape shape = grad_shape(X.n, X.dt);
    const int64_t groups = X.m ? grad_groups(X.m, shape, X.dt) : 0;
    by_params(X.dt, pt, X.n, [&](auto e, auto q, auto n) {
        using T = decltype(e);
        using PT = decltype(q);
        constexpr int N = decltype(n)::value;
        const int64_t m = X.m, d = X.n;
        const T *x = static_cast<const T*>(X.p), *dy = static_cast<const T*>(G.p);
        const PT* g = static_cast<const PT*>(gamma);
        T* dx = static_cast<T*>(dX.p);
        float* part = dgamma || dbeta ? static_cast<float*>(tmp) : nullptr;
        if (m > 0 && shape.np) {
            by_shape<N>(shape, [&](auto lanes, auto np) {
                constexpr int L = decltype(lanes)::value, NP = decltype(np)::value;
                // (more than two packs: f32 only)
                if constexpr (NP <= 2 || sizeof(T) == 4) {
                    auto launch = [&](auto most, int threads) {
                        constexpr int MOST = decltype(most)::value;
                        norm_grad_kernel<T, PT, N, L, MOST, NP><<<unsigned(groups), threads, 0, s>>>(
                            dy, G.ld, x, X.ld, m, d, mean, rstd, g, dx, dX.ld, part);
                    };
                    if constexpr (L > 0) {
                        launch(std::integral_constant<int, kGradBlock>(), kGradBlock);
                    } else {
                        if (shape.threads <= kGradBlock)
                            launch(std::integral_constant<int, kGradBlock>(), shape.threads);
                        else
                            launch(std::integral_constant<int, kRowBlock>(), shape.threads);
                    }
                }
            });
        } else if (m > 0) {
            if constexpr (N > 1) {
                norm_grad_long<T, PT><<<row_grid(m), kRowBlock, 0, s>>>(dy, G.ld, x, X.ld, m, d, mean, rstd, g, dx,
                                                                        dX.ld);
                if (part)
                    norm_params_long<T><<<dim3(unsigned(ceil_div(packs_of(d, X.dt), kWave)), unsigned(groups)), kBlock,
                                          0, s>>>(dy, G.ld, x, X.ld, m, d, mean, rstd, part);
            }
        }
        if (dgamma || dbeta)  // (of no rows: zeros)
            norm_params_join<PT><<<dim3(row_grid(ceil_div(d, kWave)), 2), kJoinBlock, 0, s>>>(
                part, groups, d, static_cast<PT*>(dgamma), static_cast<PT*>(dbeta));
    });
}

}  // namespace spsyrk
