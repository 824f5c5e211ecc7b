// Layer norm of dense rows and its gradient.
//
//     mean = sum x / d,  var = sum (x - mean)^2 / d,  rstd = 1 / sqrt(var + eps),
//     h = (x - mean) rstd,  y = gamma h + beta;
//     a = gamma dy,  dx = rstd (a - sum a / d - h sum(a h) / d),
//     dgamma = sum over rows of dy h,  dbeta = sum over rows of dy.
//
// Bound by the bytes of the rows: every row is read once and held in
// registers (16 bytes per lane and pack) between its statistics and its
// output, by one wavefront or by one workgroup; the variance is a second pass
// over the registers, not a difference of sums.  Statistics and sums are
// 32-bit floats.  The parameters' gradients are summed by the threads that
// own the columns over the rows of a workgroup, written once per workgroup,
// and added in the workgroups' order by a second launch, so that results do
// not depend on timing.  Rows too long for registers are read again instead.
#include <algorithm>

#include "internal.h"
#include "rows.h"

namespace spsyrk {
namespace {

constexpr int kRowBlock = 1024;  // threads per row, at most

// N parameters of type PT at column c (0 where none exist)
template <typename T, typename PT>
__device__ inline void load_params(const PT* p, int64_t c, int64_t d, float none, float (&out)[Pack<T>::N]) {
    constexpr int N = Pack<T>::N, NP = Pack<PT>::N;
    if (!p) {
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = none;
        return;
    }
#pragma unroll
    for (int q = 0; q < N / NP; ++q) {
        const PackV<PT> v = load_pack(p + c + q * NP, d - c - q * NP);
#pragma unroll
        for (int i = 0; i < NP; ++i) out[q * NP + i] = float(v[i]);
    }
}

// Sum over the TPR threads of a row (a wavefront, or the whole workgroup with
// buf of TPR / kWave words); every thread gets it.
template <int TPR>
__device__ inline float row_sum(float v, float* buf) {
    v = wave_reduce_sum(v);
    if constexpr (TPR == kWave) return v;
    if (lane_id() == 0) buf[threadIdx.x / kWave] = v;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < TPR / kWave; ++i) s += buf[i];
    __syncthreads();
    return s;
}

template <int TPR>
constexpr int threads_of() {
    return TPR == kWave ? kBlock : TPR;
}

template <typename T, typename PT, int TPR, int NP>
__global__ __launch_bounds__(threads_of<TPR>()) void norm_kernel(const T* __restrict__ x, int64_t ldx, int64_t m,
                                                                 int64_t d, const PT* __restrict__ gamma,
                                                                 const PT* __restrict__ beta, float eps,
                                                                 T* __restrict__ y, int64_t ldy,
                                                                 float* __restrict__ mean, float* __restrict__ rstd) {
    constexpr int N = Pack<T>::N, ROWS = threads_of<TPR>() / TPR;
    __shared__ float buf[TPR / kWave];
    const int l = threadIdx.x % TPR;
    for (int64_t r = int64_t(blockIdx.x) * ROWS + threadIdx.x / TPR; r < m; r += int64_t(gridDim.x) * ROWS) {
        PackV<T> v[NP];
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            const int64_t c = (int64_t(k) * TPR + l) * N;
            v[k] = load_pack_nt(x + r * ldx + c, d - c);
        }
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < NP; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) s += float(v[k][i]);
        const float mu = row_sum<TPR>(s, buf) / float(d);
        s = 0.f;
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            const int64_t c = (int64_t(k) * TPR + l) * N;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float z = c + i < d ? float(v[k][i]) - mu : 0.f;
                s = fmaf(z, z, s);
            }
        }
        const float rs = 1.f / sqrtf(row_sum<TPR>(s, buf) / float(d) + eps);
        if (l == 0) {
            mean[r] = mu;
            rstd[r] = rs;
        }
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            const int64_t c = (int64_t(k) * TPR + l) * N;
            if (c >= d) break;
            float g[N], b[N];
            load_params<T, PT>(gamma, c, d, 1.f, g);
            load_params<T, PT>(beta, c, d, 0.f, b);
            PackV<T> o;
#pragma unroll
            for (int i = 0; i < N; ++i) o[i] = T(fmaf((float(v[k][i]) - mu) * rs, g[i], b[i]));
            store_pack_nt(y + r * ldy + c, o, d - c);
        }
    }
}

// rows too long for registers: three readings, the later ones from the caches
template <typename T, typename PT>
__global__ __launch_bounds__(kRowBlock) void norm_long(const T* __restrict__ x, int64_t ldx, int64_t m, int64_t d,
                                                       const PT* __restrict__ gamma, const PT* __restrict__ beta,
                                                       float eps, T* __restrict__ y, int64_t ldy,
                                                       float* __restrict__ mean, float* __restrict__ rstd) {
    constexpr int N = Pack<T>::N;
    constexpr int64_t STEP = int64_t(kRowBlock) * N;
    __shared__ float buf[kRowBlock / kWave];
    for (int64_t r = blockIdx.x; r < m; r += gridDim.x) {
        const T* xr = x + r * ldx;
        float s = 0.f;
        for (int64_t c = int64_t(threadIdx.x) * N; c < d; c += STEP) {
            const PackV<T> v = load_pack(xr + c, d - c);
#pragma unroll
            for (int i = 0; i < N; ++i) s += float(v[i]);
        }
        const float mu = row_sum<kRowBlock>(s, buf) / float(d);
        s = 0.f;
        for (int64_t c = int64_t(threadIdx.x) * N; c < d; c += STEP) {
            const PackV<T> v = load_pack(xr + c, d - c);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float z = c + i < d ? float(v[i]) - mu : 0.f;
                s = fmaf(z, z, s);
            }
        }
        const float rs = 1.f / sqrtf(row_sum<kRowBlock>(s, buf) / float(d) + eps);
        if (threadIdx.x == 0) {
            mean[r] = mu;
            rstd[r] = rs;
        }
        for (int64_t c = int64_t(threadIdx.x) * N; c < d; c += STEP) {
            const PackV<T> v = load_pack(xr + c, d - c);
            float g[N], b[N];
            load_params<T, PT>(gamma, c, d, 1.f, g);
            load_params<T, PT>(beta, c, d, 0.f, b);
            PackV<T> o;
#pragma unroll
            for (int i = 0; i < N; ++i) o[i] = T(fmaf((float(v[i]) - mu) * rs, g[i], b[i]));
            store_pack_nt(y + r * ldy + c, o, d - c);
        }
    }
}

// ---- gradient

// part: per workgroup the sums of dy h over its rows (d words), then of dy
// (null: no parameters)
template <typename T, typename PT, int TPR, int NP>
__global__ __launch_bounds__(threads_of<TPR>()) void norm_grad_kernel(
    const T* __restrict__ dy, int64_t ldg, const T* __restrict__ x, int64_t ldx, int64_t m, int64_t d,
    const float* __restrict__ mean, const float* __restrict__ rstd, const PT* __restrict__ gamma, T* __restrict__ dx,
    int64_t ldd, float* __restrict__ part) {
    constexpr int N = Pack<T>::N, ROWS = threads_of<TPR>() / TPR;
    __shared__ float buf[TPR / kWave];
    const int l = threadIdx.x % TPR;
    float g[NP][N], dg[NP][N] = {}, db[NP][N] = {};
#pragma unroll
    for (int k = 0; k < NP; ++k) load_params<T, PT>(gamma, (int64_t(k) * TPR + l) * N, d, 1.f, g[k]);
    for (int64_t r = int64_t(blockIdx.x) * ROWS + threadIdx.x / TPR; r < m; r += int64_t(gridDim.x) * ROWS) {
        PackV<T> v[NP], w[NP];
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            const int64_t c = (int64_t(k) * TPR + l) * N;
            v[k] = load_pack_nt(x + r * ldx + c, d - c);
            w[k] = load_pack_nt(dy + r * ldg + c, d - c);  // (0 past the row: adds nothing below)
        }
        const float mu = mean[r], rs = rstd[r];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < NP; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float h = (float(v[k][i]) - mu) * rs, a = float(w[k][i]) * g[k][i];
                s1 += a;
                s2 = fmaf(a, h, s2);
                dg[k][i] = fmaf(float(w[k][i]), h, dg[k][i]);
                db[k][i] += float(w[k][i]);
            }
        s1 = row_sum<TPR>(s1, buf) / float(d);
        s2 = row_sum<TPR>(s2, buf) / float(d);
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            const int64_t c = (int64_t(k) * TPR + l) * N;
            if (c >= d) break;
            PackV<T> o;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float h = (float(v[k][i]) - mu) * rs;
                o[i] = T(rs * (float(w[k][i]) * g[k][i] - s1 - h * s2));
            }
            store_pack_nt(dx + r * ldd + c, o, d - c);
        }
    }
    if (!part) return;
    float* p = part + int64_t(blockIdx.x) * 2 * d;
    if constexpr (ROWS == 1) {
#pragma unroll
        for (int k = 0; k < NP; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int64_t c = (int64_t(k) * TPR + l) * N + i;
                if (c < d) {
                    p[c] = dg[k][i];
                    p[d + c] = db[k][i];
                }
            }
    } else {
        // the wavefronts' sums, added in their order
        __shared__ float sum[2][TPR * NP * N];
        for (int q = 0; q < ROWS; ++q) {
            if (int(threadIdx.x / TPR) == q) {
#pragma unroll
                for (int k = 0; k < NP; ++k)
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const int c = (k * TPR + l) * N + i;
                        sum[0][c] = dg[k][i] + (q ? sum[0][c] : 0.f);
                        sum[1][c] = db[k][i] + (q ? sum[1][c] : 0.f);
                    }
            }
            __syncthreads();
        }
        for (int64_t c = threadIdx.x; c < d; c += threads_of<TPR>()) {
            p[c] = sum[0][c];
            p[d + c] = sum[1][c];
        }
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
    constexpr int N = Pack<T>::N;
    constexpr int64_t STEP = int64_t(kRowBlock) * N;
    __shared__ float buf[kRowBlock / kWave];
    for (int64_t r = blockIdx.x; r < m; r += gridDim.x) {
        const T *xr = x + r * ldx, *gr = dy + r * ldg;
        const float mu = mean[r], rs = rstd[r];
        float s1 = 0.f, s2 = 0.f;
        for (int64_t c = int64_t(threadIdx.x) * N; c < d; c += STEP) {
            const PackV<T> v = load_pack(xr + c, d - c), w = load_pack(gr + c, d - c);
            float g[N];
            load_params<T, PT>(gamma, c, d, 1.f, g);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float a = float(w[i]) * g[i];
                s1 += a;
                s2 = fmaf(a, (float(v[i]) - mu) * rs, s2);
            }
        }
        s1 = row_sum<kRowBlock>(s1, buf) / float(d);
        s2 = row_sum<kRowBlock>(s2, buf) / float(d);
        for (int64_t c = int64_t(threadIdx.x) * N; c < d; c += STEP) {
            const PackV<T> v = load_pack(xr + c, d - c), w = load_pack(gr + c, d - c);
            float g[N];
            load_params<T, PT>(gamma, c, d, 1.f, g);
            PackV<T> o;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float h = (float(v[i]) - mu) * rs;
                o[i] = T(rs * (float(w[i]) * g[i] - s1 - h * s2));
            }
            store_pack_nt(dx + r * ldd + c, o, d - c);
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
    constexpr int N = Pack<T>::N;
    __shared__ float sum[2][kWave * N];
    const int w = threadIdx.x / kWave, l = lane_id();
    const int64_t c = (int64_t(blockIdx.x) * kWave + l) * N;
    float dg[N] = {}, db[N] = {};
    for (int64_t r = int64_t(blockIdx.y) * kWavesPerBlock + w; r < m; r += int64_t(gridDim.y) * kWavesPerBlock) {
        const PackV<T> v = load_pack(x + r * ldx + c, d - c), g = load_pack(dy + r * ldg + c, d - c);
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
    float* p = part + int64_t(blockIdx.y) * 2 * d;
    for (int i = threadIdx.x; i < kWave * N; i += kBlock) {
        const int64_t cc = int64_t(blockIdx.x) * kWave * N + i;
        if (cc < d) {
            p[cc] = sum[0][i];
            p[d + cc] = sum[1][i];
        }
    }
}

// dgamma (blockIdx.y 0) and dbeta (1): the groups' sums in their order within
// a wavefront, the wavefronts' in theirs
constexpr int kJoinBlock = 1024;
template <typename PT>
__global__ __launch_bounds__(kJoinBlock) void norm_params_join(const float* __restrict__ part, int64_t groups,
                                                               int64_t d, PT* __restrict__ dgamma,
                                                               PT* __restrict__ dbeta) {
    __shared__ float sum[kJoinBlock / kWave][kWave];
    PT* out = blockIdx.y ? dbeta : dgamma;
    if (!out) return;
    const int w = threadIdx.x / kWave, l = lane_id();
    for (int64_t c0 = int64_t(blockIdx.x) * kWave; c0 < d; c0 += int64_t(gridDim.x) * kWave) {
        const int64_t c = c0 + l;
        float s = 0.f;
        if (c < d)
            for (int64_t q = w; q < groups; q += kJoinBlock / kWave) s += part[(2 * q + blockIdx.y) * d + c];
        sum[w][l] = s;
        __syncthreads();
        if (w == 0 && c < d) {
            s = 0.f;
#pragma unroll
            for (int i = 0; i < kJoinBlock / kWave; ++i) s += sum[i][l];
            out[c] = PT(s);
        }
        __syncthreads();
    }
}

// packs held per thread, and threads per row, for rows of `packs` packs
constexpr int kWavePacks = 2;
constexpr int64_t kLongGroups = 64;

// workgroups of the gradient: four per compute unit of 256 threads, fewer of
// more (each writes 2 d sums)
inline int64_t grad_groups(int64_t m, int64_t packs) {
    if (packs <= kWavePacks * kWave) return std::min<int64_t>((m + 3) / 4, 1024);
    return std::min<int64_t>(m, packs <= 2 * kBlock ? 512 : 256);
}

template <typename F>
inline void by_params(int dt, int pt, F f) {
    by_dtype(dt, [&](auto e) {
        if (pt == kDtF32)
            f(e, float());
        else
            f(e, e);
    });
}

inline unsigned row_grid(int64_t blocks) { return unsigned(std::min<int64_t>(blocks, int64_t(1) << 20)); }

}  // namespace

void layer_norm(const DenseRows& X, const void* gamma, const void* beta, int pt, float eps, const DenseRows& Y,
                float* mean, float* rstd, hipStream_t s) {
    by_params(X.dt, pt, [&](auto e, auto q) {
        using T = decltype(e);
        using PT = decltype(q);
        const int64_t m = X.m, d = X.n, packs = (d + Pack<T>::N - 1) / Pack<T>::N;
        const T* x = static_cast<const T*>(X.p);
        const PT *g = static_cast<const PT*>(gamma), *b = static_cast<const PT*>(beta);
        T* y = static_cast<T*>(Y.p);
        if (packs <= kWave)
            norm_kernel<T, PT, kWave, 1><<<row_grid((m + 3) / 4), kBlock, 0, s>>>(x, X.ld, m, d, g, b, eps, y, Y.ld,
                                                                                  mean, rstd);
        else if (packs <= 2 * kWave)
            norm_kernel<T, PT, kWave, 2><<<row_grid((m + 3) / 4), kBlock, 0, s>>>(x, X.ld, m, d, g, b, eps, y, Y.ld,
                                                                                  mean, rstd);
        else if (packs <= 2 * kBlock)
            norm_kernel<T, PT, kBlock, 2><<<row_grid(m), kBlock, 0, s>>>(x, X.ld, m, d, g, b, eps, y, Y.ld, mean,
                                                                        rstd);
        else if (packs <= 4 * kBlock)
            norm_kernel<T, PT, kBlock, 4><<<row_grid(m), kBlock, 0, s>>>(x, X.ld, m, d, g, b, eps, y, Y.ld, mean,
                                                                        rstd);
        else if (packs <= 4 * kRowBlock)
            norm_kernel<T, PT, kRowBlock, 4><<<row_grid(m), kRowBlock, 0, s>>>(x, X.ld, m, d, g, b, eps, y, Y.ld,
                                                                              mean, rstd);
        else
            norm_long<T, PT><<<row_grid(m), kRowBlock, 0, s>>>(x, X.ld, m, d, g, b, eps, y, Y.ld, mean, rstd);
    });
}

namespace {
// rows whose packs the gradient's threads hold, at most (registers: the row of
// x and of dy, gamma and two sums per column)
template <typename T>
constexpr int grad_block_packs() {
    return sizeof(T) == 4 ? 4 : 2;
}
inline int64_t grad_most_packs(int dt) { return int64_t(dt == kDtF32 ? 4 : 2) * kRowBlock; }
inline int64_t packs_of(int64_t d, int dt) { return (d * dtype_bytes(dt) + 15) / 16; }
}  // namespace

size_t layer_norm_grad_tmp_bytes(int64_t m, int64_t d, int dt, bool params) {
    if (!params) return 0;
    const int64_t packs = packs_of(d, dt);
    const int64_t groups = packs > grad_most_packs(dt) ? kLongGroups : grad_groups(m, packs);
    return size_t(groups) * 2 * size_t(d) * sizeof(float);
}

void layer_norm_grad(const DenseRows& G, const DenseRows& X, const float* mean, const float* rstd, const void* gamma,
                     int pt, const DenseRows& dX, void* dgamma, void* dbeta, void* tmp, hipStream_t s) {
    by_params(X.dt, pt, [&](auto e, auto q) {
        using T = decltype(e);
        using PT = decltype(q);
        constexpr int BP = grad_block_packs<T>();
        const int64_t m = X.m, d = X.n, packs = packs_of(d, X.dt);
        const T *x = static_cast<const T*>(X.p), *dy = static_cast<const T*>(G.p);
        const PT* g = static_cast<const PT*>(gamma);
        T* dx = static_cast<T*>(dX.p);
        float* part = dgamma || dbeta ? static_cast<float*>(tmp) : nullptr;
        int64_t groups = grad_groups(m, packs);
        const unsigned nb = unsigned(groups);
        if (m == 0)
            ;  // (the parameters' gradients are zeros)
        else if (packs <= kWave)
            norm_grad_kernel<T, PT, kWave, 1><<<nb, kBlock, 0, s>>>(dy, G.ld, x, X.ld, m, d, mean, rstd, g, dx, dX.ld,
                                                                    part);
        else if (packs <= kWavePacks * kWave)
            norm_grad_kernel<T, PT, kWave, kWavePacks><<<nb, kBlock, 0, s>>>(dy, G.ld, x, X.ld, m, d, mean, rstd, g,
                                                                             dx, dX.ld, part);
        else if (packs <= 2 * kBlock)
            norm_grad_kernel<T, PT, kBlock, 2><<<nb, kBlock, 0, s>>>(dy, G.ld, x, X.ld, m, d, mean, rstd, g, dx,
                                                                     dX.ld, part);
        else if (packs <= 2 * 512)
            norm_grad_kernel<T, PT, 512, 2><<<nb, 512, 0, s>>>(dy, G.ld, x, X.ld, m, d, mean, rstd, g, dx, dX.ld,
                                                               part);
        else if (packs <= BP * kRowBlock)
            norm_grad_kernel<T, PT, kRowBlock, BP><<<nb, kRowBlock, 0, s>>>(dy, G.ld, x, X.ld, m, d, mean, rstd, g,
                                                                            dx, dX.ld, part);
        else {
            norm_grad_long<T, PT><<<row_grid(m), kRowBlock, 0, s>>>(dy, G.ld, x, X.ld, m, d, mean, rstd, g, dx,
                                                                    dX.ld);
            groups = kLongGroups;
            if (part)
                norm_params_long<T><<<dim3(unsigned((packs + kWave - 1) / kWave), unsigned(groups)), kBlock, 0, s>>>(
                    dy, G.ld, x, X.ld, m, d, mean, rstd, part);
        }
        if (dgamma || dbeta)
            norm_params_join<PT><<<dim3(row_grid((d + kWave - 1) / kWave), 2), kJoinBlock, 0, s>>>(
                part, groups, d, static_cast<PT*>(dgamma), static_cast<PT*>(dbeta));
    });
}

}  // namespace spsyrk
