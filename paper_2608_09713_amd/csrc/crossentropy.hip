// Softmax cross entropy of a linear layer, and its gradient.
//
//     z = s x W^T,  lse = log sum exp z,  loss = lse - z[t];
//     G = w (softmax(z) - onehot(t)),  dx = s G W,  dW = s G^T x.
//
// Bound by the matrix cores: one product for the loss, three for the gradient, and
// for few rows by the bytes of W (1 x 32000 x 2048 bf16: 31 us in a call, 22 of them
// the reading of 131 MB).  8192 x 131072 x 4096 bf16: 6.33 ms, 1390 TFLOP/s of the
// 1484 that a plain library product reaches here; the chip's clock falls to 1.9 GHz
// under either.  The gradient of 4096 such rows: 10.8 to 11.3 ms, of which the
// products take 3.4, 3.5 and 3.8 and G 0.38 (5.6 TB/s).
// The logits are not kept.  A tile of the product (a piece of the vocabulary by
// some rows) leaves each row's largest logit and the sum of the exponentials
// below it; the rows' pieces are joined by a second launch.  The target's logit
// takes no part in them but is kept apart: of a row that is nearly sure the others'
// sum e^(z - z[t]) is the loss, all of whose digits a sum with the target's 1 would
// take.  The gradient takes some rows at a time and keeps their exponentials, each
// relative to its tile's largest, in the inputs' type: a rounding of at most half a
// step of each probability, where a rounded logit would cost several.  `fold` makes
// G of them in place, the target's entry, w (e^-loss - 1), from the 32-bit loss.  The
// products that follow take W, G and x turned as they lie, with no copies but of x's
// rows that count.
//
// Exponentials are powers of two of differences times log2(e), so that logits
// up to the floats' ends keep theirs.  A tile's base is at least the lowest
// float, so that logits of -inf (and a target's place) add nothing.
#include <algorithm>
#include <cmath>

#include "internal.h"
#include "product.h"
#include "training.h"

namespace spsyrk {
namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kCus = 256;  // compute units of the chip

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }

// Powers of two that E is raised by: IEEE 16-bit floats end at 2^-24, so theirs
// take the range up to 2^15.
template <typename T>
constexpr float kRaise = std::is_same<T, _Float16>::value ? 15.f : 0.f;

__device__ inline int64_t target_of(const Targets& t, int64_t row) { return load_column(t.p, t.bytes, row * t.stride); }
__device__ inline float exp_of(float difference) { return __builtin_amdgcn_exp2f(difference * kLog2e); }
// a row's weight, 0 for padding
__device__ inline float row_weight(const Targets& t, const float* weight, int64_t V, int64_t row) {
    const int64_t c = target_of(t, row);
    return c < 0 || c >= V ? 0.f : weight ? weight[row] : 1.f;
}

// what a tile leaves of a row: the largest logit of those that are not the target's,
// and their sum of exp(logit - largest)
struct Piece {
    float top, sum;
};

// ---- the product with its statistics

template <typename T, int FM, int FN, int WM, int WN, bool KEEP>
__global__ __launch_bounds__(WM* WN* kWave) void logits_kernel(Operand W, Operand X, int64_t steps, float scale, Targets t,
                                                               int64_t tm, int64_t tn, Piece* __restrict__ pieces,
                                                               float* __restrict__ hit, T* __restrict__ E,
                                                               int64_t lde) {
    using P = TileProduct<T, FM, FN, WM, WN>;
    __shared__ __align__(1024) unsigned char buf0[P::BUFFER], buf1[P::BUFFER];
    __shared__ float part[2][WM][P::BN];
    const TileAt at = tile_at(blockIdx.x, tm, tn);
    const int64_t m0 = int64_t(at.m) * P::BM, n0 = int64_t(at.n) * P::BN;
    F4 acc[FM][FN] = {};
    P::run(W, X, m0, n0, steps, 0, buf0, buf1, acc);

    const int lane = lane_id(), w = threadIdx.x / kWave, wm = w / WN, wn = w % WN;
    // this lane's columns of W in the tile: mine + 16 i + r
    const int mine = wm * FM * 16 + 4 * (lane >> 4), valid = int(min(W.rows - m0, int64_t(P::BM)));
    const int64_t mw = m0 + mine;
    const int col = wn * FN * 16 + (lane & 15);
    float top[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        __builtin_amdgcn_sched_barrier(0);
        const int64_t n = n0 + col + j * 16;
        const int64_t target = n < X.rows ? target_of(t, n) - m0 : -1;
        const int at_target = target >= 0 && target < valid ? int(target) - mine : -1;
        float mx = -__builtin_huge_valf();
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i][j][r] *= scale;
        if (valid < P::BM)
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (mine + i * 16 + r >= valid) acc[i][j][r] = -__builtin_huge_valf();
        // (few tiles hold a target of a wavefront's rows)
        if (__any(at_target >= 0)) {
            float h = 0.f;
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (at_target == i * 16 + r) {
                        h = acc[i][j][r];
                        acc[i][j][r] = -__builtin_huge_valf();
                    }
            if (at_target >= 0 && at_target < FM * 16 && (at_target & 15) < 4) hit[n] = h;
        }
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) mx = fmaxf(mx, acc[i][j][r]);
        mx = fmaxf(mx, __shfl_xor(mx, 16, kWave));
        top[j] = fmaxf(mx, __shfl_xor(mx, 32, kWave));
        if (lane < 16) part[0][wm][col + j * 16] = top[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        float mx = -3.402823466e38f;
#pragma unroll
        for (int q = 0; q < WM; ++q) mx = fmaxf(mx, part[0][q][col + j * 16]);
        top[j] = mx;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float e = exp_of(acc[i][j][r] - mx);
                acc[i][j][r] = e;
                s += e;
            }
        s += __shfl_xor(s, 16, kWave);
        s += __shfl_xor(s, 32, kWave);
        if (lane < 16) part[1][wm][col + j * 16] = s;
    }
    __syncthreads();
    for (int q = threadIdx.x; q < P::BN; q += P::THREADS) {
        const int64_t n = n0 + q;
        if (n >= X.rows) break;
        float mx = -3.402823466e38f, s = 0.f;
#pragma unroll
        for (int i = 0; i < WM; ++i) {
            mx = fmaxf(mx, part[0][i][q]);
            s += part[1][i][q];
        }
        pieces[n * tm + at.m] = {mx, s};
    }
    if constexpr (KEEP) {
        const float raise = __builtin_amdgcn_exp2f(kRaise<T>);
        if constexpr (sizeof(T) == 2) {
            __builtin_amdgcn_sched_barrier(0);
            store_rows<T, FM, FN, WM * WN>(acc, buf0, buf1, w, raise, [&](int n1, int m1, Vec<T, 8> v) {
                const int64_t n = n0 + wn * FN * 16 + n1, m = m0 + wm * FM * 16 + m1;
                if (n < X.rows && m < lde) store_vec<T, 8>(E + n * lde + m, v);  // (lde is a multiple of eight)
            });
        } else {
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                __builtin_amdgcn_sched_barrier(0);  // (addresses of all packs at once would spill)
                const int64_t n = n0 + col + j * 16;
                if (n >= X.rows) continue;
#pragma unroll
                for (int i = 0; i < FM; ++i) {
                    const int64_t m = mw + i * 16;
                    if (m < lde) *reinterpret_cast<F4*>(E + n * lde + m) = acc[i][j];
                }
            }
        }
    }
}

// ---- the same for few rows: one reading of W, from memory into the registers of
// the matrix instructions.  A workgroup takes kFewColumns rows of W, its wavefronts
// a quarter of k each; rows of any alignment, past their ends zeros.  Bound by W's
// bytes (32000 x 2048 bf16, one row: 22 us, 5.9 TB/s; of W eight steps under way, 27.2
// us a call, four 27.7 and two 28.0; with loads that pass the caches by 35.7, of 31.9
// then).

constexpr int kFewColumns = 64, kFewRows = 64;  // a piece's columns; rows at most

// elements [c, c + N) of a row of d, zeros past its end
template <typename T, int N>
__device__ inline Vec<T, N> row_part(const T* row, int64_t c, int64_t d) {
    if (c + N <= d) return load_vec<T, N>(row + c);
    Vec<T, N> v;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = c + i < d ? row[c + i] : T(0.f);
    return v;
}

template <typename T, int NB>
__global__ __launch_bounds__(kBlock) void logits_few(const T* __restrict__ w, int64_t ldw, int64_t V,
                                                     const T* __restrict__ x, int64_t ldx, int64_t rows, int64_t d,
                                                     float scale, Targets t, int64_t tm, Piece* __restrict__ pieces,
                                                     float* __restrict__ hit) {
    constexpr int FM = kFewColumns / 16, N = 16 / int(sizeof(T)), STEP = 4 * N, AHEAD = NB == 1 ? 8 : 2;
    using C = typename Chunk<T>::V;
    __shared__ F4 sums[kWavesPerBlock][FM][NB][kWave];
    __shared__ float part[2][kWavesPerBlock][NB * 16];
    const int lane = lane_id(), wave = int(uniform(threadIdx.x / kWave)), g = lane >> 4, r16 = lane & 15;
    const int64_t m0 = int64_t(blockIdx.x) * kFewColumns;
    const T *pw[FM], *px[NB];
    bool there[NB];
#pragma unroll
    for (int i = 0; i < FM; ++i) pw[i] = w + min(m0 + i * 16 + r16, V - 1) * ldw;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        there[j] = j * 16 + r16 < rows;
        px[j] = x + (there[j] ? j * 16 + r16 : 0) * ldx;
    }
    F4 acc[FM][NB] = {};
    const int64_t steps = (d + STEP - 1) / STEP, whole = d / STEP;
    const int64_t k0 = steps * wave / kWavesPerBlock, k1 = steps * (wave + 1) / kWavesPerBlock;
    auto multiply = [&](const Vec<T, N> (&a)[FM], const Vec<T, N> (&b)[NB]) {
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const C cb = __builtin_bit_cast(C, b[j]);
#pragma unroll
            for (int i = 0; i < FM; ++i) acc[i][j] = Chunk<T>::mul(__builtin_bit_cast(C, a[i]), cb, acc[i][j]);
        }
    };
    Vec<T, N> none;
#pragma unroll
    for (int i = 0; i < N; ++i) none[i] = T(0.f);
    int64_t k = k0;
    for (; k + AHEAD <= min(k1, whole); k += AHEAD) {
        Vec<T, N> a[AHEAD][FM], b[AHEAD][NB];
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) {
            const int64_t c = (k + q) * STEP + g * N;
#pragma unroll
            for (int i = 0; i < FM; ++i) a[q][i] = load_vec<T, N>(pw[i] + c);
#pragma unroll
            for (int j = 0; j < NB; ++j) b[q][j] = there[j] ? load_vec<T, N>(px[j] + c) : none;
        }
        __builtin_amdgcn_sched_barrier(0);  // (all of them are under way before the first is used)
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) multiply(a[q], b[q]);
    }
    for (; k < k1; ++k) {
        Vec<T, N> a[FM], b[NB];
        const int64_t c = k * STEP + g * N;
#pragma unroll
        for (int i = 0; i < FM; ++i) a[i] = row_part<T, N>(pw[i], c, d);
#pragma unroll
        for (int j = 0; j < NB; ++j) b[j] = there[j] ? row_part<T, N>(px[j], c, d) : none;
        multiply(a, b);
    }
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) sums[wave][i][j][lane] = acc[i][j];
    __syncthreads();
    // (a wavefront goes on with 16 of the columns: the quarters of k in their order)
    const int64_t m = m0 + wave * 16 + 4 * g;
    F4 v[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        v[j] = sums[0][wave][j][lane];
#pragma unroll
        for (int q = 1; q < kWavesPerBlock; ++q) v[j] += sums[q][wave][j][lane];
        const int64_t n = j * 16 + r16;
        const int64_t target = n < rows ? target_of(t, n) : -1;
        float mx = -__builtin_huge_valf();
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            v[j][r] = m + r < V ? v[j][r] * scale : -__builtin_huge_valf();
            if (m + r == target && m + r < V) {
                hit[n] = v[j][r];
                v[j][r] = -__builtin_huge_valf();
            }
            mx = fmaxf(mx, v[j][r]);
        }
        mx = fmaxf(mx, __shfl_xor(mx, 16, kWave));
        mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
        if (lane < 16) part[0][wave][j * 16 + lane] = mx;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        float mx = -3.402823466e38f, s = 0.f;
#pragma unroll
        for (int q = 0; q < kWavesPerBlock; ++q) mx = fmaxf(mx, part[0][q][j * 16 + r16]);
#pragma unroll
        for (int r = 0; r < 4; ++r) s += exp_of(v[j][r] - mx);
        s += __shfl_xor(s, 16, kWave);
        s += __shfl_xor(s, 32, kWave);
        if (lane < 16) part[1][wave][j * 16 + lane] = s;
    }
    __syncthreads();
    const int64_t n = threadIdx.x;
    if (n >= min(rows, int64_t(NB * 16))) return;
    float mx = -3.402823466e38f, s = 0.f;
#pragma unroll
    for (int q = 0; q < kWavesPerBlock; ++q) {
        mx = fmaxf(mx, part[0][q][n]);
        s += part[1][q][n];
    }
    pieces[n * tm + blockIdx.x] = {mx, s};
}

__device__ inline float log_of(float v) { return __builtin_amdgcn_logf(v) * kLn2; }

// A row's pieces joined with the target's logit: loss and lse (may be null).
__global__ __launch_bounds__(kBlock) void join_pieces(const Piece* __restrict__ pieces, int64_t tm, int64_t rows,
                                                      const float* __restrict__ hit, Targets t, int64_t V,
                                                      float* __restrict__ loss, float* __restrict__ lse) {
    for (int64_t n = int64_t(blockIdx.x) * kWavesPerBlock + threadIdx.x / kWave; n < rows;
         n += int64_t(gridDim.x) * kWavesPerBlock) {
        const Piece* p = pieces + n * tm;
        // (under way beside the pieces: after them they would be waited for one by one)
        const int64_t target = target_of(t, n);
        const bool named = target >= 0 && target < V;
        const float h = named ? hit[n] : 0.f;
        float top = -3.402823466e38f, s = 0.f;
#pragma unroll 8
        for (int64_t i = lane_id(); i < tm; i += kWave) {
            const Piece q = p[i];
            const float high = fmaxf(top, q.top);
            s = s * exp_of(top - high) + q.sum * exp_of(q.top - high);
            top = high;
        }
        const float mx = wave_max(top);
        s = wave_total(s * exp_of(top - mx));
        if (lane_id() != 0) continue;
        if (!named) {
            loss[n] = 0.f;
            if (lse) lse[n] = mx + log_of(s);
            continue;
        }
        // log(1 + e^d s), by the larger of the two terms
        const float d = mx - h;
        float l, all;
        if (d <= 0.f) {
            l = log1pf(s * exp_of(d)) + (h - h);  // (of an infinite h NaN)
            all = h + l;
        } else {
            const float more = log_of(s + exp_of(-d));
            l = d + more;
            all = mx + more;
        }
        loss[n] = l;
        if (lse) lse[n] = all;
    }
}

// What G is divided by where it is held in 16 bits: the rows' largest weight, so
// that rows of one weight have G = q - onehot whatever that weight is (of 1/N,
// say, every row's target would have the same rounding), and for IEEE floats
// 2^-14 times it, which takes G's entries to their range.
__global__ __launch_bounds__(1024) void weight_unit(Targets t, const float* __restrict__ weight, int64_t V,
                                                    int64_t rows, float below, float* __restrict__ unit) {
    __shared__ float most[1024 / kWave];
    float mx = 0.f;
    for (int64_t n = threadIdx.x; n < rows; n += 1024) {
        const float w = fabsf(row_weight(t, weight, V, n));
        if (w < __builtin_huge_valf()) mx = fmaxf(mx, w);
    }
    mx = wave_max(mx);
    if (lane_id() == 0) most[threadIdx.x / kWave] = mx;
    __syncthreads();
    if (threadIdx.x) return;
    for (int i = 0; i < 1024 / kWave; ++i) mx = fmaxf(mx, most[i]);
    // (a normal number, and a weight of it or less divided by it no infinity)
    unit[0] = (mx > 0.f ? fminf(fmaxf(mx, 0x1p-100f), 0x1p127f) : 1.f) * below;
}

// ---- layouts for the products

// dst: rows of `cols` elements, zeros up to ldd, and (MASK) rows of zeros for those
// without weight
template <typename T, bool MASK>
__global__ __launch_bounds__(kBlock) void pack_rows(const T* __restrict__ src, int64_t ld, int64_t rows, int64_t cols,
                                                    T* __restrict__ dst, int64_t ldd, Targets t,
                                                    const float* __restrict__ weight, int64_t V) {
    constexpr int N = 16 / int(sizeof(T));
    const int64_t packs = ldd / N;
    for (int64_t q = int64_t(blockIdx.x) * kBlock + threadIdx.x; q < rows * packs; q += int64_t(gridDim.x) * kBlock) {
        const int64_t r = q / packs, c = q % packs * N;
        Vec<T, N> v;
        if (MASK && row_weight(t, weight, V, r) == 0.f) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = T(0.f);
        } else if (c + N <= cols) {
            v = load_vec<T, N>(src + r * ld + c);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = c + i < cols ? src[r * ld + c + i] : T(0.f);
        }
        store_vec<T, N>(dst + r * ldd + c, v);
    }
}

// G in E's place, zeros from V to lde.  piece: columns that share a base.
constexpr int kFoldPacks = 4;  // of a thread, a workgroup's width apart
template <typename T>
__global__ __launch_bounds__(kBlock) void fold(T* __restrict__ E, int64_t lde, int64_t rows, int64_t V,
                                               const Piece* __restrict__ pieces, int64_t tm, int piece,
                                               const float* __restrict__ lse, const float* __restrict__ loss,
                                               Targets t, const float* __restrict__ weight,
                                               const float* __restrict__ unit) {
    constexpr int N = 16 / int(sizeof(T)), SPAN = kBlock * kFoldPacks * N;
    const int64_t across = (lde + SPAN - 1) / SPAN;
    const int64_t r = blockIdx.x / across, c0 = blockIdx.x % across * SPAN + threadIdx.x * N;
    const float w = row_weight(t, weight, V, r) / (unit ? unit[0] : 1.f);
    T* row = E + r * lde;
    Vec<T, N> e[kFoldPacks];
    float f[kFoldPacks];
    if (w != 0.f) {
        const float l = lse[r];
#pragma unroll
        for (int q = 0; q < kFoldPacks; ++q) {
            const int64_t c = c0 + q * kBlock * N;
            if (c >= lde) break;
            e[q] = load_vec<T, N>(row + c);
            f[q] = w * __builtin_amdgcn_exp2f((pieces[r * tm + min(c, V - 1) / piece].top - l) * kLog2e - kRaise<T>);
        }
    }
    const int64_t target = w != 0.f ? target_of(t, r) : -1;
#pragma unroll
    for (int q = 0; q < kFoldPacks; ++q) {
        const int64_t c = c0 + q * kBlock * N;
        if (c >= lde) break;
        Vec<T, N> o;
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = w != 0.f && c + i < V ? T(float(e[q][i]) * f[q]) : T(0.f);
        if (target >= c && target < c + N) {
            const T g = T(w * expm1f(-loss[r]));
#pragma unroll
            for (int i = 0; i < N; ++i) o[i] = c + i == target ? g : o[i];
        }
        store_vec<T, N>(row + c, o);
    }
}

// ---- plain products

// Products of a turned A (W, or the rows of x that count) with B in rows of k (G) or
// turned too.  What becomes of out[n][m]: rounded to T (kStore), a part of k as 32-bit
// floats (kPart, part z behind rows x ldo each), or added to 32-bit floats
// (kAdd; the first addition writes), the last time rounded to T as well.
enum Into { kStore, kPart, kAdd };
struct Product {
    void* out = nullptr;  // T
    int64_t ldo = 0;
    float alpha = 1.f;
    const float* unit = nullptr;  // times unit[0]
    Targets t;                    // with t.p: rows n without weight are zeros
    const float* weight = nullptr;
    int64_t V = 0;
    float* sums = nullptr;  // kPart, kAdd: rows of lds floats
    int64_t lds = 0, plane = 0;
    bool first = true, last = true;  // kAdd
};

template <typename T>
__device__ inline void store_four(const Product& o, int64_t n, int64_t m, int64_t M, float alpha, bool keep, F4 v) {
    T* p = static_cast<T*>(o.out) + n * o.ldo + m;
    Vec<T, 4> q;
#pragma unroll
    for (int r = 0; r < 4; ++r) q[r] = keep ? T(v[r] * alpha) : T(0.f);
    if (m + 4 <= M) {
        store_vec<T, 4>(p, q);
    } else {
        for (int r = 0; r < 4; ++r)
            if (m + r < M) p[r] = q[r];
    }
}

template <typename T, int FM, int FN, int WM, int WN, bool TB, int INTO>
__global__ __launch_bounds__(WM* WN* kWave) void product_kernel(Operand A, Operand B, int64_t steps, int64_t per,
                                                                int64_t tm, int64_t tn, Product o) {
    using P = TileProduct<T, FM, FN, WM, WN, true, TB>;
    __shared__ __align__(1024) unsigned char buf0[P::BUFFER], buf1[P::BUFFER];
    const TileAt at = tile_at(blockIdx.x, tm, tn);
    const int64_t m0 = int64_t(at.m) * P::BM, n0 = int64_t(at.n) * P::BN;
    const int64_t s0 = int64_t(blockIdx.y) * per;
    F4 acc[FM][FN] = {};
    P::run(A, B, m0, n0, min(per, steps - s0), s0, buf0, buf1, acc);

    const int lane = lane_id(), w = threadIdx.x / kWave, wm = w / WN, wn = w % WN;
    const float alpha = o.unit ? o.alpha * o.unit[0] : o.alpha;
    if constexpr (INTO == kStore && sizeof(T) == 2) {
        __syncthreads();  // (the buffers are free)
        store_rows<T, FM, FN, WM * WN>(acc, buf0, buf1, w, alpha, [&](int n1, int m1, Vec<T, 8> v) {
            const int64_t n = n0 + wn * FN * 16 + n1, m = m0 + wm * FM * 16 + m1;
            if (n >= B.rows || m >= A.rows) return;
            if (o.t.p && row_weight(o.t, o.weight, o.V, n) == 0.f)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = T(0.f);
            T* p = static_cast<T*>(o.out) + n * o.ldo + m;
            if (m + 8 <= A.rows) {
                store_vec<T, 8>(p, v);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (m + i < A.rows) p[i] = v[i];
            }
        });
        return;
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        __builtin_amdgcn_sched_barrier(0);  // (addresses of all packs at once would spill)
        const int64_t n = n0 + wn * FN * 16 + j * 16 + (lane & 15);
        if (n >= B.rows) continue;
        const bool keep = !o.t.p || INTO != kStore || row_weight(o.t, o.weight, o.V, n) != 0.f;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int64_t m = m0 + wm * FM * 16 + i * 16 + 4 * (lane >> 4);
            if (m >= A.rows) continue;
            if constexpr (INTO == kStore) {
                store_four<T>(o, n, m, A.rows, alpha, keep, acc[i][j]);
            } else {
                // (lds is a multiple of four)
                F4* p = reinterpret_cast<F4*>(o.sums + int64_t(blockIdx.y) * o.plane + n * o.lds + m);
                F4 v = acc[i][j];
                if (INTO == kAdd && !o.first) v += *p;
                if (INTO == kAdd && o.last)
                    store_four<T>(o, n, m, A.rows, alpha, true, v);
                else
                    *p = v;
            }
        }
    }
}

// the parts of k added in their order (64 parts of 25 x 257: 18 us with one load under
// way at a time, 7 with eight)
template <typename T>
__global__ __launch_bounds__(kBlock) void join_parts(Product o, int64_t parts, int64_t N, int64_t M) {
    const float alpha = o.unit ? o.alpha * o.unit[0] : o.alpha;
    const int64_t packs = o.lds / 4;
    for (int64_t q = int64_t(blockIdx.x) * kBlock + threadIdx.x; q < N * packs; q += int64_t(gridDim.x) * kBlock) {
        const int64_t n = q / packs, m = q % packs * 4;
        if (m >= M) continue;
        const float* p = o.sums + n * o.lds + m;
        F4 v = *reinterpret_cast<const F4*>(p);
#pragma unroll 8
        for (int64_t i = 1; i < parts; ++i) v += *reinterpret_cast<const F4*>(p + i * o.plane);
        const bool keep = !o.t.p || row_weight(o.t, o.weight, o.V, n) != 0.f;
        store_four<T>(o, n, m, M, alpha, keep, v);
    }
}

// Tiles of m by n.  16-bit products go by 256 x 256 and eight wavefronts where such
// tiles fill three quarters of the chip (8192 x 131072 x 4096 bf16: 6.25 ms, by the
// others 7.89), else by 128 x 128 and four.  Where k can be split, its parts count
// as tiles (2047 x 1001 x 50021 f16: 197 us with eight parts, 237 by small tiles),
// unless large tiles would be padded by a quarter more.  32-bit products, whose
// fragments feed the matrix cores four times as long, go by small tiles, which leave
// less of the last round idle (1001 x 50021 x 250: 244 us, 288 by large ones; 300 x
// 100000 x 2048: 0.98 ms and 1.90; but 2048 x 32768 x 1024, whole rounds of either:
// 1.00 and 0.97), or by 128 x 64 where the busiest compute unit has less to do by
// those (217 x 36096 x 1472: 235 us, 274 by 128 x 128; 25 x 44003 x 257 with its
// gradient: 112 and 155).
struct Tile {
    int m, n;
};
constexpr Tile kLarge{256, 256}, kSmall{128, 128}, kSlim{128, 64};
inline int64_t tiles_of(int64_t M, int64_t N, Tile t) { return ceil_div(M, t.m) * ceil_div(N, t.n); }
// parts of k that fill the chip with tiles, each of eight steps at least
inline int64_t parts_of(int64_t M, int64_t N, int64_t steps, Tile t) {
    const int64_t tiles = tiles_of(M, N, t), room = t.m == kLarge.m ? kCus : 2 * kCus;
    if (tiles == 0 || 2 * tiles > room) return 1;
    return std::max<int64_t>(1, std::min<int64_t>({room / tiles, steps / 8, 64}));
}
inline Tile tile_of(int64_t M, int64_t N, int dt, int64_t split_steps = 0) {
    if (dt == kDtF32) {
        auto busiest = [&](Tile t) {
            const int64_t parts = split_steps ? parts_of(M, N, split_steps, t) : 1;
            return ceil_div(tiles_of(M, N, t) * parts, kCus) * ceil_div(std::max<int64_t>(split_steps, 1), parts) * t.n;
        };
        return busiest(kSlim) < busiest(kSmall) ? kSlim : kSmall;
    }
    const int64_t large = tiles_of(M, N, kLarge), small = tiles_of(M, N, kSmall);
    const int64_t parts = split_steps ? parts_of(M, N, split_steps, kLarge) : 1;
    if (parts > 1 && 16 * large > 5 * small) return kSmall;
    return large * parts >= kCus * 3 / 4 ? kLarge : kSmall;
}

// f(fragments of A and of B, wavefronts along A and along B) of a tile
template <typename T, typename F>
void by_tile(Tile t, F f) {
    using std::integral_constant;
    using Two = integral_constant<int, 2>;
    using Four = integral_constant<int, 4>;
    if constexpr (sizeof(T) == 2) {
        if (t.m == kLarge.m) return f(integral_constant<int, 8>(), Four(), Two(), Four());
    } else {
        if (t.n == kSlim.n) return f(Four(), Two(), Two(), Two());
    }
    f(Four(), Four(), Two(), Two());
}

template <typename T, bool KEEP>
void launch_logits(const Operand& W, const Operand& X, int64_t steps, float scale, const Targets& t, Tile tile,
                   Piece* pieces, float* hit, T* E, int64_t lde, hipStream_t s) {
    by_tile<T>(tile, [&](auto fm, auto fn, auto wm, auto wn) {
        constexpr int FM = decltype(fm)::value, FN = decltype(fn)::value, WM = decltype(wm)::value,
                      WN = decltype(wn)::value;
        const int64_t tm = ceil_div(W.rows, tile.m), tn = ceil_div(X.rows, tile.n);
        logits_kernel<T, FM, FN, WM, WN, KEEP><<<unsigned(tm * tn), WM * WN * kWave, 0, s>>>(
            W, X, steps, scale, t, tm, tn, pieces, hit, E, lde);
    });
}

template <typename T, bool TB, int INTO>
void launch_product(const Operand& A, const Operand& B, int64_t steps, int64_t parts, Tile tile, const Product& o,
                    hipStream_t s) {
    by_tile<T>(tile, [&](auto fm, auto fn, auto wm, auto wn) {
        constexpr int FM = decltype(fm)::value, FN = decltype(fn)::value, WM = decltype(wm)::value,
                      WN = decltype(wn)::value;
        const int64_t tm = ceil_div(A.rows, tile.m), tn = ceil_div(B.rows, tile.n);
        product_kernel<T, FM, FN, WM, WN, TB, INTO><<<dim3(unsigned(tm * tn), unsigned(parts)), WM * WN * kWave, 0, s>>>(
            A, B, steps, ceil_div(steps, parts), tm, tn, o);
    });
}

inline unsigned grid_of(int64_t items) { return unsigned(std::min<int64_t>(ceil_div(items, kBlock), 16 * kCus)); }

// ---- a call's workspace, laid out once for its size and once for its use

struct Carver {
    char* base;
    size_t used = 0;
    template <typename T>
    T* get(int64_t count) {
        T* p = base ? reinterpret_cast<T*>(base + used) : nullptr;
        used += (size_t(count) * sizeof(T) + 1023) & ~size_t(1023);
        return p;
    }
};

inline Targets from_row(Targets t, int64_t row) {
    t.p = static_cast<const char*>(t.p) + row * t.stride * t.bytes;
    return t;
}

constexpr int64_t kKeptBytes = int64_t(2) << 30;  // exponentials of the rows taken at a time, at most

template <typename T, bool MASK>
Operand packed(const DenseRows& x, T* p, int64_t ld, const Targets& t, const float* weight, int64_t V, hipStream_t s) {
    if (x.m > 0)
        pack_rows<T, MASK><<<grid_of(x.m * ld * int64_t(sizeof(T)) / 16), kBlock, 0, s>>>(
            static_cast<const T*>(x.p), x.ld, x.m, x.n, p, ld, t, weight, V);
    return {p, ld, x.m, 0};
}
// rows as an operand: as they are, or packed to whole steps
inline bool as_they_are(const DenseRows& x) {
    return on_boundaries(x.p, x.ld, x.dt) && x.n % step_elements(x.dt) == 0 &&
           x.ld * dtype_bytes(x.dt) < kMostStride;
}
template <typename T>
Operand operand_rows(const DenseRows& x, Carver& c, hipStream_t s) {
    if (as_they_are(x)) return {x.p, x.ld, x.m, 0};
    const int64_t ld = round_up(x.n, kStepBytes / int64_t(sizeof(T)));
    T* p = c.get<T>(x.m * ld);
    if (!c.base) return {nullptr, ld, x.m, 0};
    return packed<T, false>(x, p, ld, Targets(), nullptr, 0, s);
}
// the same memory with its rows as the depth of a product
inline Operand turned(const Operand& o, int64_t columns) { return {o.p, o.ld, columns, o.rows}; }

// Whether the loss of some rows goes by one reading of W (kernel above): up to 16;
// up to 64 where W would have to be packed for the tiles, or makes too few of them
// (32 rows of 2000 x 2048 bf16: 17 us, tiles 23; 24 of 50021 x 1001 f16: 53 and 67,
// though 64 of them 77 and 68; but 64 of 131072 x 4096 bf16: 303 and 223, 32 of
// 32000 x 2048: 32.4 and 31.3; in 32 bits 24 of 50021 x 1024: 70 and 72, 64: 116 and
// 74).
inline bool few_rows(const DenseRows& X, const DenseRows& W) {
    if (X.m <= (X.dt == kDtF32 ? 32 : 16)) return true;
    return X.m <= kFewRows && (!as_they_are(W) || 4 * ceil_div(W.m, kSmall.m) < 3 * kCus);
}

template <typename T>
size_t cross_entropy(const DenseRows& X, const DenseRows& W, const Targets& t, float scale, float* loss, float* lse,
                     char* tmp, hipStream_t s) {
    Carver c{tmp};
    if (few_rows(X, W)) {
        const int64_t tm = ceil_div(W.m, kFewColumns);
        Piece* pieces = c.get<Piece>(X.m * tm);
        float* hit = c.get<float>(X.m);
        if (!tmp) return c.used;
        auto few = [&](auto nb) {
            logits_few<T, decltype(nb)::value><<<unsigned(tm), kBlock, 0, s>>>(
                static_cast<const T*>(W.p), W.ld, W.m, static_cast<const T*>(X.p), X.ld, X.m, X.n, scale, t, tm, pieces,
                hit);
        };
        if (X.m <= 16)
            few(std::integral_constant<int, 1>());
        else if (X.m <= 32)
            few(std::integral_constant<int, 2>());
        else
            few(std::integral_constant<int, 4>());
        join_pieces<<<grid_of(X.m * kWave), kBlock, 0, s>>>(pieces, tm, X.m, hit, t, W.m, loss, lse);
        return 0;
    }
    const Operand x = operand_rows<T>(X, c, s), w = operand_rows<T>(W, c, s);
    // rows at a time: 256 MB of pieces at most, but 256 rows at least (16 V bytes of them)
    const int64_t chunk =
        std::max<int64_t>(kLarge.m, std::min(X.m, (int64_t(1) << 25) / ceil_div(W.m, kSmall.m) / kLarge.m * kLarge.m));
    const int64_t most = std::min(X.m, chunk);
    Piece* pieces = c.get<Piece>(most * ceil_div(W.m, kSmall.m));
    float* hit = c.get<float>(most);
    if (!tmp) return c.used;
    const int64_t steps = ceil_div(X.n, kStepBytes / int(sizeof(T)));
    for (int64_t r0 = 0; r0 < X.m; r0 += chunk) {
        const int64_t n = std::min(chunk, X.m - r0);
        const Operand xr{static_cast<const T*>(x.p) + r0 * x.ld, x.ld, n, 0};
        const Targets tr = from_row(t, r0);
        const Tile tile = tile_of(W.m, n, W.dt);
        launch_logits<T, false>(w, xr, steps, scale, tr, tile, pieces, hit, nullptr, 0, s);
        join_pieces<<<grid_of(n * kWave), kBlock, 0, s>>>(pieces, ceil_div(W.m, tile.m), n, hit, tr, W.m, loss + r0,
                                                         lse ? lse + r0 : nullptr);
    }
    return 0;
}

template <typename T>
size_t cross_entropy_grad(const DenseRows& X, const DenseRows& W, const Targets& t, float scale, const float* weight,
                          float* loss, const DenseRows& dX, const DenseRows& dW, char* tmp, hipStream_t s) {
    constexpr int64_t STEP = kStepBytes / int(sizeof(T));
    const int64_t V = W.m, D = W.n, Vp = round_up(V, STEP);
    // rows at a time: whole tiles
    const int64_t chunk =
        std::max<int64_t>(kLarge.m, std::min({round_up(X.m, kLarge.m), kKeptBytes / int64_t(sizeof(T)) / Vp / kLarge.m * kLarge.m,
                                           int64_t(1) << 17}));
    const int64_t chunks = ceil_div(X.m, chunk), most = std::min(X.m, chunk);
    Carver c{tmp};
    const Operand x = operand_rows<T>(X, c, s), w = operand_rows<T>(W, c, s);
    Piece* pieces = c.get<Piece>(most * ceil_div(V, kSmall.m));
    float *hit = c.get<float>(most), *lse = c.get<float>(most), *unit = c.get<float>(1);
    T* E = c.get<T>(most * Vp);
    const int64_t xld = round_up(D, 16 / int64_t(sizeof(T)));
    T* XM = c.get<T>(most * xld);
    const int64_t sumld = round_up(D, 4), steps_v = Vp / STEP;
    float* sums = chunks > 1 ? c.get<float>(V * sumld) : nullptr;
    // (parts of dX's products: of whole turns, and of the last one)
    auto dx_parts = [&](int64_t n) { return parts_of(D, n, steps_v, tile_of(D, n, W.dt, steps_v)); };
    auto dx_floats = [&](int64_t n) { return dx_parts(n) > 1 ? dx_parts(n) * n * sumld : 0; };
    const int64_t rest = X.m - (chunks - 1) * chunk;
    float* dxparts = c.get<float>(chunks ? std::max(dx_floats(most), dx_floats(rest)) : 0);
    if (!tmp) return c.used;

    constexpr bool HALF = sizeof(T) == 2;
    if (HALF)
        weight_unit<<<1, 1024, 0, s>>>(t, weight, V, X.m, std::is_same<T, _Float16>::value ? 0x1p-14f : 1.f, unit);
    Product out;
    out.alpha = scale;
    out.unit = HALF ? unit : nullptr;
    for (int64_t r0 = 0; r0 < X.m || r0 == 0; r0 += chunk) {
        const int64_t n = std::min(chunk, X.m - r0);
        const Targets tr = from_row(t, r0);
        const float* wr = weight ? weight + r0 : nullptr;
        DenseRows xr = X;
        xr.m = n;
        xr.p = static_cast<char*>(X.p) + r0 * X.ld * int64_t(sizeof(T));
        if (n > 0) {
            const Operand xo{static_cast<const T*>(x.p) + r0 * x.ld, x.ld, n, 0};
            const Tile here = tile_of(V, n, W.dt);
            const int64_t tm = ceil_div(V, here.m);
            launch_logits<T, true>(w, xo, ceil_div(D, STEP), scale, tr, here, pieces, hit, E, Vp, s);
            join_pieces<<<grid_of(n * kWave), kBlock, 0, s>>>(pieces, tm, n, hit, tr, V, loss + r0, lse);
            const int64_t span = kBlock * kFoldPacks * 16 / int64_t(sizeof(T));
            fold<T><<<unsigned(n * ceil_div(Vp, span)), kBlock, 0, s>>>(E, Vp, n, V, pieces, tm, here.m, lse, loss + r0,
                                                                       tr, wr, out.unit);
            // dx = G W
            Product dx = out;
            dx.out = static_cast<T*>(dX.p) + r0 * dX.ld;
            dx.ldo = dX.ld;
            dx.t = tr;
            dx.weight = wr;
            dx.V = V;
            const Operand g{E, Vp, n, 0}, wt = turned(w, D);
            const int64_t p = dx_parts(n);
            const Tile tile = tile_of(D, n, W.dt, steps_v);
            if (p > 1) {
                dx.sums = dxparts;
                dx.lds = sumld;
                dx.plane = n * sumld;
                launch_product<T, false, kPart>(wt, g, steps_v, p, tile, dx, s);
                join_parts<T><<<grid_of(n * sumld / 4), kBlock, 0, s>>>(dx, p, n, D);
            } else {
                launch_product<T, false, kStore>(wt, g, steps_v, 1, tile, dx, s);
            }
        }
        // dW = G^T x
        Product dw = out;
        dw.out = dW.p;
        dw.ldo = dW.ld;
        dw.sums = sums;
        dw.lds = sumld;
        dw.first = r0 == 0;
        dw.last = r0 + chunk >= X.m;
        const Operand xt = turned(packed<T, true>(xr, XM, xld, tr, wr, V, s), D), gt{E, Vp, V, n};
        const Tile tile = tile_of(D, V, W.dt);
        if (sums)
            launch_product<T, true, kAdd>(xt, gt, ceil_div(n, STEP), 1, tile, dw, s);
        else
            launch_product<T, true, kStore>(xt, gt, ceil_div(n, STEP), 1, tile, dw, s);
    }
    return 0;
}

}  // namespace

size_t linear_cross_entropy_tmp_bytes(const DenseRows& X, const DenseRows& W) {
    size_t bytes = 0;
    by_dtype(X.dt, [&](auto e) {
        bytes = cross_entropy<decltype(e)>(X, W, Targets(), 1.f, nullptr, nullptr, nullptr, nullptr);
    });
    return bytes;
}

void linear_cross_entropy(const DenseRows& X, const DenseRows& W, const Targets& t, float scale, float* loss,
                          float* lse, void* tmp, hipStream_t s) {
    by_dtype(X.dt, [&](auto e) {
        cross_entropy<decltype(e)>(X, W, t, scale, loss, lse, static_cast<char*>(tmp), s);
    });
}

size_t linear_cross_entropy_grad_tmp_bytes(const DenseRows& X, const DenseRows& W) {
    size_t bytes = 0;
    by_dtype(X.dt, [&](auto e) {
        bytes = cross_entropy_grad<decltype(e)>(X, W, Targets(), 1.f, nullptr, nullptr, DenseRows(), DenseRows(),
                                                nullptr, nullptr);
    });
    return bytes;
}

void linear_cross_entropy_grad(const DenseRows& X, const DenseRows& W, const Targets& t, float scale,
                               const float* weight, float* loss, const DenseRows& dX, const DenseRows& dW, void* tmp,
                               hipStream_t s) {
    by_dtype(X.dt, [&](auto e) {
        cross_entropy_grad<decltype(e)>(X, W, t, scale, weight, loss, dX, dW, static_cast<char*>(tmp), s);
    });
}

}  // namespace spsyrk
