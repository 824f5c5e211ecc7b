// An AdamW step over many tensors.
//
//     m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
//     w = w - lr decay w - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps).
//
// Bound by bytes: parameter, gradient and states are read once, parameter and
// states written once.  The tensors' addresses travel in the launch's arguments,
// so a call needs no memory of its own and can be captured; a workgroup finds
// its tensor among them by its number.
//
// States in 8 bits: kAdamBlock elements of a tensor share a scale S, their
// largest magnitude after the step; m = sign (c / 127)^2 S with c from -127 to
// 127, v = (c / 255)^4 S with c from 0 to 255: small values get finer steps, and
// sqrt(v), which the update divides by, the same ones as m.  A v above zero has
// c of at least 1, so that no update divides by a lost denominator.  Codes are
// the nearest in c, decided in 64 bits against the border half-way between two
// codes, so that they are those of the formula however a sum was ordered.
#include <algorithm>
#include <cmath>

#include "internal.h"
#include "training.h"

namespace spsyrk {
namespace {

constexpr int kAt = 8;                        // elements per thread and turn: 16 bytes of the shortest type
constexpr int kChunk = kBlock * kAt;          // elements of a workgroup
constexpr int kTensors = 56;                  // in a launch's arguments (4 KB)
static_assert(kAdamBlock == 32 * kAt, "half a wavefront holds the elements of a scale");

struct Batch {
    AdamTensor t[kTensors];
    uint32_t first[kTensors + 1];  // workgroup that a tensor starts with
    int count;
};
static_assert(sizeof(Batch) + sizeof(AdamRates) + 16 <= 4096, "launch arguments");

__device__ inline int tensor_of(const Batch& b) {
    int lo = 0, hi = b.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (b.first[mid] <= blockIdx.x)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

// up to kAt elements from i on; those past n are `none`
template <typename T>
__device__ inline void load_some(const T* p, int64_t i, int64_t n, float (&out)[kAt]) {
    constexpr int N = std::min(kAt, 16 / int(sizeof(T)));
    if (i + kAt <= n) {
#pragma unroll
        for (int q = 0; q < kAt / N; ++q) {
            const Vec<T, N> v = load_vec_nt<T, N>(p + i + q * N);
#pragma unroll
            for (int k = 0; k < N; ++k) out[q * N + k] = float(v[k]);
        }
    } else {
#pragma unroll
        for (int k = 0; k < kAt; ++k) out[k] = i + k < n ? float(p[i + k]) : 0.f;
    }
}
template <typename T>
__device__ inline void store_some(T* p, int64_t i, int64_t n, const float (&v)[kAt]) {
    constexpr int N = std::min(kAt, 16 / int(sizeof(T)));
    if (i + kAt <= n) {
#pragma unroll
        for (int q = 0; q < kAt / N; ++q) {
            Vec<T, N> o;
#pragma unroll
            for (int k = 0; k < N; ++k) o[k] = T(v[q * N + k]);
            store_vec_nt<T, N>(p + i + q * N, o);
        }
    } else {
#pragma unroll
        for (int k = 0; k < kAt; ++k)
            if (i + k < n) p[i + k] = T(v[k]);
    }
}

// The parameters after the step, from the states after it.
__device__ inline float stepped(float w, float m, float v, const AdamRates& r) {
    return fmaf(-r.lr_decay, w, w) - r.lr_m * m / (sqrtf(v * r.inv_v) + r.eps);
}

template <typename P, bool MASTER>
__device__ inline void load_parameters(const AdamTensor& t, int64_t i, float (&w)[kAt]) {
    if constexpr (MASTER)
        load_some(t.master, i, t.n, w);
    else
        load_some(static_cast<const P*>(t.p), i, t.n, w);
}
template <typename P, bool MASTER>
__device__ inline void store_parameters(const AdamTensor& t, int64_t i, const float (&w)[kAt]) {
    if constexpr (MASTER) store_some(t.master, i, t.n, w);
    store_some(static_cast<P*>(t.p), i, t.n, w);
}

template <typename P, typename G, bool MASTER>
__global__ __launch_bounds__(kBlock) void adamw_wide(Batch b, AdamRates r) {
    const int k = tensor_of(b);
    const AdamTensor t = b.t[k];
    const int64_t i = int64_t(blockIdx.x - b.first[k]) * kChunk + int64_t(threadIdx.x) * kAt;
    if (i >= t.n) return;
    float w[kAt], g[kAt], m[kAt], v[kAt];
    load_some(static_cast<const G*>(t.g), i, t.n, g);
    load_some(static_cast<const float*>(t.m), i, t.n, m);
    load_some(static_cast<const float*>(t.v), i, t.n, v);
    load_parameters<P, MASTER>(t, i, w);
    const float gs = r.grad_scale ? r.grad_scale[0] : 1.f;
#pragma unroll
    for (int q = 0; q < kAt; ++q) {
        const float x = g[q] * gs;
        m[q] = fmaf(r.b1, m[q], r.a1 * x);
        v[q] = fmaf(r.b2, v[q], r.a2 * x * x);
        w[q] = stepped(w[q], m[q], v[q], r);
    }
    store_some(static_cast<float*>(t.m), i, t.n, m);
    store_some(static_cast<float*>(t.v), i, t.n, v);
    store_parameters<P, MASTER>(t, i, w);
}

// largest over 32 lanes, in every one of them
__device__ inline float half_max(float v) {
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, kWave));
    return v;
}
// whether any of the 32 lanes' flags is set
__device__ inline bool half_any(bool x) {
    const uint64_t all = __ballot(x);
    return uint32_t(lane_id() < 32 ? all : all >> 32) != 0;
}

// The code of y >= 0 for the scale S > 0: nearest in c, where y = (c / LEVELS)^POWER S.
template <int LEVELS, int POWER>
__device__ inline int code_of(double y, float S) {
    const float up = S < 0x1p-60f ? 0x1p80f : 1.f;  // (so that S has a reciprocal)
    float x = float(y * up) * __builtin_amdgcn_rcpf(S * up);
    x = sqrtf(x);
    if constexpr (POWER == 4) x = sqrtf(x);
    const int c = min(int(rintf(x * LEVELS)), LEVELS);
    // the border below c and the one above it, in 64 bits
    auto border = [&](double c2) {
        double q = c2 * (1.0 / LEVELS);
        q *= q;
        if constexpr (POWER == 4) q *= q;
        return q * double(S);
    };
    if (c < LEVELS && y > border(c + 0.5)) return c + 1;
    if (c > 0 && y < border(c - 0.5)) return c - 1;
    return c;
}

__device__ inline double value_m(int c, float S) {
    const double q = c * (1.0 / 127);
    return q * fabs(q) * double(S);
}
__device__ inline double value_v(int c, float S) {
    double q = c * (1.0 / 255);
    q *= q;
    return q * q * double(S);
}

template <typename C>
__device__ inline void load_codes(const C* p, int64_t i, int64_t n, int (&out)[kAt]) {
    if (i + kAt <= n) {
        const Vec<C, kAt> v = *reinterpret_cast<const Vec<C, kAt>*>(p + i);
#pragma unroll
        for (int k = 0; k < kAt; ++k) out[k] = v[k];
    } else {
#pragma unroll
        for (int k = 0; k < kAt; ++k) out[k] = i + k < n ? p[i + k] : 0;
    }
}
template <typename C>
__device__ inline void store_codes(C* p, int64_t i, int64_t n, const int (&v)[kAt]) {
    if (i + kAt <= n) {
        Vec<C, kAt> o;
#pragma unroll
        for (int k = 0; k < kAt; ++k) o[k] = C(v[k]);
        *reinterpret_cast<Vec<C, kAt>*>(p + i) = o;
    } else {
#pragma unroll
        for (int k = 0; k < kAt; ++k)
            if (i + k < n) p[i + k] = C(v[k]);
    }
}

template <typename P, typename G, bool MASTER>
__global__ __launch_bounds__(kBlock) void adamw_narrow(Batch b, AdamRates r) {
    const int k = tensor_of(b);
    const AdamTensor t = b.t[k];
    const int64_t i = int64_t(blockIdx.x - b.first[k]) * kChunk + int64_t(threadIdx.x) * kAt;
    const int64_t block = i / kAdamBlock;
    const bool there = block * kAdamBlock < t.n;  // (the same for all that share a scale)
    float w[kAt], g[kAt];
    int mc[kAt], vc[kAt];
    load_some(static_cast<const G*>(t.g), i, t.n, g);
    load_codes(static_cast<const int8_t*>(t.m), i, t.n, mc);
    load_codes(static_cast<const uint8_t*>(t.v), i, t.n, vc);
    load_parameters<P, MASTER>(t, i, w);
    const float ms = there ? t.m_scale[block] : 0.f, vs = there ? t.v_scale[block] : 0.f;
    const float gs = r.grad_scale ? r.grad_scale[0] : 1.f;
    double m[kAt], v[kAt];
    float most_m = 0.f, most_v = 0.f;
    bool bad = false;
#pragma unroll
    for (int q = 0; q < kAt; ++q) {
        const double x = double(g[q]) * double(gs);
        m[q] = fma(r.d1, value_m(mc[q], ms), (1.0 - r.d1) * x);
        v[q] = fma(r.d2, value_v(vc[q], vs), (1.0 - r.d2) * (x * x));
        if (i + q >= t.n) m[q] = v[q] = 0.0;
        const float fm = float(m[q]), fv = float(v[q]);
        bad = bad || !(fabsf(fm) < __builtin_huge_valf()) || !(fv < __builtin_huge_valf());
        most_m = fmaxf(most_m, fabsf(fm));
        most_v = fmaxf(most_v, fv);
        w[q] = stepped(w[q], fm, fv, r);
    }
    most_m = half_max(most_m);
    most_v = half_max(most_v);
    if (half_any(bad)) most_m = most_v = __builtin_nanf("");  // (a scale of NaN: all its values are)
#pragma unroll
    for (int q = 0; q < kAt; ++q) {
        mc[q] = most_m > 0.f ? code_of<127, 2>(fabs(m[q]), most_m) : 0;
        if (m[q] < 0.0) mc[q] = -mc[q];
        vc[q] = most_v > 0.f ? code_of<255, 4>(v[q], most_v) : 0;
        if (v[q] > 0.0 && most_v > 0.f) vc[q] = max(vc[q], 1);
    }
    if (i < t.n) {
        store_codes(static_cast<int8_t*>(t.m), i, t.n, mc);
        store_codes(static_cast<uint8_t*>(t.v), i, t.n, vc);
        store_parameters<P, MASTER>(t, i, w);
    }
    if (there && i % kAdamBlock == 0) {
        t.m_scale[block] = most_m;
        t.v_scale[block] = most_v;
    }
}

// the values that 8-bit states stand for, into 32-bit floats (t.p for m, t.master for v)
__global__ __launch_bounds__(kBlock) void adam_values_kernel(Batch b) {
    const int k = tensor_of(b);
    const AdamTensor t = b.t[k];
    const int64_t i = int64_t(blockIdx.x - b.first[k]) * kChunk + int64_t(threadIdx.x) * kAt;
    if (i >= t.n) return;
    int mc[kAt], vc[kAt];
    load_codes(static_cast<const int8_t*>(t.m), i, t.n, mc);
    load_codes(static_cast<const uint8_t*>(t.v), i, t.n, vc);
    const float ms = t.m_scale[i / kAdamBlock], vs = t.v_scale[i / kAdamBlock];
    float m[kAt], v[kAt];
#pragma unroll
    for (int q = 0; q < kAt; ++q) {
        m[q] = float(value_m(mc[q], ms));
        v[q] = float(value_v(vc[q], vs));
    }
    store_some(static_cast<float*>(t.p), i, t.n, m);
    store_some(t.master, i, t.n, v);
}

// f(batch, workgroups) over the tensors, as many at a time as the arguments hold
template <typename F>
void by_batch(const AdamTensor* t, int64_t count, F f) {
    Batch b;
    b.count = 0;
    int64_t blocks = 0;
    auto flush = [&] {
        if (b.count) {
            for (int q = b.count; q <= kTensors; ++q) b.first[q] = uint32_t(blocks);
            f(b, unsigned(blocks));
        }
        b.count = 0;
        blocks = 0;
    };
    for (int64_t q = 0; q < count; ++q) {
        if (t[q].n <= 0) continue;
        const int64_t more = (t[q].n + kChunk - 1) / kChunk;
        // (a launch has fewer than 2^24 workgroups, 2^32 threads)
        if (b.count == kTensors || (b.count && blocks + more >= (int64_t(1) << 23))) flush();
        b.first[b.count] = uint32_t(blocks);
        b.t[b.count++] = t[q];
        blocks += more;
    }
    flush();
}

}  // namespace

void adamw(const AdamTensor* t, int64_t count, int param_dtype, int grad_dtype, int bits, bool master,
           const AdamRates& r, hipStream_t s) {
    by_batch(t, count, [&](const Batch& b, unsigned blocks) {
        by_dtype(param_dtype, [&](auto e) {
            using P = decltype(e);
            auto launch = [&](auto gt, auto wide) {
                using G = decltype(gt);
                constexpr bool MASTER = decltype(wide)::value;
                if (bits == 32)
                    adamw_wide<P, G, MASTER><<<blocks, kBlock, 0, s>>>(b, r);
                else
                    adamw_narrow<P, G, MASTER><<<blocks, kBlock, 0, s>>>(b, r);
            };
            const std::integral_constant<bool, false> no;
            const std::integral_constant<bool, true> yes;
            if constexpr (sizeof(P) == 4) {
                launch(float(), no);
            } else if (grad_dtype == kDtF32) {
                if (master)
                    launch(float(), yes);
                else
                    launch(float(), no);
            } else {
                if (master)
                    launch(P(), yes);
                else
                    launch(P(), no);
            }
        });
    });
}

void adam_values(const AdamTensor* t, int64_t count, hipStream_t s) {
    by_batch(t, count, [&](const Batch& b, unsigned blocks) { adam_values_kernel<<<blocks, kBlock, 0, s>>>(b); });
}

}  // namespace spsyrk
