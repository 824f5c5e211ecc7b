// An AdamW step over many tensors.
//
//     m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
//     w = w - lr decay w - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps).
//
// Bound by bytes: parameter, gradient and states are read once, parameter and
// states written once.  The tensors' addresses travel in the launch's arguments,
// so a call needs no memory of its own and can be captured; a workgroup finds
// its tensor among them by its number.  160 M elements of bf16 with copies and
// states in 32 bits: 880 us, 5.1 TB/s; 64 M with states in 8: 172 us, 3.7 TB/s
// (each pack's scale is known only when all of it is summed, and the codes' roots
// and comparisons follow before its stores).
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

constexpr int kAt = 4;  // elements of a pack: 16 bytes of 32-bit floats
// Packs of a thread, a workgroup's width apart, and threads of a workgroup.  States
// of 32 bits: the widest chunks are read and written fastest (160 M elements of
// bf16 with copies: 965 us by 128 threads, 896 by 256, 888 by 1024; two packs a
// thread 988).  Of 8 bits, where a wavefront's arithmetic counts, two packs by
// 256 threads (64 M, with the values: 260 us, by 1024 threads 296; one pack, which took
// 10 us more before values next to a border had one comparison, 256).
template <bool NARROW>
constexpr int kPacks = NARROW ? 2 : 1;
template <bool NARROW>
constexpr int kThreads = NARROW ? 256 : 1024;
template <bool NARROW>
constexpr int kWidth = kThreads<NARROW>* kAt;
template <bool NARROW>
constexpr int kChunk = kWidth<NARROW>* kPacks<NARROW>;  // elements of a workgroup
static_assert(kAdamBlock == kWave * kAt, "a wavefront's pack holds the elements of a scale");

// Tensors whose addresses a launch's arguments (4 KB) have room for: POINTERS of
// AdamTensor's, in its order without those that the kernel does not use.
template <int POINTERS>
struct Batch {
    static constexpr int MOST = (4096 - int(sizeof(AdamRates)) - 16) / (POINTERS * 8 + 12);
    void* at[MOST][POINTERS];
    int64_t n[MOST];
    uint32_t first[MOST];  // workgroup that a tensor starts with; past the last one no workgroup's number
};
template <int POINTERS>
constexpr bool fits = sizeof(Batch<POINTERS>) + sizeof(AdamRates) + 8 <= 4096;
static_assert(fits<4> && fits<5> && fits<6> && fits<7>, "launch arguments");

// This workgroup's tensor, by one look at all starts (a search would take a
// chain of reads, each as long as the whole step of a small tensor).
template <bool NARROW, bool MASTER, int POINTERS>
__device__ inline AdamTensor tensor_of(const Batch<POINTERS>& b, int64_t* chunk) {
    int k = -1;
    constexpr int MOST = Batch<POINTERS>::MOST;
#pragma unroll
    for (int q = 0; q < MOST; q += kWave) {
        const int i = q + lane_id();
        k += __builtin_popcountll(__ballot(i < MOST && b.first[min(i, MOST - 1)] <= blockIdx.x));
    }
    k = int(uniform(uint32_t(k)));
    *chunk = blockIdx.x - b.first[k];
    AdamTensor t{};
    void* const* p = b.at[k];
    t.n = b.n[k];
    t.p = p[0];
    t.g = p[1];
    t.m = p[2];
    t.v = p[3];
    if constexpr (NARROW) {
        t.m_scale = static_cast<float*>(p[4]);
        t.v_scale = static_cast<float*>(p[5]);
    }
    if constexpr (MASTER) t.master = static_cast<float*>(p[POINTERS - 1]);
    return t;
}

// the elements of the pack from i on that lie in [0, n); the others are 0 (FULL:
// all of them do)
template <bool FULL, typename T>
__device__ inline void load_some(const T* p, int64_t i, int64_t n, float (&out)[kAt]) {
    if (FULL || (i >= 0 && i + kAt <= n)) {
        const Vec<T, kAt> v = load_vec_nt<T, kAt>(p + i);
#pragma unroll
        for (int k = 0; k < kAt; ++k) out[k] = float(v[k]);
    } else {
#pragma unroll
        for (int k = 0; k < kAt; ++k) out[k] = i + k >= 0 && i + k < n ? float(p[i + k]) : 0.f;
    }
}
template <bool FULL, typename T>
__device__ inline void store_some(T* p, int64_t i, int64_t n, const float (&v)[kAt]) {
    if (FULL || (i >= 0 && i + kAt <= n)) {
        Vec<T, kAt> o;
#pragma unroll
        for (int k = 0; k < kAt; ++k) o[k] = T(v[k]);
        store_vec_nt<T, kAt>(p + i, o);
    } else {
#pragma unroll
        for (int k = 0; k < kAt; ++k)
            if (i + k >= 0 && i + k < n) p[i + k] = T(v[k]);
    }
}

// The parameters after the step, from the states after it.
__device__ inline float stepped(float w, float m, float v, const AdamRates& r) {
    return fmaf(-r.lr_decay, w, w) - r.lr_m * m / (sqrtf(v * r.inv_v) + r.eps);
}

template <bool FULL, typename P, bool MASTER>
__device__ inline void load_parameters(const AdamTensor& t, int64_t i, float (&w)[kAt]) {
    if constexpr (MASTER)
        load_some<FULL>(t.master, i, t.n, w);
    else
        load_some<FULL>(static_cast<const P*>(t.p), i, t.n, w);
}
template <bool FULL, typename P, bool MASTER>
__device__ inline void store_parameters(const AdamTensor& t, int64_t i, float (&w)[kAt]) {
    if constexpr (MASTER) {
        // (the copy's value is what is rounded: kept from instructions that round the
        // last operation's unrounded result to 16 bits)
#pragma unroll
        for (int k = 0; k < kAt; ++k) asm volatile("" : "+v"(w[k]));
        store_some<FULL>(t.master, i, t.n, w);
    }
    store_some<FULL>(static_cast<P*>(t.p), i, t.n, w);
}

template <bool FULL, typename P, typename G, bool MASTER>
__device__ inline void step_wide(const AdamTensor& t, int64_t i0, const AdamRates& r) {
    float w[kPacks<false>][kAt], g[kPacks<false>][kAt], m[kPacks<false>][kAt], v[kPacks<false>][kAt];
#pragma unroll
    for (int j = 0; j < kPacks<false>; ++j) {
        const int64_t i = i0 + j * kWidth<false>;
        load_some<FULL>(static_cast<const G*>(t.g), i, t.n, g[j]);
        load_some<FULL>(static_cast<const float*>(t.m), i, t.n, m[j]);
        load_some<FULL>(static_cast<const float*>(t.v), i, t.n, v[j]);
        load_parameters<FULL, P, MASTER>(t, i, w[j]);
    }
    const float gs = r.grad_scale ? r.grad_scale[0] : 1.f;
    __builtin_amdgcn_sched_barrier(0);  // (all loads are under way before the first is used)
#pragma unroll
    for (int j = 0; j < kPacks<false>; ++j) {
        const int64_t i = i0 + j * kWidth<false>;
#pragma unroll
        for (int q = 0; q < kAt; ++q) {
            const float x = g[j][q] * gs;
            m[j][q] = fmaf(r.b1, m[j][q], r.a1 * x);
            v[j][q] = fmaf(r.b2, v[j][q], r.a2 * x * x);
            w[j][q] = stepped(w[j][q], m[j][q], v[j][q], r);
        }
        store_some<FULL>(static_cast<float*>(t.m), i, t.n, m[j]);
        store_some<FULL>(static_cast<float*>(t.v), i, t.n, v[j]);
        store_parameters<FULL, P, MASTER>(t, i, w[j]);
    }
}

template <typename P, typename G, bool MASTER>
__global__ __launch_bounds__(kThreads<false>) void adamw_wide(Batch<MASTER ? 5 : 4> b, AdamRates r) {
    int64_t chunk;
    const AdamTensor t = tensor_of<false, MASTER>(b, &chunk);
    // (packs start on 16-byte boundaries of the states, wherever the tensor does)
    const int head = int(reinterpret_cast<uintptr_t>(t.m) / sizeof(float) % kAt);
    const int64_t c0 = chunk * kChunk<false> - head, i0 = c0 + threadIdx.x * kAt;
    if (c0 >= 0 && c0 + kChunk<false> <= t.n)
        step_wide<true, P, G, MASTER>(t, i0, r);
    else
        step_wide<false, P, G, MASTER>(t, i0, r);
}

// what codes stand for, in units of S / 127^2 and S / 255^4 (the largest codes: S itself)
constexpr double kSquares = 1.0 / (127.0 * 127.0), kFourths = 1.0 / (255.0 * 255.0 * 255.0 * 255.0);
static_assert(127.0 * 127.0 * kSquares == 1.0 && 255.0 * 255.0 * 255.0 * 255.0 * kFourths == 1.0, "");
__device__ inline int squared(int c) { return c * abs(c); }
__device__ inline uint32_t fourth(int c) { return uint32_t(c * c) * uint32_t(c * c); }

// The code of y >= 0 for the scale S > 0, nearest in c, where y = (c / LEVELS)^POWER S.
// code_near: from y as a float and about 1 / S.  32 bits give LEVELS times the root
// within 2^-13 (6 units of 2^-24 relative, 255 levels); *near: it is within twice
// that of a border, and code_at has to compare it with the border, in 64 bits.
template <int LEVELS, int POWER>
__device__ inline float code_root(float f, float inv) {
    float x = __builtin_amdgcn_sqrtf(f * inv);
    if constexpr (POWER == 4) x = __builtin_amdgcn_sqrtf(x);
    return fminf(x * LEVELS, float(LEVELS));
}
template <int LEVELS, int POWER>
__device__ inline int code_near(float f, float inv, bool* near) {
    const float x = code_root<LEVELS, POWER>(f, inv), c = rintf(x);
    *near = *near || fabsf(x - c) > 0.5f - 0x1p-12f;
    return int(c);
}
template <int LEVELS, int POWER>
__device__ inline int code_at(double y, float f, float inv, float S) {
    const float x = code_root<LEVELS, POWER>(f, inv), c = rintf(x);
    if (fabsf(x - c) <= 0.5f - 0x1p-12f) return int(c);
    const double border = (floorf(x) + 0.5) * (1.0 / LEVELS), q = border * border;
    return int(floorf(x)) + (y > (POWER == 4 ? q * q : q) * double(S) ? 1 : 0);
}

template <bool FULL, typename C>
__device__ inline void load_codes(const C* p, int64_t i, int64_t n, int (&out)[kAt]) {
    if (FULL || i + kAt <= n) {
        const Vec<C, kAt> v = *reinterpret_cast<const Vec<C, kAt>*>(p + i);
#pragma unroll
        for (int k = 0; k < kAt; ++k) out[k] = v[k];
    } else {
#pragma unroll
        for (int k = 0; k < kAt; ++k) out[k] = i + k < n ? p[i + k] : 0;
    }
}
template <bool FULL, typename C>
__device__ inline void store_codes(C* p, int64_t i, int64_t n, const int (&v)[kAt]) {
    if (FULL || i + kAt <= n) {
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

__device__ inline double blend(double rate, double a, double b) {
#pragma clang fp contract(off)
    const double p = rate * a, q = (1.0 - rate) * b;
    return p + q;
}

template <bool FULL, typename P, typename G, bool MASTER>
__device__ inline void step_narrow(const AdamTensor& t, int64_t i0, const AdamRates& r) {
    const double gs = r.grad_scale ? double(r.grad_scale[0]) : 1.0;
    float w[kPacks<true>][kAt], g[kPacks<true>][kAt], ms[kPacks<true>], vs[kPacks<true>];
    int mc[kPacks<true>][kAt], vc[kPacks<true>][kAt];
#pragma unroll
    for (int j = 0; j < kPacks<true>; ++j) {
        const int64_t i = i0 + j * kWidth<true>, block = i / kAdamBlock;
        load_some<FULL>(static_cast<const G*>(t.g), i, t.n, g[j]);
        load_codes<FULL>(static_cast<const int8_t*>(t.m), i, t.n, mc[j]);
        load_codes<FULL>(static_cast<const uint8_t*>(t.v), i, t.n, vc[j]);
        load_parameters<FULL, P, MASTER>(t, i, w[j]);
        const bool there = FULL || block * kAdamBlock < t.n;  // (the same for the wavefront)
        ms[j] = there ? t.m_scale[block] : 0.f;
        vs[j] = there ? t.v_scale[block] : 0.f;
    }
#pragma unroll
    for (int j = 0; j < kPacks<true>; ++j) {
        const int64_t i = i0 + j * kWidth<true>, block = i / kAdamBlock;
        if (!FULL && block * kAdamBlock >= t.n) return;
        const double sm = double(ms[j]), sv = double(vs[j]);
        double m[kAt], v[kAt];
        float fm[kAt], fv[kAt], most_m = 0.f, most_v = 0.f;
        bool bad = false;
#pragma unroll
        for (int q = 0; q < kAt; ++q) {
            // (each product rounded: beta S + (1 - beta) g of a block's largest is a
            // tie between two scales often enough for its last bit to count)
            const double x = double(g[j][q]) * gs;
            m[q] = blend(r.d1, double(squared(mc[j][q])) * kSquares * sm, x);
            v[q] = blend(r.d2, double(fourth(vc[j][q])) * kFourths * sv, x * x);
            if (!FULL && i + q >= t.n) m[q] = v[q] = 0.0;
            fm[q] = float(m[q]);
            fv[q] = float(v[q]);
            bad = bad || !(fabsf(fm[q]) < __builtin_huge_valf()) || !(fv[q] < __builtin_huge_valf());
            most_m = fmaxf(most_m, fabsf(fm[q]));
            most_v = fmaxf(most_v, fv[q]);
            w[j][q] = fmaf(-r.lr_decay, w[j][q], w[j][q]) -
                      r.lr_m * fm[q] * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(fv[q] * r.inv_v) + r.eps);
        }
        most_m = wave_max(most_m);
        most_v = wave_max(most_v);
        if (__any(bad)) most_m = most_v = __builtin_nanf("");  // (a scale of NaN: all its values are)
        // (scales and values of the smallest are raised together, to have reciprocals)
        const float um = most_m < 0x1p-60f ? 0x1p80f : 1.f, uv = most_v < 0x1p-60f ? 0x1p80f : 1.f;
        const float im = __builtin_amdgcn_rcpf(most_m * um), iv = __builtin_amdgcn_rcpf(most_v * uv);
        if (um != 1.f || uv != 1.f)
#pragma unroll
            for (int q = 0; q < kAt; ++q) {
                fm[q] = float(m[q] * um);
                fv[q] = float(v[q] * uv);
            }
        if (most_m > 0.f && most_v > 0.f) {
            bool near = false;
#pragma unroll
            for (int q = 0; q < kAt; ++q) {
                mc[j][q] = code_near<127, 2>(fabsf(fm[q]), im, &near);
                vc[j][q] = code_near<255, 4>(fv[q], iv, &near);
            }
            if (__any(near))
#pragma unroll
                for (int q = 0; q < kAt; ++q) {
                    mc[j][q] = code_at<127, 2>(fabs(m[q]), fabsf(fm[q]), im, most_m);
                    vc[j][q] = code_at<255, 4>(v[q], fv[q], iv, most_v);
                }
        } else {
#pragma unroll
            for (int q = 0; q < kAt; ++q) {
                mc[j][q] = most_m > 0.f ? code_at<127, 2>(fabs(m[q]), fabsf(fm[q]), im, most_m) : 0;
                vc[j][q] = most_v > 0.f ? code_at<255, 4>(v[q], fv[q], iv, most_v) : 0;
            }
        }
#pragma unroll
        for (int q = 0; q < kAt; ++q) {
            if (m[q] < 0.0) mc[j][q] = -mc[j][q];
            if (most_v > 0.f && v[q] > 0.0) vc[j][q] = max(vc[j][q], 1);
        }
        store_codes<FULL>(static_cast<int8_t*>(t.m), i, t.n, mc[j]);
        store_codes<FULL>(static_cast<uint8_t*>(t.v), i, t.n, vc[j]);
        store_parameters<FULL, P, MASTER>(t, i, w[j]);
        if (lane_id() == 0) {
            t.m_scale[block] = most_m;
            t.v_scale[block] = most_v;
        }
    }
}

template <typename P, typename G, bool MASTER>
__global__ __launch_bounds__(kThreads<true>) void adamw_narrow(Batch<MASTER ? 7 : 6> b, AdamRates r) {
    int64_t chunk;
    const AdamTensor t = tensor_of<true, MASTER>(b, &chunk);
    const int64_t c0 = chunk * kChunk<true>, i0 = c0 + threadIdx.x * kAt;
    if (c0 + kChunk<true> <= t.n)
        step_narrow<true, P, G, MASTER>(t, i0, r);
    else
        step_narrow<false, P, G, MASTER>(t, i0, r);
}

// the values that 8-bit states stand for, into 32-bit floats (t.p for m, t.master for v)
template <bool FULL>
__device__ inline void values_of(const AdamTensor& t, int64_t i0) {
    int mc[kPacks<true>][kAt], vc[kPacks<true>][kAt];
    float ms[kPacks<true>], vs[kPacks<true>];
#pragma unroll
    for (int j = 0; j < kPacks<true>; ++j) {
        const int64_t i = i0 + j * kWidth<true>, block = i / kAdamBlock;
        load_codes<FULL>(static_cast<const int8_t*>(t.m), i, t.n, mc[j]);
        load_codes<FULL>(static_cast<const uint8_t*>(t.v), i, t.n, vc[j]);
        const bool there = FULL || block * kAdamBlock < t.n;
        ms[j] = there ? t.m_scale[block] : 0.f;
        vs[j] = there ? t.v_scale[block] : 0.f;
    }
#pragma unroll
    for (int j = 0; j < kPacks<true>; ++j) {
        const int64_t i = i0 + j * kWidth<true>;
        const double km = kSquares * double(ms[j]), kv = kFourths * double(vs[j]);
        float m[kAt], v[kAt];
#pragma unroll
        for (int q = 0; q < kAt; ++q) {
            m[q] = float(squared(mc[j][q]) * km);
            v[q] = float(fourth(vc[j][q]) * kv);
        }
        store_some<FULL>(static_cast<float*>(t.p), i, t.n, m);
        store_some<FULL>(t.master, i, t.n, v);
    }
}

__global__ __launch_bounds__(kThreads<true>) void adam_values_kernel(Batch<7> b) {
    int64_t chunk;
    const AdamTensor t = tensor_of<true, true>(b, &chunk);
    const int64_t c0 = chunk * kChunk<true>, i0 = c0 + threadIdx.x * kAt;
    if (c0 + kChunk<true> <= t.n)
        values_of<true>(t, i0);
    else
        values_of<false>(t, i0);
}

// f(batch, workgroups) over the tensors, as many at a time as the arguments hold
template <bool NARROW, bool MASTER, typename F>
void by_batch(const AdamTensor* t, int64_t count, F f) {
    constexpr int POINTERS = 4 + (NARROW ? 2 : 0) + (MASTER ? 1 : 0);
    Batch<POINTERS> b;
    int have = 0;
    int64_t blocks = 0;
    auto flush = [&] {
        for (int q = have; q < b.MOST; ++q) b.first[q] = 0xffffffffu;
        if (have) f(b, unsigned(blocks));
        have = 0;
        blocks = 0;
    };
    for (int64_t q = 0; q < count; ++q) {
        if (t[q].n <= 0) continue;
        const int64_t more = (t[q].n + kAt - 1 + kChunk<NARROW> - 1) / kChunk<NARROW>;  // (with what comes before the first pack)
        // (a launch has at most 2^22 workgroups and so 2^32 threads, or those of one tensor)
        if (have == b.MOST || (have && blocks + more > (int64_t(1) << 22) - 1)) flush();
        void** p = b.at[have];
        p[0] = t[q].p;
        p[1] = const_cast<void*>(t[q].g);
        p[2] = t[q].m;
        p[3] = t[q].v;
        if (NARROW) {
            p[4] = t[q].m_scale;
            p[5] = t[q].v_scale;
        }
        if (MASTER) p[POINTERS - 1] = t[q].master;
        b.n[have] = t[q].n;
        b.first[have++] = uint32_t(blocks);
        blocks += more;
    }
    flush();
}

}  // namespace

void adamw(const AdamTensor* t, int64_t count, int param_dtype, int grad_dtype, int bits, bool master,
           const AdamRates& r, hipStream_t s) {
    by_dtype(param_dtype, [&](auto e) {
        using P = decltype(e);
        auto launch = [&](auto gt, auto wide) {
            using G = decltype(gt);
            constexpr bool MASTER = decltype(wide)::value;
            if (bits == 32)
                by_batch<false, MASTER>(t, count, [&](const auto& b, unsigned blocks) {
                    adamw_wide<P, G, MASTER><<<blocks, kThreads<false>, 0, s>>>(b, r);
                });
            else
                by_batch<true, MASTER>(t, count, [&](const auto& b, unsigned blocks) {
                    adamw_narrow<P, G, MASTER><<<blocks, kThreads<true>, 0, s>>>(b, r);
                });
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
}

void adam_values(const AdamTensor* t, int64_t count, hipStream_t s) {
    by_batch<true, true>(t, count,
                         [&](const auto& b, unsigned blocks) { adam_values_kernel<<<blocks, kThreads<true>, 0, s>>>(b); });
}

}  // namespace spsyrk
