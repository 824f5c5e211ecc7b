// Dense rows of 16- and 32-bit floats next to sparse rows: element types,
// 16-byte packs, and the arguments of the lookup, layer norm and distillation
// kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "common.h"

namespace spsyrk {

// element types (same values as spsyrk_dtype)
enum Dtype : int { kDtF32 = 0, kDtF16 = 1, kDtBF16 = 2 };
inline int dtype_bytes(int dt) { return dt == kDtF32 ? 4 : 2; }

// f(element) for an element of the type (the dispatch of every launch below)
template <typename F>
inline void by_dtype(int dt, F f) {
    if (dt == kDtF32)
        f(float());
    else if (dt == kDtF16)
        f(_Float16());
    else
        f(__bf16());
}

// N elements: a pack of 16 bytes, or one element for rows shorter than a pack.
// The vector type is aligned as one element: gfx950 loads and stores 16 bytes at
// any element's address with one instruction, so rows of odd lengths and strides
// go through the same code as aligned ones.
template <typename T, int N>
struct VecOf {
    typedef T V __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};
template <typename T, int N>
using Vec = typename VecOf<T, N>::V;

// Where the N elements from column c on (c > -N) are taken in a row of d >= N
// columns: a pack that would pass one of the row's ends is moved back into it.
// Only those elements i with mine(shift, i) are then the pack's own, the others
// belong to the next or the last pack too (none is if c >= d: shift >= N).
// Maps may write them twice, with one value; sums leave them out.
struct Place {
    int c, shift;
};
template <int N>
__device__ inline Place place(int64_t c, int64_t d) {
    const int64_t at = max(min(c, d - N), int64_t(0));
    return {int(at), int(min(c - at, int64_t(N)))};
}
template <int N>
__device__ inline bool mine(int shift, int i) {
    return uint32_t(i - shift) < uint32_t(N);
}
// Elements between the last 16-byte boundary and p.  Packs that start so many
// columns before a row lie on boundaries: 16 bytes off them, and worst off
// those of 4 bytes, cost up to half of a stream's rate.
template <typename T, int N>
__device__ inline int misaligned(const T* p) {
    return N == 1 ? 0 : int(reinterpret_cast<uintptr_t>(p) % 16 / sizeof(T));
}
inline bool on_boundaries(const void* p, int64_t ld, int dt) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * dtype_bytes(dt) % 16 == 0;
}
template <typename T, int N>
__device__ inline Vec<T, N> load_vec(const T* p) {
    return *reinterpret_cast<const Vec<T, N>*>(p);
}
template <typename T, int N>
__device__ inline Vec<T, N> load_vec_nt(const T* p) {
    return __builtin_nontemporal_load(reinterpret_cast<const Vec<T, N>*>(p));
}
template <typename T, int N>
__device__ inline void store_vec(T* p, Vec<T, N> v) {
    *reinterpret_cast<Vec<T, N>*>(p) = v;
}
template <typename T, int N>
__device__ inline void store_vec_nt(T* p, Vec<T, N> v) {
    __builtin_nontemporal_store(v, reinterpret_cast<Vec<T, N>*>(p));
}

// Sum over the wavefront, in every lane: four steps within rows of 16 lanes
// and two across them, each one instruction (a shuffle through LDS takes far
// longer, and sums like these stand between a row's loads and its stores).
__device__ inline float wave_total(float v) {
    auto add = [&](auto ctrl, auto rows) {
        const int o = __builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, decltype(rows)::value,
                                                  0xf, false);
        v += __int_as_float(o);
    };
    using std::integral_constant;
    add(integral_constant<int, 0x111>(), integral_constant<int, 0xf>());  // from 1 lane below
    add(integral_constant<int, 0x112>(), integral_constant<int, 0xf>());  // 2
    add(integral_constant<int, 0x114>(), integral_constant<int, 0xf>());  // 4
    add(integral_constant<int, 0x118>(), integral_constant<int, 0xf>());  // 8: lane 15 of a row has its sum
    add(integral_constant<int, 0x142>(), integral_constant<int, 0xa>());  // to rows 1 and 3 from the row before
    add(integral_constant<int, 0x143>(), integral_constant<int, 0xc>());  // to rows 2 and 3 from row 1
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), kWave - 1));
}

// Maximum over the wavefront, in every lane (NaN is passed over).
__device__ inline float wave_max(float v) {
    auto step = [&](auto ctrl, auto rows) {
        const int o = __builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), decltype(ctrl)::value,
                                                  decltype(rows)::value, 0xf, false);
        v = fmaxf(v, __int_as_float(o));
    };
    using std::integral_constant;
    step(integral_constant<int, 0x111>(), integral_constant<int, 0xf>());
    step(integral_constant<int, 0x112>(), integral_constant<int, 0xf>());
    step(integral_constant<int, 0x114>(), integral_constant<int, 0xf>());
    step(integral_constant<int, 0x118>(), integral_constant<int, 0xf>());
    step(integral_constant<int, 0x142>(), integral_constant<int, 0xa>());
    step(integral_constant<int, 0x143>(), integral_constant<int, 0xc>());
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), kWave - 1));
}

// A workgroup's barrier for what it exchanges through LDS: unlike
// __syncthreads it orders no access to memory, so loads in flight stay so.
__device__ inline void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// f(element, width): the pack width for rows of d columns
template <typename F>
inline void by_width(int dt, int64_t d, F f) {
    by_dtype(dt, [&](auto e) {
        using T = decltype(e);
        constexpr int N = 16 / int(sizeof(T));
        if (d >= N)
            f(e, std::integral_constant<int, N>());
        else
            f(e, std::integral_constant<int, 1>());
    });
}

// one value of a run-time type
__device__ inline float load_value(const void* p, int dt, int64_t i) {
    if (dt == kDtF32) return static_cast<const float*>(p)[i];
    if (dt == kDtF16) return float(static_cast<const _Float16*>(p)[i]);
    return float(static_cast<const __bf16*>(p)[i]);
}

// Sparse rows: CSR (rp), or rectangular rows of per_row entries, row r's
// columns from idx[r * istride] and values from val[r * vstride].  Columns of
// 4 or 8 bytes (ib); those outside [0, n) are padding.
struct Entries {
    int64_t m = 0, n = 0, nnz = 0;
    const int64_t* rp = nullptr;
    int64_t per_row = 0, istride = 0, vstride = 0;
    const void* idx = nullptr;
    int ib = 4;
    const void* val = nullptr;  // null: every value is 1
    int vt = kDtF32;
};

__device__ inline int64_t load_column(const void* idx, int ib, int64_t i) {
    return ib == 4 ? int64_t(static_cast<const int32_t*>(idx)[i]) : static_cast<const int64_t*>(idx)[i];
}

struct DenseRows {
    int64_t m = 0, n = 0, ld = 0;
    int dt = kDtF32;
    void* p = nullptr;
};

// ---- embed.hip
// Y = scale A W: one column per row (tokens), or CSR rows.
void embed_tokens(const Entries& A, const DenseRows& W, float scale, const DenseRows& Y, hipStream_t s);
size_t embed_csr_tmp_bytes(int64_t nnz, int64_t d);
void embed_csr(const Entries& A, const DenseRows& W, float scale, const DenseRows& Y, void* tmp, hipStream_t s);
// dW = scale A^T G, dW of A.n rows.  tmp: embed_grad_tmp_bytes(A, d)
size_t embed_grad_tmp_bytes(const Entries& A, int64_t d);
void embed_grad(const Entries& A, const DenseRows& G, float scale, const DenseRows& dW, void* tmp, hipStream_t s);

// ---- norm.hip
// Parameters and their gradients are of type pt; null: none.
void layer_norm(const DenseRows& X, const void* gamma, const void* beta, int pt, float eps, const DenseRows& Y,
                float* mean, float* rstd, hipStream_t s);
size_t layer_norm_grad_tmp_bytes(int64_t m, int64_t d, int dt, bool params);
void layer_norm_grad(const DenseRows& G, const DenseRows& X, const float* mean, const float* rstd, const void* gamma,
                     int pt, const DenseRows& dX, void* dgamma, void* dbeta, void* tmp, hipStream_t s);

// ---- distill.hip
// loss of every row; with dS.p its gradient too, times weight (null: 1)
size_t distill_tmp_bytes(const DenseRows& S, bool grad);
void distill(const DenseRows& S, const Entries& teacher, float temperature, const float* weight, float* loss,
             const DenseRows& dS, void* tmp, hipStream_t s);

}  // namespace spsyrk
