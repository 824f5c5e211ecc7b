// Lookup of dense rows by sparse rows, Y = scale A W, and the gradient of the
// table, dW = scale A^T G.
//
// Tokens (one column per row) are a copy of table rows: bound by the bytes of
// the rows read and written.  CSR rows and the gradient are the same sum,
//     out[t] = scale * sum over the entries e of target t of w_e src[from_e],
// with the entries grouped by target: the rows of A for the lookup, the
// columns of A for the gradient, whose entries are sorted by column first
// (stable, so a column's entries are added in their order in A and the result
// is the same on every run).  Sums are held in 32-bit floats and rounded once.
//
// A wavefront takes a target's columns 16 bytes a lane, kUnroll packs of a
// row at once; targets of narrow rows share a wavefront.  A target of more
// than a tile of entries (a frequent token) would be walked by one wavefront:
// such targets are left to a second launch, in which every tile of entries
// sums its part of the (at most two) long targets that reach into it, and a
// third adds a target's parts in tile order.
#include <algorithm>

#include "internal.h"
#include "rows.h"

namespace spsyrk {
namespace {

constexpr int kUnroll = 4;  // packs of one row per lane

// Lanes per row (a power of two, at most a wavefront) for rows of `packs` packs.
inline int lane_bits(int64_t packs) {
    int lg = 0;
    while (lg < 6 && (int64_t(1) << lg) < packs) ++lg;
    return lg;
}

inline unsigned grid_for(int64_t waves) {
    const int64_t blocks = (waves + kWavesPerBlock - 1) / kWavesPerBlock;
    return unsigned(std::min<int64_t>(std::max<int64_t>(blocks, 1), int64_t(1) << 20));
}

__device__ inline int64_t first_wave() { return int64_t(blockIdx.x) * kWavesPerBlock + threadIdx.x / kWave; }
__device__ inline int64_t all_waves() { return int64_t(gridDim.x) * kWavesPerBlock; }

// ---- tokens

template <typename T, int U>
__global__ __launch_bounds__(kBlock) void tokens_kernel(Entries A, const T* __restrict__ W, int64_t ldw, int64_t d,
                                                        float scale, T* __restrict__ Y, int64_t ldy, int lg,
                                                        int64_t chunks, int64_t units) {
    constexpr int N = Pack<T>::N;
    const int lane = lane_id(), sub = lane >> lg, l = lane & ((1 << lg) - 1);
    const int rows = kWave >> lg;
    for (int64_t u = first_wave(); u < units; u += all_waves()) {
        const int64_t row = u / chunks * rows + sub;
        if (row >= A.m) continue;
        const int64_t c0 = (u % chunks * (int64_t(U) << lg) + l) * N;
        const int64_t col = load_column(A.idx, A.ib, row * A.istride);
        const bool named = col >= 0 && col < A.n;
        const T* src = W + (named ? col * ldw : 0);
        PackV<T> v[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t c = c0 + (int64_t(k) << lg) * N;
            v[k] = load_pack(src + c, named ? d - c : 0);
        }
        T* dst = Y + row * ldy;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t c = c0 + (int64_t(k) << lg) * N;
            PackV<T> o;
#pragma unroll
            for (int i = 0; i < N; ++i) o[i] = T(float(v[k][i]) * scale);
            store_pack_nt(dst + c, o, d - c);
        }
    }
}

// ---- sums over entries grouped by target

// start of target t: P is int64 (row pointers of A, kept inside [0, nnz] here
// whatever they hold) or uint32 (starts found by this file's kernels)
template <typename P>
struct Targets {
    const P* start;  // targets + 1
    int64_t targets;
    int64_t nnz;
    const void* from;  // source row of every entry
    int ib;
    const void* w;  // weight of every entry (null: 1)
    int wt;
    __device__ inline int64_t at(int64_t t) const {
        const int64_t s = int64_t(start[t]);
        return s < 0 ? 0 : (s > nnz ? nnz : s);
    }
};

// acc += sum of the entries [a, b) over the lane's packs at c0, c0 + (N << lg), ...
// Every group of 1 << lg lanes reads its entries' rows and weights one per
// lane and takes them from there by lane reads.
template <typename T, int U, typename P>
__device__ inline void sum_entries(const Targets<P>& t, int64_t a, int64_t b, const T* __restrict__ src,
                                   int64_t nsrc, int64_t ld, int64_t d, int64_t c0, int lg,
                                   float (&acc)[U][Pack<T>::N]) {
    constexpr int N = Pack<T>::N;
    const int width = 1 << lg, l = lane_id() & (width - 1);
    for (int64_t base = a; base < b; base += width) {
        int64_t row = -1;
        float w = 0.f;
        if (base + l < b) {
            row = load_column(t.from, t.ib, base + l);
            w = t.w ? load_value(t.w, t.wt, base + l) : 1.f;
            if (row < 0 || row >= nsrc) row = -1;
        }
        const int n = int(min(int64_t(width), b - base));
        for (int j = 0; j < n; ++j) {
            const int64_t r = __shfl(row, j, width);
            const float wj = __shfl(w, j, width);
            if (r < 0) continue;
            const T* p = src + r * ld;
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int64_t c = c0 + (int64_t(k) << lg) * N;
                const PackV<T> v = load_pack(p + c, d - c);
#pragma unroll
                for (int i = 0; i < N; ++i) acc[k][i] = fmaf(wj, float(v[i]), acc[k][i]);
            }
        }
    }
}

template <typename T, int U, typename P>
__global__ __launch_bounds__(kBlock) void sum_targets(Targets<P> t, const T* __restrict__ src, int64_t nsrc,
                                                      int64_t lds, int64_t d, float scale, T* __restrict__ out,
                                                      int64_t ldo, int lg, int64_t chunks, int64_t units,
                                                      int64_t tile) {
    constexpr int N = Pack<T>::N;
    const int lane = lane_id(), sub = lane >> lg, l = lane & ((1 << lg) - 1);
    const int rows = kWave >> lg;
    for (int64_t u = first_wave(); u < units; u += all_waves()) {
        const int64_t target = u / chunks * rows + sub;
        if (target >= t.targets) continue;
        const int64_t a = t.at(target), b = t.at(target + 1);
        if (b - a > tile) continue;
        const int64_t c0 = (u % chunks * (int64_t(U) << lg) + l) * N;
        float acc[U][N] = {};
        sum_entries<T, U>(t, a, b, src, nsrc, lds, d, c0, lg, acc);
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t c = c0 + (int64_t(k) << lg) * N;
            PackV<T> o;
#pragma unroll
            for (int i = 0; i < N; ++i) o[i] = T(acc[k][i] * scale);
            store_pack_nt(out + target * ldo + c, o, d - c);
        }
    }
}

// the target that holds entry e: the largest t in [0, targets) with start[t] <= e
template <typename P>
__device__ inline int64_t target_of(const Targets<P>& t, int64_t e) {
    int64_t lo = 0, hi = t.targets - 1;
    while (lo < hi) {
        const int64_t mid = (lo + hi + 1) >> 1;
        if (t.at(mid) <= e)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

// Tile q's part of the long targets that hold its first and its last entry,
// into part[2 q] and part[2 q + 1] (the latter only for a target that starts
// inside the tile).
template <typename T, int U, typename P>
__global__ __launch_bounds__(kBlock) void sum_tiles(Targets<P> t, const T* __restrict__ src, int64_t nsrc,
                                                    int64_t lds, int64_t d, float* __restrict__ part, int64_t tile,
                                                    int lg, int64_t chunks, int64_t units, int64_t ntiles) {
    constexpr int N = Pack<T>::N;
    const int lane = lane_id(), sub = lane >> lg, l = lane & ((1 << lg) - 1);
    const int rows = kWave >> lg;
    const int64_t end = t.at(t.targets);
    for (int64_t u = first_wave(); u < units; u += all_waves()) {
        const int64_t q = u / chunks * rows + sub;
        const int64_t e0 = q * tile, e1 = min(end, e0 + tile);
        if (q >= ntiles || e0 >= e1) continue;
        const int64_t c0 = (u % chunks * (int64_t(U) << lg) + l) * N;
        const int64_t first = target_of(t, e0), last = target_of(t, e1 - 1);
        for (int k2 = 0; k2 < 2; ++k2) {
            const int64_t target = k2 ? last : first;
            if (k2 && last == first) break;
            const int64_t a = t.at(target), b = t.at(target + 1);
            if (b - a <= tile) continue;
            float acc[U][N] = {};
            sum_entries<T, U>(t, max(a, e0), min(b, e1), src, nsrc, lds, d, c0, lg, acc);
            float* dst = part + (2 * q + k2) * d;
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int64_t c = c0 + (int64_t(k) << lg) * N;
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (c + i < d) dst[c + i] = acc[k][i];
            }
        }
    }
}

// The long target that starts in tile q, if any (it holds the tile's last
// entry): its parts in tile order, 64 columns per workgroup.
template <typename T, typename P>
__global__ __launch_bounds__(kBlock) void join_tiles(Targets<P> t, const float* __restrict__ part, int64_t d,
                                                     float scale, T* __restrict__ out, int64_t ldo, int64_t tile,
                                                     int64_t ntiles) {
    __shared__ float sum[kWavesPerBlock][kWave];
    const int64_t q = blockIdx.x;
    const int64_t end = t.at(t.targets);
    const int64_t e0 = q * tile, e1 = min(end, e0 + tile);
    if (e0 >= e1) return;
    const int64_t target = target_of(t, e1 - 1);
    const int64_t a = t.at(target), b = t.at(target + 1);
    if (b - a <= tile || a < e0 || a >= e1) return;
    const int64_t tiles = min((b - 1) / tile, ntiles - 1) - q + 1;
    // the target's part of its first tile is the second one if another target
    // holds that tile's first entry
    const int64_t skip = target_of(t, e0) == target ? 0 : 1;
    const int w = threadIdx.x / kWave, lane = lane_id();
    const int64_t per = (tiles + kWavesPerBlock - 1) / kWavesPerBlock;
    for (int64_t c = int64_t(blockIdx.y) * kWave + lane; c - lane < d; c += int64_t(gridDim.y) * kWave) {
        float s = 0.f;
        if (c < d)
            for (int64_t x = w * per; x < min(tiles, (w + 1) * per); ++x)
                s += part[(2 * (q + x) + (x == 0 ? skip : 0)) * d + c];
        sum[w][lane] = s;
        __syncthreads();
        if (w == 0 && c < d) {
            float r = 0.f;
            for (int i = 0; i < kWavesPerBlock; ++i) r += sum[i][lane];
            out[target * ldo + c] = T(r * scale);
        }
        __syncthreads();
    }
}

// Entries per tile: 64, doubled for every fourfold of 2^16 entries, so that
// neither a tile nor the parts of one target grow past the square root of
// the entries by much.
inline int64_t sum_tile(int64_t nnz) {
    int64_t t = 64;
    while (t * t * 16 < nnz) t *= 2;
    return t;
}

inline size_t round256(size_t b) { return (b + 255) & ~size_t(255); }

inline size_t part_bytes(int64_t nnz, int64_t d) {
    const int64_t tile = sum_tile(nnz);
    return nnz > tile ? size_t((nnz + tile - 1) / tile) * 2 * size_t(d) * sizeof(float) : 0;
}

template <typename T, int U, typename P>
void launch_sums(const Targets<P>& t, const DenseRows& src, float scale, const DenseRows& out, float* part,
                 int64_t packs, int lg, hipStream_t s) {
    const int64_t chunks = (packs + (int64_t(U) << lg) - 1) / (int64_t(U) << lg);
    const int64_t rows = kWave >> lg, d = out.n;
    const int64_t tile = sum_tile(t.nnz);
    const int64_t units = (t.targets + rows - 1) / rows * chunks;
    const T* sp = static_cast<const T*>(src.p);
    T* op = static_cast<T*>(out.p);
    sum_targets<T, U, P><<<grid_for(units), kBlock, 0, s>>>(t, sp, src.m, src.ld, d, scale, op, out.ld, lg, chunks,
                                                            units, tile);
    if (t.nnz <= tile) return;  // (no target is long)
    const int64_t ntiles = (t.nnz + tile - 1) / tile;
    const int64_t tunits = (ntiles + rows - 1) / rows * chunks;
    sum_tiles<T, U, P><<<grid_for(tunits), kBlock, 0, s>>>(t, sp, src.m, src.ld, d, part, tile, lg, chunks, tunits,
                                                           ntiles);
    join_tiles<T, P><<<dim3(unsigned(ntiles), unsigned(std::min<int64_t>((d + kWave - 1) / kWave, 64))), kBlock, 0,
                       s>>>(t, part, d, scale, op, out.ld, tile, ntiles);
}

template <typename P>
void grouped_sums(const Targets<P>& t, const DenseRows& src, float scale, const DenseRows& out, float* part,
                  hipStream_t s) {
    by_dtype(out.dt, [&](auto e) {
        using T = decltype(e);
        const int64_t packs = (out.n + Pack<T>::N - 1) / Pack<T>::N;
        const int lg = lane_bits(packs);
        if (packs <= kWave)
            launch_sums<T, 1, P>(t, src, scale, out, part, packs, lg, s);
        else
            launch_sums<T, kUnroll, P>(t, src, scale, out, part, packs, lg, s);
    });
}

// ---- the gradient's entries sorted by column

// the row that holds entry e (row pointers kept inside [0, nnz])
__device__ inline int64_t row_of(const int64_t* rp, int64_t m, int64_t e) {
    int64_t lo = 0, hi = m - 1;
    while (lo < hi) {
        const int64_t mid = (lo + hi + 1) >> 1;
        if (rp[mid] <= e)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

// Sort records: the column (n for padding, which sorts past every column),
// the row and the weight of every entry.
__global__ __launch_bounds__(kBlock) void sort_records(Entries A, uint32_t* __restrict__ key,
                                                       uint32_t* __restrict__ row, float* __restrict__ w) {
    const int64_t stride = int64_t(gridDim.x) * kBlock;
    for (int64_t e = int64_t(blockIdx.x) * kBlock + threadIdx.x; e < A.nnz; e += stride) {
        const int64_t r = A.rp ? row_of(A.rp, A.m, e) : e;
        const int64_t c = load_column(A.idx, A.ib, A.rp ? e : e * A.istride);
        key[e] = uint32_t(c >= 0 && c < A.n ? c : A.n);
        row[e] = uint32_t(r);
        if (w) w[e] = load_value(A.val, A.vt, e);
    }
}

// start[c] = sorted entries of columns before c, c = 0 .. n
__global__ __launch_bounds__(kBlock) void column_bounds(const uint32_t* __restrict__ key, int64_t nnz, int64_t n,
                                                        uint32_t* __restrict__ start) {
    const int64_t stride = int64_t(gridDim.x) * kBlock;
    for (int64_t c = int64_t(blockIdx.x) * kBlock + threadIdx.x; c <= n; c += stride)
        start[c] = uint32_t(lower_bound_u32(key, 0, nnz, uint64_t(c)));
}

inline unsigned thread_grid(int64_t n) {
    return unsigned(std::min<int64_t>((n + kBlock - 1) / kBlock, int64_t(1) << 16));
}

}  // namespace

void embed_tokens(const Entries& A, const DenseRows& W, float scale, const DenseRows& Y, hipStream_t s) {
    by_dtype(Y.dt, [&](auto e) {
        using T = decltype(e);
        const int64_t packs = (Y.n + Pack<T>::N - 1) / Pack<T>::N;
        const int lg = lane_bits(packs);
        const int64_t per = packs <= kWave ? 1 : kUnroll;
        const int64_t chunks = (packs + (per << lg) - 1) / (per << lg);
        const int64_t rows = kWave >> lg;
        const int64_t units = (A.m + rows - 1) / rows * chunks;
        const T* w = static_cast<const T*>(W.p);
        T* y = static_cast<T*>(Y.p);
        if (per == 1)
            tokens_kernel<T, 1><<<grid_for(units), kBlock, 0, s>>>(A, w, W.ld, Y.n, scale, y, Y.ld, lg, chunks, units);
        else
            tokens_kernel<T, kUnroll><<<grid_for(units), kBlock, 0, s>>>(A, w, W.ld, Y.n, scale, y, Y.ld, lg, chunks,
                                                                         units);
    });
}

size_t embed_csr_tmp_bytes(int64_t nnz, int64_t d) { return part_bytes(nnz, d); }

void embed_csr(const Entries& A, const DenseRows& W, float scale, const DenseRows& Y, void* tmp, hipStream_t s) {
    Targets<int64_t> t{A.rp, A.m, A.nnz, A.idx, A.ib, A.val, A.vt};
    grouped_sums(t, W, scale, Y, static_cast<float*>(tmp), s);
}

size_t embed_grad_tmp_bytes(const Entries& A, int64_t d) {
    const size_t words = round256(size_t(A.nnz) * sizeof(uint32_t));
    return words * (A.val ? 6 : 4) + round256(size_t(A.n + 1) * sizeof(uint32_t)) +
           round256(radix_tmp_bytes(A.nnz)) + part_bytes(A.nnz, d);
}

void embed_grad(const Entries& A, const DenseRows& G, float scale, const DenseRows& dW, void* tmp, hipStream_t s) {
    char* at = static_cast<char*>(tmp);
    auto take = [&](size_t bytes) {
        char* p = at;
        at += round256(bytes);
        return p;
    };
    const size_t words = size_t(A.nnz) * sizeof(uint32_t);
    uint32_t* start = reinterpret_cast<uint32_t*>(take(size_t(A.n + 1) * sizeof(uint32_t)));
    uint32_t *key[2], *row[2];
    float* w[2] = {nullptr, nullptr};
    for (int i = 0; i < 2; ++i) {
        key[i] = reinterpret_cast<uint32_t*>(take(words));
        row[i] = reinterpret_cast<uint32_t*>(take(words));
        if (A.val) w[i] = reinterpret_cast<float*>(take(words));
    }
    void* sort_tmp = take(radix_tmp_bytes(A.nnz));
    int which = 0;
    if (A.nnz > 0) {
        sort_records<<<thread_grid(A.nnz), kBlock, 0, s>>>(A, key[0], row[0], w[0]);
        which = radix_sort(key[0], key[1], row[0], row[1], w[0], w[1], A.val ? 4 : 0, A.nnz,
                           bit_width_u64(uint64_t(A.n)), sort_tmp, s);
    }
    column_bounds<<<thread_grid(A.n + 1), kBlock, 0, s>>>(key[which], A.nnz, A.n, start);
    Targets<uint32_t> t{start, A.n, A.nnz, row[which], 4, w[which], kDtF32};
    grouped_sums(t, G, scale, dW, reinterpret_cast<float*>(at), s);
}

}  // namespace spsyrk
