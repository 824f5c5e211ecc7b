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
// A wavefront takes a target's columns 16 bytes a lane, several entries' rows
// at once (two packs a lane of four entries: 355 us against 325 with one pack
// of eight, 65536 tokens over 131072 x 4096 bf16); targets of narrow rows share
// a wavefront.  A target of more than a tile of entries (a frequent token)
// would be walked by one wavefront: the first workgroups of the same launch
// take tiles of entries instead, each of which sums its part of the (at most
// two) long targets that reach into it, and a second launch adds a target's
// parts in tile order.
#include <algorithm>

#include "internal.h"
#include "rows.h"

namespace spsyrk {
namespace {

constexpr int kUnroll = 4;  // packs of one row per lane (tokens)

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

template <typename T, int N, int U>
__global__ __launch_bounds__(kBlock) void tokens_kernel(Entries A, const T* __restrict__ W, int64_t ldw, int64_t d,
                                                        float scale, T* __restrict__ Y, int64_t ldy, int lg,
                                                        int64_t chunks, int64_t units) {
    const int lane = lane_id(), sub = lane >> lg, l = lane & ((1 << lg) - 1);
    const int rows = kWave >> lg;
    for (int64_t u = first_wave(); u < units; u += all_waves()) {
        const int64_t row = u / chunks * rows + sub;
        if (row >= A.m) continue;
        const int64_t c0 = (u % chunks * (int64_t(U) << lg) + l) * N;
        const int64_t col = load_column(A.idx, A.ib, row * A.istride);
        const bool named = col >= 0 && col < A.n;
        const T* src = W + col * ldw;
        Vec<T, N> v[U];
        Place at[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            at[k] = place<N>(c0 + (int64_t(k) << lg) * N, d);
            v[k] = Vec<T, N>(T(0.f));
            if (named) v[k] = load_vec<T, N>(src + at[k].c);
        }
        T* dst = Y + row * ldy;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (at[k].shift >= N) break;
            Vec<T, N> o;
#pragma unroll
            for (int i = 0; i < N; ++i) o[i] = T(float(v[k][i]) * scale);
            store_vec_nt<T, N>(dst + at[k].c, o);
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
    const uint32_t* owner;  // target of every tile's first and last entry, by entry (null: found by search)
    int step;               // words from an entry's row, and weight, to the next one's
    __device__ inline int64_t at(int64_t t) const {
        const int64_t s = int64_t(start[t]);
        return s < 0 ? 0 : (s > nnz ? nnz : s);
    }
};

constexpr int kSumEntries = 8;

// acc += sum of the entries [a, b) over the lane's pack.
// Every group of 1 << lg lanes reads its entries' rows and weights one per
// lane and takes them from there by lane reads; E entries' packs are in
// flight at once.
template <typename T, int N, int E, typename P>
__device__ inline void sum_entries(const Targets<P>& t, int64_t a, int64_t b, const T* __restrict__ src,
                                   int64_t nsrc, int64_t ld, const Place& at, int lg, float (&acc)[N]) {
    const int width = 1 << lg, l = lane_id() & (width - 1);
    for (int64_t base = a; base < b; base += width) {
        int64_t row = -1;
        float w = 0.f;
        if (base + l < b) {
            row = load_column(t.from, t.ib, (base + l) * t.step);
            w = t.w ? load_value(t.w, t.wt, (base + l) * t.step) : 1.f;
            if (row < 0 || row >= nsrc) row = -1;
        }
        const int n = int(min(int64_t(width), b - base));
        for (int j = 0; j < n; j += E) {
            Vec<T, N> v[E];
            float wj[E];
#pragma unroll
            for (int x = 0; x < E; ++x) {
                const int y = min(j + x, width - 1);
                int64_t r = __shfl(row, y, width);
                wj[x] = __shfl(w, y, width);
                if (j + x >= n) r = -1;
                // (nothing is read for padding, which adds zeros whatever its weight)
                if (r < 0) wj[x] = 0.f;
                v[x] = Vec<T, N>(T(0.f));
                if (r >= 0) v[x] = load_vec<T, N>(src + r * ld + at.c);
            }
#pragma unroll
            for (int x = 0; x < E; ++x)
#pragma unroll
                for (int i = 0; i < N; ++i) acc[i] = fmaf(wj[x], float(v[x][i]), acc[i]);
        }
    }
}

// What one launch of the sums works on.
template <typename T, typename P>
struct Sums {
    Targets<P> t;
    const T* src;
    int64_t nsrc, lds, d;
    float scale;
    T* out;
    int64_t ldo;
    int lg;
    int64_t chunks;            // wavefronts per target
    int64_t tile, ntiles;
    float* part;               // two rows of dp sums per tile
    int64_t dp;
    int32_t* long_of;          // the targets that those belong to (-1: none)
    unsigned tile_blocks;      // workgroups of the tiles, before those of the targets
    int64_t tile_units, target_units;
    int per;                   // targets that a group of lanes takes, one after another
};

// the target that holds entry e: the largest t in [0, targets) with start[t] <= e
template <typename P>
__device__ inline int64_t target_of(const Targets<P>& t, int64_t e) {
    if (t.owner) return t.owner[e];
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
template <typename T, int N, typename P>
__device__ inline void sum_tile(const Sums<T, P>& a, int64_t q, int64_t chunk, int l, int64_t end) {
    const int64_t e0 = q * a.tile, e1 = min(end, e0 + a.tile);
    int64_t of[2] = {-1, -1};
    if (e0 < e1) {
        of[0] = target_of(a.t, e0);
        of[1] = target_of(a.t, e1 - 1);
        if (of[1] == of[0]) of[1] = -1;
    }
    const Place at = place<N>(((chunk << a.lg) + l) * N, a.d);
#pragma unroll
    for (int z = 0; z < 2; ++z) {
        int64_t x0 = 0, x1 = 0;
        if (of[z] >= 0) {
            x0 = a.t.at(of[z]);
            x1 = a.t.at(of[z] + 1);
            if (x1 - x0 <= a.tile) of[z] = -1;
        }
        if (chunk == 0 && l == 0) a.long_of[2 * q + z] = int32_t(of[z]);
        if (of[z] < 0) continue;
        float acc[N] = {};
        sum_entries<T, N, kSumEntries>(a.t, max(x0, e0), min(x1, e1), a.src, a.nsrc, a.lds, at, a.lg, acc);
        if (at.shift >= N) continue;
        Vec<float, N> o;
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = acc[i];
        store_vec<float, N>(a.part + (2 * q + z) * a.dp + at.c, o);
    }
}

// Targets t0 + j .. t0 + r - 1, whose entries are [x0, end): kSumEntries
// entries' packs are in flight at once, across targets.
template <typename T, int N, typename P, typename S>
__device__ inline void sum_run(const Sums<T, P>& a, int64_t t0, int j, int r, int64_t x0, int64_t end,
                               const S& start, const Place& at) {
    constexpr int E = kSumEntries;
    const int width = 1 << a.lg, l = lane_id() & (width - 1);
    float acc[N] = {};
    int64_t next = start(j + 1);
    auto flush = [&]() {
        Vec<T, N> o;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            o[i] = T(acc[i] * a.scale);
            acc[i] = 0.f;
        }
        if (at.shift < N) store_vec_nt<T, N>(a.out + (t0 + j) * a.ldo + at.c, o);
        ++j;
        if (j < r) next = start(j + 1);
    };
    for (int64_t base = x0; base < end; base += width) {
        int64_t row = -1;
        float w = 0.f;
        if (base + l < end) {
            row = load_column(a.t.from, a.t.ib, (base + l) * a.t.step);
            w = a.t.w ? load_value(a.t.w, a.t.wt, (base + l) * a.t.step) : 1.f;
            if (row < 0 || row >= a.nsrc) row = -1;
        }
        const int n = int(min(int64_t(width), end - base));
        for (int y = 0; y < n; y += E) {
            Vec<T, N> v[E];
            float wj[E];
#pragma unroll
            for (int x = 0; x < E; ++x) {
                int64_t q = __shfl(row, min(y + x, width - 1), width);
                wj[x] = __shfl(w, min(y + x, width - 1), width);
                if (y + x >= n) q = -1;
                // (nothing is read for padding, which adds zeros whatever its weight)
                if (q < 0) wj[x] = 0.f;
                v[x] = Vec<T, N>(T(0.f));
                if (q >= 0) v[x] = load_vec<T, N>(a.src + q * a.lds + at.c);
            }
#pragma unroll
            for (int x = 0; x < E; ++x) {
                if (y + x < n)
                    while (base + y + x >= next) flush();
#pragma unroll
                for (int i = 0; i < N; ++i) acc[i] = fmaf(wj[x], float(v[x][i]), acc[i]);
            }
        }
    }
    while (j < r) flush();
}

template <typename T, int N, typename P>
__global__ __launch_bounds__(kBlock) void sums_kernel(Sums<T, P> a) {
    const int lane = lane_id(), sub = lane >> a.lg, l = lane & ((1 << a.lg) - 1);
    const int rows = kWave >> a.lg;
    const int w = threadIdx.x / kWave;
    if (blockIdx.x < a.tile_blocks) {
        const int64_t end = a.t.at(a.t.targets);
        for (int64_t u = int64_t(blockIdx.x) * kWavesPerBlock + w; u < a.tile_units;
             u += int64_t(a.tile_blocks) * kWavesPerBlock) {
            const int64_t q = u / a.chunks * rows + sub;
            if (q < a.ntiles) sum_tile<T, N>(a, q, u % a.chunks, l, end);
        }
        return;
    }
    for (int64_t u = int64_t(blockIdx.x - a.tile_blocks) * kWavesPerBlock + w; u < a.target_units;
         u += int64_t(gridDim.x - a.tile_blocks) * kWavesPerBlock) {
        const int64_t t0 = (u / a.chunks * rows + sub) * a.per;
        if (t0 >= a.t.targets) continue;
        const Place at = place<N>((((u % a.chunks) << a.lg) + l) * N, a.d);
        // the starts of the group's targets, one per lane (per < 1 << lg, or one target)
        const int n = int(min(int64_t(a.per), a.t.targets - t0)), width = 1 << a.lg;
        const int64_t s = a.t.at(t0 + min(l, n));
        auto start = [&](int j) { return a.per == 1 ? a.t.at(t0 + j) : __shfl(s, j, width); };
        for (int j = 0; j < n;) {
            // a run of targets none of which is long: their entries follow one
            // another and are read without regard to where a target ends
            const int64_t x0 = start(j);
            int64_t end = x0;
            int r = j;
            for (; r < n; ++r) {
                const int64_t next = start(r + 1);
                if (next - end > a.tile) break;
                end = next;
            }
            if (r > j)
                sum_run<T, N>(a, t0, j, r, x0, end, start, at);
            else
                ++r;
            j = r;
        }
    }
}

// The long target that starts in tile q, if any (it holds the tile's last
// entry): its parts in tile order within a wavefront, the wavefronts' in
// theirs; 256 columns at a time.
template <typename T, typename P>
__global__ __launch_bounds__(kBlock) void join_tiles(Sums<T, P> a) {
    __shared__ float4 sum[kWavesPerBlock][kWave];
    const int64_t q = blockIdx.x;
    const int z = a.long_of[2 * q + 1] >= 0 ? 1 : 0;
    const int64_t target = a.long_of[2 * q + z];
    if (target < 0) return;
    const int64_t x0 = a.t.at(target), x1 = a.t.at(target + 1);
    if (x1 <= x0 || x0 / a.tile != q) return;
    const int64_t tiles = min((x1 - 1) / a.tile, a.ntiles - 1) - q + 1;
    const int w = threadIdx.x / kWave, l = lane_id();
    const int64_t per = (tiles + kWavesPerBlock - 1) / kWavesPerBlock;
    const float* p = a.part + 2 * q * a.dp;
    for (int64_t c = int64_t(blockIdx.y) * 4 * kWave + 4 * l; c - 4 * l < a.d; c += int64_t(gridDim.y) * 4 * kWave) {
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c < a.d) {
            const int64_t end = min(tiles, (w + 1) * per);
#pragma unroll 4
            for (int64_t x = w * per; x < end; ++x) {
                const float4 v = *reinterpret_cast<const float4*>(p + (2 * x + (x == 0 ? z : 0)) * a.dp + c);
                s.x += v.x;
                s.y += v.y;
                s.z += v.z;
                s.w += v.w;
            }
        }
        sum[w][l] = s;
        __syncthreads();
        if (w == 0 && c < a.d) {
#pragma unroll
            for (int i = 1; i < kWavesPerBlock; ++i) {
                const float4 v = sum[i][l];
                s.x += v.x;
                s.y += v.y;
                s.z += v.z;
                s.w += v.w;
            }
            const float r[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (c + i < a.d) a.out[target * a.ldo + c + i] = T(r[i] * a.scale);
        }
        __syncthreads();
    }
}

// Entries per tile: 64 for up to 2^16 entries, doubled for every fourfold of
// them, so that neither a tile nor the parts of one target grow past the square
// root of the entries by much.
inline int64_t doubled(int64_t t, int64_t per, int64_t nnz) {
    while (t * t * per < nnz) t *= 2;
    return t;
}
inline int64_t row_tile(int64_t nnz) { return doubled(64, 16, nnz); }

// The gradient's tiles start at 16: a frequent token's column, or a tile of it,
// is a chain of reads, and short chains are what few entries need (4096 tokens
// over 32000 x 64 bf16: 37 us with 64, 23 with 16; 8192 over 32000 x 4096: 141
// and 135).  Rows of up to 256 columns, whose parts cost little, keep tiles half
// as long (30000 tokens over 100000 x 64 bf16: 43 us, 37 so; 1.57 M entries over
// 3000 x 250 f32: 338 and 301; but 8192 tokens over 32000 x 4096: 134 and 136).
// Up to 1024 entries few columns are long, and parts cost more than they save
// (512 tokens over 50000 x 1024: 26.6 us, 27.7 with tiles of 16).  Rows of a
// CSR keep to the longer tiles, as typical ones would otherwise go through parts.
inline int64_t column_tile(int64_t nnz, int64_t d) {
    return nnz <= 1024 ? row_tile(nnz) : doubled(16, d <= 256 ? 64 : 16, nnz);
}

inline size_t round256(size_t b) { return (b + 255) & ~size_t(255); }

inline int64_t part_columns(int64_t d) { return (d + 3) & ~int64_t(3); }

inline size_t part_bytes(int64_t nnz, int64_t tile, int64_t d) {
    if (nnz <= tile) return 0;
    const size_t rows = size_t((nnz + tile - 1) / tile) * 2;
    return round256(rows * size_t(part_columns(d)) * sizeof(float)) + round256(rows * sizeof(int32_t));
}

template <typename T, int N, typename P>
void launch_sums(const Targets<P>& t, const DenseRows& src, float scale, const DenseRows& out, void* tmp,
                 int64_t tile, int64_t packs, int lg, hipStream_t s) {
    Sums<T, P> a;
    a.t = t;
    a.src = static_cast<const T*>(src.p);
    a.nsrc = src.m;
    a.lds = src.ld;
    a.d = out.n;
    a.scale = scale;
    a.out = static_cast<T*>(out.p);
    a.ldo = out.ld;
    a.lg = lg;
    a.chunks = (packs + (int64_t(1) << lg) - 1) >> lg;
    const int64_t rows = kWave >> lg;
    a.tile = tile;
    a.ntiles = t.nnz > a.tile ? (t.nnz + a.tile - 1) / a.tile : 0;  // (no target is long)
    a.dp = part_columns(a.d);
    a.part = static_cast<float*>(tmp);
    a.long_of = reinterpret_cast<int32_t*>(static_cast<char*>(tmp) +
                                           round256(size_t(a.ntiles) * 2 * size_t(a.dp) * sizeof(float)));
    a.tile_units = (a.ntiles + rows - 1) / rows * a.chunks;
    a.tile_blocks = a.ntiles ? grid_for(a.tile_units) : 0;
    // Eight targets of a group of lanes follow one another where there are many
    // (from 2^15 on), so that short ones do not wait for each other: gradients of
    // 8192 tokens over 32768 x 4096 bf16 take 67 us, 139 with one target each, of
    // 65536 over 32768 x 256 45 and 51, of 512 over 131072 x 1024 56 and 114.
    // Where few targets hold many entries each, the wavefronts are too few then
    // (65536 tokens over 4096 x 256: 64 us, 43 with one each; 16384 rows of 24
    // over 4096 x 128 f32, looked up: 56 and 27).  The limit is on the safe side:
    // tables of 16384 and 32000 rows under few tokens are past the turn already
    // (8192 tokens over 32000 x 4096: 135 us with one each, 66 with eight), while
    // a lookup of long rows is not yet (65537 rows of 24 over 200003 x 250 f32:
    // 273 us with eight, 250 with one).
    a.per = lg >= 4 && t.targets >= (int64_t(1) << 15) ? 8 : 1;
    a.target_units = (t.targets + rows * a.per - 1) / (rows * a.per) * a.chunks;
    sums_kernel<T, N, P><<<a.tile_blocks + grid_for(a.target_units), kBlock, 0, s>>>(a);
    if (a.ntiles)
        join_tiles<T, P><<<dim3(unsigned(a.ntiles), unsigned(std::min<int64_t>((a.d + 255) / 256, 16))), kBlock, 0,
                           s>>>(a);
}

template <typename P>
void grouped_sums(const Targets<P>& t, const DenseRows& src, float scale, const DenseRows& out, void* tmp,
                  int64_t tile, hipStream_t s) {
    by_width(out.dt, out.n, [&](auto e, auto width) {
        using T = decltype(e);
        constexpr int N = decltype(width)::value;
        const int64_t packs = (out.n + N - 1) / N;
        const int lg = lane_bits(packs);
        launch_sums<T, N, P>(t, src, scale, out, tmp, tile, packs, lg, s);
    });
}

// ---- the gradient's entries sorted by column

// The row that holds entry e, found by a whole wavefront: 64 probes a step.
// (Any row pointers end the search, inside [0, m).)
__device__ inline int64_t row_of(const int64_t* rp, int64_t m, int64_t e) {
    int64_t lo = 0, hi = m - 1;
    while (lo < hi) {
        const int64_t n = hi - lo, step = (n + kWave - 1) / kWave;
        const uint64_t below = __ballot(rp[lo + min((lane_id() + 1) * step, n)] <= e);
        const int64_t c = below == ~uint64_t(0) ? kWave : __builtin_ctzll(~below);
        hi = min(hi, lo + (c + 1) * step - 1);
        lo += min(c * step, n);
    }
    return max(lo, int64_t(0));
}

// start[c] = sorted entries of columns before c, c = 0 .. n
__global__ __launch_bounds__(kBlock) void column_bounds(const uint32_t* __restrict__ key, int64_t nnz, int64_t n,
                                                        uint32_t* __restrict__ start) {
    const int64_t stride = int64_t(gridDim.x) * kBlock;
    for (int64_t c = int64_t(blockIdx.x) * kBlock + threadIdx.x; c <= n; c += stride)
        start[c] = uint32_t(lower_bound_u32(key, 0, nnz, uint64_t(c)));
}

// Up to kFewEntries entries over up to 2^19 columns are sorted in two launches,
// against three or four per digit and two more of the radix sort, which for so
// few records is mostly launches and latency (65536 tokens of 131072: 17 us,
// 65 by digits; 1.57 M weighted CSR entries of 200003: 67 us, 121 by digits).
// The columns are dealt to at most kSortGroups groups of consecutive columns.
// First, tiles of entries are split by group (stable, padding left out), with
// every tile's first record of every group; then one workgroup per group takes
// its records from the tiles in order and sorts them by column: rows, or with
// weights pairs of row and weight.
constexpr int kSortBlock = 1024;
constexpr int kSortWaves = kSortBlock / kWave;
constexpr int kSortBins = 1024;   // columns per group, at most
constexpr int kSortGroups = 512;
constexpr int kSortBatch = 4;     // groups of 64 records read at once
constexpr int kSortTiles = 1024;  // tiles, at most
constexpr int kSortItems = 4;     // entries per thread of a tile, past kSmallEntries
constexpr int64_t kSmallEntries = int64_t(1) << 17;
constexpr int64_t kFewEntries = int64_t(kSortTiles) * kSortBlock * kSortItems;

// Lanes of the wavefront with a lane's value (of `bits` bits), among those of `in`.
__device__ inline uint64_t lanes_of(uint32_t x, int bits, bool in) {
    uint64_t same = __ballot(in);
    for (int b = 0; b < bits; ++b) {
        const bool one = (x >> b) & 1;
        const uint64_t m = __ballot(one);
        same &= one ? m : ~m;
    }
    return same;
}

// LDS accesses of a wavefront before and after it stay in order (the hardware
// keeps them so; rows of hist are used by one wavefront each).
__device__ inline void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
}

// Turns the counts hist[wavefront][x], x < n <= kSortBlock, into first places
// from `first` on, by x and then by wavefront; returns x's first place to
// thread x and the end to all.
template <int W>
__device__ inline uint32_t places(uint32_t (*hist)[W], int n, uint32_t first, uint32_t* scratch, uint32_t* end) {
    uint32_t own = 0, total;
    const int x = threadIdx.x;
    if (x < n)
        for (int i = 0; i < kSortWaves; ++i) own += hist[i][x];
    const uint32_t at = first + block_exclusive_scan<uint32_t, kSortBlock>(own, scratch, &total);
    uint32_t next = at;
    if (x < n)
        for (int i = 0; i < kSortWaves; ++i) {
            const uint32_t c = hist[i][x];
            hist[i][x] = next;
            next += c;
        }
    *end = first + total;
    __syncthreads();
    return at;
}

// Rows of the entries [e0, e1) of a workgroup: the pointers of theirs are
// searched in LDS where they fit, else in memory (every thread calls find_rows).
constexpr int kRecordRows = 2048;
struct RowFinder {
    int64_t r0, n;
    const int64_t* ptr;
    __device__ inline int64_t row(int64_t e) const {
        if (!ptr) return e;
        int64_t lo = 0, hi = n - 1;
        while (lo < hi) {
            const int64_t mid = (lo + hi + 1) >> 1;
            if (ptr[mid] <= e)
                lo = mid;
            else
                hi = mid - 1;
        }
        return r0 + lo;
    }
};
template <int NT>
__device__ inline RowFinder find_rows(const Entries& A, int64_t e0, int64_t e1, int64_t* range, int64_t* ptr) {
    if (!A.rp) return {0, 0, nullptr};
    __syncthreads();
    const int w = threadIdx.x / kWave;
    if (w < 2) {
        const int64_t r = row_of(A.rp, A.m, w ? e1 - 1 : e0);
        if (lane_id() == 0) range[w] = r;
    }
    __syncthreads();
    const int64_t r0 = range[0], n = range[1] - r0 + 1;
    if (n < 1 || n > kRecordRows) return {0, A.m, A.rp};
    for (int i = threadIdx.x; i < n; i += NT) ptr[i] = A.rp[r0 + i];
    __syncthreads();
    return {r0, n, ptr};
}

template <typename I, int ITEMS>
__global__ __launch_bounds__(kSortBlock) void split_entries(Entries A, int lgbins, int groups, int bits,
                                                            uint2* __restrict__ rec, float* __restrict__ recw,
                                                            uint32_t* __restrict__ first) {
    __shared__ uint32_t hist[kSortWaves][kSortGroups];
    __shared__ uint32_t scratch[kSortWaves];
    __shared__ int64_t range[2], ptr[kRecordRows];
    const int w = threadIdx.x / kWave, l = lane_id();
    for (int i = threadIdx.x; i < kSortWaves * kSortGroups; i += kSortBlock) hist[0][i] = 0;
    const int64_t base = int64_t(blockIdx.x) * kSortBlock * ITEMS;
    // a wavefront's entries are consecutive
    const int64_t e0 = base + int64_t(w) * kWave * ITEMS + l;
    const I* idx = static_cast<const I*>(A.idx);
    const int64_t stride = A.rp ? 1 : A.istride;
    I t[ITEMS];
    float wv[ITEMS];
    uint32_t rank[ITEMS];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        const int64_t e = e0 + k * kWave;
        t[k] = e < A.nnz ? idx[e * stride] : I(-1);
        wv[k] = recw && e < A.nnz ? load_value(A.val, A.vt, e) : 0.f;
    }
    const RowFinder rows = find_rows<kSortBlock>(A, base, min(A.nnz, base + kSortBlock * ITEMS), range, ptr);
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
        if (t[k] >= A.n) t[k] = -1;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        const bool in = t[k] >= 0;
        const uint32_t g = in ? uint32_t(t[k]) >> lgbins : 0;
        const uint64_t same = lanes_of(g, bits, in);
        const uint32_t lower = __popcll(same & lanemask_lt());
        rank[k] = hist[w][g] + lower;
        wave_order();
        if (in && lower == 0) hist[w][g] += __popcll(same);
        wave_order();
    }
    __syncthreads();
    uint32_t end;
    const uint32_t at = places(hist, groups, 0, scratch, &end);
    uint32_t* f = first + int64_t(blockIdx.x) * (groups + 1);
    if (int(threadIdx.x) < groups) f[threadIdx.x] = at;
    if (threadIdx.x == 0) f[groups] = end;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        if (t[k] < 0) continue;
        const int64_t e = e0 + k * kWave;
        const int64_t pos = base + hist[w][uint32_t(t[k]) >> lgbins] + rank[k];
        rec[pos] = make_uint2(uint32_t(t[k]), uint32_t(rows.row(e)));
        if (recw) recw[pos] = wv[k];
    }
}

__global__ __launch_bounds__(kSortBlock) void sort_groups(const uint2* __restrict__ rec,
                                                          const float* __restrict__ recw,
                                                          const uint32_t* __restrict__ first, int tiles, int tile,
                                                          int groups, int lgbins, int64_t v,
                                                          uint32_t* __restrict__ start, int part,
                                                          uint32_t* __restrict__ key, uint32_t* __restrict__ row) {
    __shared__ uint32_t hist[kSortWaves][kSortBins];
    __shared__ uint32_t scratch[kSortWaves];
    __shared__ uint32_t upto[kSortTiles + 1], from[kSortTiles];  // the group's records before each tile, and in it
    const int g = blockIdx.x, bins = 1 << lgbins;
    const int w = threadIdx.x / kWave, l = lane_id();
    for (int i = threadIdx.x; i < kSortWaves * bins; i += kSortBlock) hist[i >> lgbins][i & (bins - 1)] = 0;
    uint32_t before = 0, count = 0;
    if (int(threadIdx.x) < tiles) {
        const uint32_t* f = first + int64_t(threadIdx.x) * (groups + 1) + g;
        before = f[0];
        count = f[1] - before;
        from[threadIdx.x] = threadIdx.x * tile + before;
    }
    uint32_t m, all;
    const uint32_t mine = block_exclusive_scan<uint32_t, kSortBlock>(count, scratch, &m);
    (void)block_exclusive_scan<uint32_t, kSortBlock>(before, scratch, &all);
    upto[threadIdx.x] = mine;  // (m past the tiles)
    if (threadIdx.x == 0) upto[kSortTiles] = m;
    __syncthreads();
    // records of consecutive stretches, whole groups of 64, one stretch per wavefront
    const uint32_t per = ((m + kSortWaves - 1) / kSortWaves + kWave - 1) / kWave * kWave;
    const uint32_t i0 = w * per, i1 = min(m, i0 + per);
    const uint32_t lo = uint32_t(g) << lgbins;
    uint2 r[kSortBatch];
    float rw[kSortBatch];
    auto load = [&](uint32_t base) {
#pragma unroll
        for (int k = 0; k < kSortBatch; ++k) {
            const uint32_t i = base + k * kWave + l;
            r[k] = make_uint2(~0u, 0u);
            if (i < i1) {
                const int q = upper_bound_lds(upto, 0, tiles, i) - 1;
                const uint32_t src = from[q] + (i - upto[q]);
                r[k] = rec[src];
                if (recw) rw[k] = recw[src];
            }
        }
    };
    for (uint32_t i = i0; i < i1; i += kSortBatch * kWave) {
        load(i);
#pragma unroll
        for (int k = 0; k < kSortBatch; ++k)
            if (r[k].x != ~0u) atomicAdd(&hist[w][r[k].x - lo], 1u);
    }
    __syncthreads();
    uint32_t end;
    const uint32_t at = places(hist, bins, all, scratch, &end);
    if (int(threadIdx.x) < bins && int64_t(lo) + threadIdx.x < v) start[lo + threadIdx.x] = at;
    if (g == groups - 1 && threadIdx.x == 0) start[v] = end;
    for (uint32_t i = i0; i < i1; i += kSortBatch * kWave) {
        if (per > kSortBatch * kWave) load(i);  // (else they are still held)
#pragma unroll
        for (int k = 0; k < kSortBatch; ++k) {
            const bool in = r[k].x != ~0u;
            const uint32_t bin = in ? r[k].x - lo : 0;
            const uint64_t same = lanes_of(bin, lgbins, in);
            const uint32_t rank = __popcll(same & lanemask_lt());
            if (in) {
                const uint32_t pos = hist[w][bin] + rank;
                if (recw)
                    reinterpret_cast<uint2*>(row)[pos] = make_uint2(r[k].y, __float_as_uint(rw[k]));
                else
                    row[pos] = r[k].y;
                // (the sums ask for the columns of their tiles' first and last entries)
                if (pos % part == 0 || pos % part == part - 1 || pos == end - 1) key[pos] = r[k].x;
            }
            wave_order();
            if (in && rank == 0) hist[w][bin] += __popcll(same);
            wave_order();
        }
    }
}

// Sort records of the radix sort: the column (n for padding, which sorts past
// every column), the row and the weight of every entry.
constexpr int kRecords = 2048;
__global__ __launch_bounds__(kBlock) void sort_records(Entries A, uint32_t* __restrict__ key,
                                                       uint32_t* __restrict__ row, float* __restrict__ w) {
    __shared__ int64_t range[2], ptr[kRecordRows];
    for (int64_t e0 = int64_t(blockIdx.x) * kRecords; e0 < A.nnz; e0 += int64_t(gridDim.x) * kRecords) {
        const int64_t e1 = min(A.nnz, e0 + kRecords);
        const RowFinder rows = find_rows<kBlock>(A, e0, e1, range, ptr);
        for (int64_t e = e0 + threadIdx.x; e < e1; e += kBlock) {
            const int64_t c = load_column(A.idx, A.ib, A.rp ? e : e * A.istride);
            key[e] = uint32_t(c >= 0 && c < A.n ? c : A.n);
            row[e] = uint32_t(rows.row(e));
            if (w) w[e] = load_value(A.val, A.vt, e);
        }
    }
}

// One launch for tokens that one workgroup holds: every group's workgroup reads
// them all, one a thread, and sorts its own.
template <typename I>
__global__ __launch_bounds__(kSortBlock) void sort_few_tokens(Entries A, int groups, int lgbins,
                                                              uint32_t* __restrict__ start, int part,
                                                              uint32_t* __restrict__ key,
                                                              uint32_t* __restrict__ row) {
    __shared__ uint32_t hist[kSortWaves][kSortBins];
    __shared__ uint32_t scratch[kSortWaves], lower_s[kSortWaves];
    const int g = blockIdx.x, bins = 1 << lgbins, w = threadIdx.x / kWave;
    const int64_t lo = int64_t(g) << lgbins, e = threadIdx.x;
    int64_t t = e < A.nnz ? int64_t(static_cast<const I*>(A.idx)[e * A.istride]) : -1;
    if (t >= A.n) t = -1;
    for (int i = threadIdx.x; i < kSortWaves * bins; i += kSortBlock) hist[i >> lgbins][i & (bins - 1)] = 0;
    const uint64_t lower = __ballot(t >= 0 && t < lo);
    if (lane_id() == 0) lower_s[w] = __popcll(lower);
    const bool in = t >= lo && t < lo + bins;
    const uint32_t bin = in ? uint32_t(t - lo) : 0;
    const uint64_t same = lanes_of(bin, lgbins, in);
    const uint32_t rank = __popcll(same & lanemask_lt());
    __syncthreads();
    if (in && rank == 0) hist[w][bin] = __popcll(same);
    uint32_t before = 0, end;
#pragma unroll
    for (int i = 0; i < kSortWaves; ++i) before += lower_s[i];
    __syncthreads();
    const uint32_t at = places(hist, bins, before, scratch, &end);
    if (int(threadIdx.x) < bins && lo + threadIdx.x < A.n) start[lo + threadIdx.x] = at;
    if (g == groups - 1 && threadIdx.x == 0) start[A.n] = end;
    if (in) {
        const uint32_t pos = hist[w][bin] + rank;
        row[pos] = uint32_t(e);
        if (pos % part == 0 || pos % part == part - 1 || pos == end - 1) key[pos] = uint32_t(t);
    }
}

// log2 of the columns per group (-1: the entries go by the radix sort)
inline int few_entries_bins(const Entries& A) {
    if (A.nnz > kFewEntries || A.n > int64_t(kSortBins) * kSortGroups) return -1;
    int lg = 0;
    const int64_t groups = A.nnz > kSmallEntries ? kSortGroups : 256;
    while ((groups << lg) < A.n && (1 << lg) < kSortBins) ++lg;
    return lg;
}

inline unsigned thread_grid(int64_t n) {
    return unsigned(std::min<int64_t>((n + kBlock - 1) / kBlock, int64_t(1) << 16));
}

}  // namespace

void embed_tokens(const Entries& A, const DenseRows& W, float scale, const DenseRows& Y, hipStream_t s) {
    by_width(Y.dt, Y.n, [&](auto e, auto width) {
        using T = decltype(e);
        constexpr int N = decltype(width)::value;
        const int64_t packs = (Y.n + N - 1) / N;
        const int lg = lane_bits(packs);
        const int64_t per = packs <= kWave ? 1 : kUnroll;
        const int64_t chunks = (packs + (per << lg) - 1) / (per << lg);
        const int64_t rows = kWave >> lg;
        const int64_t units = (A.m + rows - 1) / rows * chunks;
        const T* w = static_cast<const T*>(W.p);
        T* y = static_cast<T*>(Y.p);
        if constexpr (N > 1)
            if (per > 1) {
                tokens_kernel<T, N, kUnroll><<<grid_for(units), kBlock, 0, s>>>(A, w, W.ld, Y.n, scale, y, Y.ld, lg,
                                                                                chunks, units);
                return;
            }
        tokens_kernel<T, N, 1><<<grid_for(units), kBlock, 0, s>>>(A, w, W.ld, Y.n, scale, y, Y.ld, lg, chunks, units);
    });
}

size_t embed_csr_tmp_bytes(int64_t nnz, int64_t d) {
    return part_bytes(nnz, row_tile(nnz), d);
}

void embed_csr(const Entries& A, const DenseRows& W, float scale, const DenseRows& Y, void* tmp, hipStream_t s) {
    Targets<int64_t> t{A.rp, A.m, A.nnz, A.idx, A.ib, A.val, A.vt, nullptr, 1};
    grouped_sums(t, W, scale, Y, tmp, row_tile(A.nnz), s);
}

// entries per tile of the two-launch sort
static int sort_tile(int64_t nnz) { return nnz <= kSmallEntries ? kSortBlock : kSortBlock * kSortItems; }

// Scratch of the sort: the radix sort's, or every tile's first records by group.
static size_t sort_scratch_bytes(const Entries& A) {
    if (few_entries_bins(A) < 0) return round256(radix_tmp_bytes(A.nnz));
    const int tile = sort_tile(A.nnz);
    return round256(size_t((A.nnz + tile - 1) / tile) * (kSortGroups + 1) * sizeof(uint32_t));
}

// Bytes of each of the sort's buffers: keys, rows and weights, sorted and
// before.  (Key and row before the sort hold the split's records, which end at
// most a tile past the entries.)
static size_t sort_buffer_bytes(int64_t nnz) {
    return round256((size_t(nnz) + kSortBlock * kSortItems) * sizeof(uint32_t));
}

size_t embed_grad_tmp_bytes(const Entries& A, int64_t d) {
    return sort_buffer_bytes(A.nnz) * (A.val ? 6 : 4) + round256(size_t(A.n + 1) * sizeof(uint32_t)) +
           sort_scratch_bytes(A) + part_bytes(A.nnz, column_tile(A.nnz, d), d);
}

void embed_grad(const Entries& A, const DenseRows& G, float scale, const DenseRows& dW, void* tmp, hipStream_t s) {
    char* at = static_cast<char*>(tmp);
    auto take = [&](size_t bytes) {
        char* p = at;
        at += round256(bytes);
        return p;
    };
    const size_t words = sort_buffer_bytes(A.nnz);
    uint32_t* start = reinterpret_cast<uint32_t*>(take(size_t(A.n + 1) * sizeof(uint32_t)));
    uint32_t *key[2], *row[2];
    float* w[2];
    for (int i = 0; i < 2; ++i) {
        key[i] = reinterpret_cast<uint32_t*>(take(words));
        row[i] = reinterpret_cast<uint32_t*>(take(words));
        w[i] = A.val ? reinterpret_cast<float*>(take(words)) : nullptr;
    }
    void* sort_tmp = take(sort_scratch_bytes(A));
    const int64_t sums_tile = column_tile(A.nnz, dW.n);
    int which = 0, step = 1;
    const int lgbins = few_entries_bins(A);
    if (lgbins >= 0) {
        const int groups = int((A.n + (int64_t(1) << lgbins) - 1) >> lgbins);
        const int tile = sort_tile(A.nnz);
        const int tiles = int((A.nnz + tile - 1) / tile);
        const int bits = bit_width_u64(uint64_t(groups - 1));
        uint2* rec = reinterpret_cast<uint2*>(key[1]);  // (two of the sort's buffers)
        uint32_t* first = static_cast<uint32_t*>(sort_tmp);
        auto split = [&](auto kernel) {
            kernel<<<tiles, kSortBlock, 0, s>>>(A, lgbins, groups, bits, rec, w[1], first);
        };
        const int part = int(sums_tile);
        const bool one = !A.rp && A.nnz <= kSortBlock;
        if (one) {
            auto sort = [&](auto kernel) {
                kernel<<<groups, kSortBlock, 0, s>>>(A, groups, lgbins, start, part, key[0], row[0]);
            };
            A.ib == 4 ? sort(sort_few_tokens<int32_t>) : sort(sort_few_tokens<int64_t>);
        } else if (tiles > 0) {
            if (tile == kSortBlock)
                A.ib == 4 ? split(split_entries<int32_t, 1>) : split(split_entries<int64_t, 1>);
            else
                A.ib == 4 ? split(split_entries<int32_t, kSortItems>) : split(split_entries<int64_t, kSortItems>);
        }
        // (row[0] and w[0] hold the pairs)
        if (!one)
            sort_groups<<<groups, kSortBlock, 0, s>>>(rec, w[1], first, tiles, tile, groups, lgbins, A.n, start, part,
                                                      key[0], row[0]);
        if (A.val) {
            w[0] = reinterpret_cast<float*>(row[0]) + 1;
            step = 2;
        }
    } else if (A.nnz > 0) {
        sort_records<<<unsigned(std::min<int64_t>((A.nnz + kRecords - 1) / kRecords, 1 << 16)), kBlock, 0, s>>>(A, key[0], row[0], w[0]);
        which = radix_sort(key[0], key[1], row[0], row[1], w[0], w[1], A.val ? 4 : 0, A.nnz,
                           bit_width_u64(uint64_t(A.n)), sort_tmp, s);
    }
    if (lgbins < 0) column_bounds<<<thread_grid(A.n + 1), kBlock, 0, s>>>(key[which], A.nnz, A.n, start);
    Targets<uint32_t> t{start, A.n, A.nnz, row[which], 4, w[which], kDtF32, key[which], step};
    grouped_sums(t, G, scale, dW, at, sums_tile, s);
}

}  // namespace spsyrk
