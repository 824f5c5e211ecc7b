// Products of tiles on the matrix cores: out[n][m] = sum over k of A(m, k) B(n, k),
// 32-bit sums.  An operand's elements lie in rows of k (one row for each m or n),
// or turned: in rows of m or n, one for each k.
//
// A workgroup of WM x WN wavefronts takes a tile of BM x BN and walks k in steps
// of 128 bytes' elements.  A step's part of an operand goes from memory into LDS
// without passing through registers, in two buffers; the fragments of a half step
// are read from LDS while the half step before is multiplied, so that the matrix
// cores wait neither for LDS nor, but where a step takes less time than memory
// needs, for the loads.  One barrier a step: it stands where a buffer's last
// fragments have been read and the other buffer has landed.  (Products alone,
// 4096 x 4096 x 131072 bf16: 1376 TFLOP/s; with a barrier around each step
// and fragments read by the step that uses them 1255; matrix instructions of 32
// rows 1272.)
//
// LDS holds what the loads write in lane order; which chunk a lane fetches is
// chosen so that reads touch all banks once.  Rows of k: chunk c of row r stands
// at c ^ (r % 8).  Turned rows of 16-bit elements are read transposed by the
// hardware, four rows of 16 elements at a time by 16 lanes: pair p of 16-byte
// chunks of row k stands at p ^ (k % 4 + 4 (k / 8 % 2)).  (A turned operand costs its
// product about a tenth, a transposed copy of W or G before it more: 131072 x 4096
// bf16 860 us.)  Of 32-bit elements:
// group of 16 elements at p ^ (k / 4 % 4).  Rows past an operand's end are zeros;
// what lies past a turned row's end goes into products that are not stored.
//
// A is the operand whose rows become the contiguous dimension of the output: a
// lane holds four consecutive m of one n.
#pragma once

#include "rows.h"

namespace spsyrk {

typedef float F4 __attribute__((ext_vector_type(4)));

// a 16-byte chunk of k per lane: 16 rows of A by 16 rows of B, four chunks of k
template <typename T>
struct Chunk;
template <>
struct Chunk<__bf16> {
    typedef __bf16 V __attribute__((ext_vector_type(8)));
    __device__ static F4 mul(V a, V b, F4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Chunk<_Float16> {
    typedef _Float16 V __attribute__((ext_vector_type(8)));
    __device__ static F4 mul(V a, V b, F4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <>
struct Chunk<float> {
    typedef float V __attribute__((ext_vector_type(4)));
    // (k's order within a chunk is the same for both operands, which is all that counts)
    __device__ static F4 mul(V a, V b, F4 c) {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
        return c;
    }
};

constexpr int kStepBytes = 128;  // of k, per row and step
inline int step_elements(int dt) { return kStepBytes / dtype_bytes(dt); }

// An operand of `rows` m or n, on 16-byte boundaries and strides of 16 bytes below
// kMostStride.  In rows of k: a whole number of steps, with zeros past its end.
// Turned: `depth` rows.
constexpr int64_t kMostStride = int64_t(1) << 24;  // bytes: 256 rows in 32-bit offsets
struct Operand {
    const void* p = nullptr;
    int64_t ld = 0;
    int64_t rows = 0;
    int64_t depth = 0;
};

// A tile's place among tm x tn: XCDs take the workgroups in turn, so each gets
// a contiguous part of an order in which bands of eight n walk over m; the
// workgroups of an XCD then share their rows in its L2.
struct TileAt {
    int m, n;
};
__device__ inline TileAt tile_at(int64_t id, int64_t tm, int64_t tn) {
    const int64_t total = tm * tn, per = total / kXcds, rest = total % kXcds;
    const int64_t x = id % kXcds, j = id / kXcds;
    const int64_t t = x * per + min(x, rest) + j;
    constexpr int64_t BAND = 8;
    const int64_t band = t / (BAND * tm), in = t % (BAND * tm);
    const int64_t wide = min(BAND, tn - band * BAND);
    return {int(in / wide), int(band * BAND + in % wide)};
}

// what a wavefront loads and reads of one operand; R: the tile's rows of it
template <typename T, int R, int WAVES, bool TURNED>
struct Side {
    static constexpr int CHUNK = 16 / int(sizeof(T)), STEP = kStepBytes / int(sizeof(T));
    static constexpr int LOADS = R / 8 / WAVES;  // of a wavefront per step, 1 KB each
    static_assert(LOADS * 8 * WAVES == R, "whole loads");
    static constexpr int ROW = TURNED ? R * int(sizeof(T)) : kStepBytes;  // bytes of a row in LDS
    static constexpr int PER = 1024 / ROW;                                // rows of a load
    using V = typename Chunk<T>::V;

    // The loads of a lane are EVERY rows apart, which leaves a turned row's XOR the
    // same (of 32-bit elements: every second one's), so that one offset (two) and
    // multiples of a stride make all of them.  Offsets are 32 bits from the tile's
    // first row (turned: the step's), past the operand's end the loads give zeros.
    static constexpr int EVERY = WAVES * PER, SAME = TURNED && EVERY < 16 ? 16 / EVERY : 1;

    const char* base;
    int64_t left;          // bytes from base to the operand's end
    int64_t stride;        // turned: bytes from step to step
    uint32_t from[SAME], ld;
    int at, turned;        // this lane's part of a fragment's place in LDS, and of a turned row's XOR

    __device__ static int turn(int k) {
        return sizeof(T) == 2 ? (k & 3) | (k >> 3 & 1) << 2 : k >> 2 & 3;
    }
    static constexpr int UNIT = sizeof(T) == 2 ? 32 : 64;  // bytes that the XOR keeps together
    // (a value to be computed with where it is used: the places of all fragments
    // and the offsets of all loads, computed ahead, would take the sums' registers)
    template <typename I>
    __device__ static I opaque(I v) {
        asm volatile("" : "+v"(v));
        return v;
    }

    __device__ void init(const Operand& o, int64_t r0, int wave, int lane) {
        base = static_cast<const char*>(o.p);
        const int64_t wide = o.ld * int64_t(sizeof(T));
        ld = uint32_t(wide);
        if constexpr (TURNED) {
            base += r0 * int64_t(sizeof(T));
            stride = wide * STEP;
            // (the last row ends with its last pack, not with the stride)
            left = (o.depth - 1) * wide + (o.rows + CHUNK - 1) / CHUNK * 16 - r0 * int64_t(sizeof(T));
            const int within = lane * 16 % ROW, first = wave * PER + lane * 16 / ROW;
#pragma unroll
            for (int i = 0; i < SAME; ++i) {
                const int k = first + i * EVERY;
                from[i] = uint32_t(k) * ld + uint32_t((within / UNIT ^ turn(k)) * UNIT + within % UNIT);
            }
            const int g = lane >> 4;
            if constexpr (sizeof(T) == 2) {
                at = (g * 8 + (lane & 15) / 4) * ROW + (lane & 3) * 8;
                turned = ((lane & 15) / 4 | (g & 1) << 2) * UNIT;
            } else {
                at = g * 4 * ROW + (lane & 15) * 4;
                turned = g * UNIT;
            }
        } else {
            base += r0 * wide;
            stride = 0;
            left = (o.rows - r0) * wide;
            from[0] = uint32_t(wave * 8 + (lane >> 3)) * ld + uint32_t(((lane & 7) ^ (lane >> 3)) * 16);
            // (chunk lane / 16 of row lane % 16; the other half step's is four on)
            at = (lane & 15) * kStepBytes + ((lane >> 4) ^ (lane & 7)) * 16;
        }
    }

    // a step's rows into LDS (the operand's part of a buffer)
    __device__ void fetch(int64_t step, unsigned char* lds, int wave) const {
        typedef __attribute__((address_space(3))) void* Local;
        const int64_t bytes = left - step * stride;
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base + step * stride), 0,
                                                            int(uint32_t(min(bytes, int64_t(0xffffffff)))), 0x00020000);
        uint32_t start[SAME];
#pragma unroll
        for (int i = 0; i < SAME; ++i) start[i] = opaque(from[i]);
        // (the scalar offset takes no part in the bounds: straight rows have theirs
        // by the row, and a step lies within one)
        const int go = TURNED ? 0 : int(step * kStepBytes);
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (Local)(lds + (i * WAVES + wave) * 1024), 16,
                                                     int(start[i % SAME] + uint32_t(i / SAME * SAME * EVERY) * ld), go,
                                                     0, 0);
    }

    // where this lane reads the fragments of half step s (of rows from f on, with
    // the fragment's own part in read)
    __device__ const unsigned char* place(const unsigned char* lds, int f, int s) const {
        if constexpr (!TURNED)
            return lds + f * 16 * kStepBytes + (opaque(at) ^ s * 64);
        else
            return lds + opaque(at) + s * (STEP / 2) * ROW;
    }
    // fragment f + q (16 rows)
    __device__ V read(const unsigned char* place, int f, int q) const {
        if constexpr (!TURNED) {
            return *reinterpret_cast<const V*>(place + q * 16 * kStepBytes);
        } else if constexpr (sizeof(T) == 2) {
            typedef short S4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) S4* Local;
            const unsigned char* p = place + ((f + q) * UNIT ^ opaque(turned));
            const S4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Local)(p));
            const S4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Local)(p + 4 * ROW));
            return __builtin_bit_cast(V, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            const unsigned char* p = place + ((f + q) * UNIT ^ opaque(turned));
            V v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const float*>(p + j * ROW);
            return v;
        }
    }
};

template <typename T, int FM, int FN, int WM, int WN, bool TA = false, bool TB = false>
struct TileProduct {
    static constexpr int BM = FM * WM * 16, BN = FN * WN * 16, WAVES = WM * WN, THREADS = WAVES * kWave;
    static constexpr int BUFFER = (BM + BN) * kStepBytes;
    using V = typename Chunk<T>::V;
    using A = Side<T, BM, WAVES, TA>;
    using B = Side<T, BN, WAVES, TB>;
    static constexpr int LOADS = A::LOADS + B::LOADS;

    // acc[i][j]: rows 16 i + 4 (lane / 16) + r of the wavefront's part of A, row
    // 16 j + lane % 16 of its part of B; all `steps` from step0 on
    __device__ static void run(const Operand& oa, const Operand& ob, int64_t m0, int64_t n0, int64_t steps,
                               int64_t step0, unsigned char* __restrict__ buf0, unsigned char* __restrict__ buf1,
                               F4 (&acc)[FM][FN]) {
        if (steps <= 0) return;
        const int lane = lane_id(), w = int(uniform(threadIdx.x / kWave));
        const int fa = w / WN * FM, fb = w % WN * FN;
        constexpr int SECOND = BM * kStepBytes;  // B's part of a buffer
        A sa;
        B sb;
        sa.init(oa, m0, w, lane);
        sb.init(ob, n0, w, lane);
        // (past the last step: the last one again, so that every step waits for as many loads)
        auto fetch = [&](int64_t step, unsigned char* buf) {
            step = step0 + min(step, steps - 1);
            sa.fetch(step, buf, w);
            sb.fetch(step, buf + SECOND, w);
        };
        V a0[FM], b0[FN], a1[FM], b1[FN];
        // products of one half step while the fragments of the next are read, in
        // the first rows' time (the last rows' covers the reads' own)
        auto phase = [&](V(&a)[FM], V(&b)[FN], V(&na)[FM], V(&nb)[FN], const unsigned char* next, int s) {
            const unsigned char *pa = sa.place(next, fa, s), *pb = sb.place(next + SECOND, fb, s);
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = Chunk<T>::mul(a[i], b[j], acc[i][j]);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int q = 2 * i; q < 2 * i + 2; ++q) {
                    if (q < FN)
                        nb[q] = sb.read(pb, fb, q);
                    else if (q < FN + FM)
                        na[q - FN] = sa.read(pa, fa, q - FN);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        static_assert(FN <= FM, "all fragments are read within FM rows");
        auto barrier = [] {
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        constexpr int kNone = 0x0070, kAllButVm = 0x0F70;  // wait for everything; for vector memory only
        auto step = [&](int64_t k, unsigned char* buf, unsigned char* other) {
            phase(a0, b0, a1, b1, buf, 1);
            // this step's fragments are read and the next one's part has landed, for all
            __builtin_amdgcn_s_waitcnt(kNone);
            barrier();
            fetch(k + 2, buf);
            phase(a1, b1, a0, b0, other, 0);
        };
        fetch(0, buf0);
        fetch(1, buf1);
        __builtin_amdgcn_s_waitcnt(kAllButVm | LOADS);
        barrier();
        const unsigned char *pa = sa.place(buf0, fa, 0), *pb = sb.place(buf0 + SECOND, fb, 0);
#pragma unroll
        for (int i = 0; i < FM; ++i) a0[i] = sa.read(pa, fa, i);
#pragma unroll
        for (int j = 0; j < FN; ++j) b0[j] = sb.read(pb, fb, j);
        int64_t k = 0;
        for (; k + 1 < steps; k += 2) {
            step(k, buf0, buf1);
            step(k + 1, buf1, buf0);
        }
        if (k < steps) step(k, buf0, buf1);
        __builtin_amdgcn_s_waitcnt(kNone);  // (no load is under way when the workgroup ends)
    }
};

// A wavefront's part of a tile, of 16-bit elements, through LDS: a lane holds four
// elements of 16 rows' worth of lanes, so stores from the registers would be of 32
// bytes a row; behind LDS they are of whole lines.  out(n, m, pack of eight): n
// and m within the wavefront's part.  The buffers must not be read any more.
template <typename T, int FM, int FN, int WAVES, typename F>
__device__ inline void store_rows(const F4 (&acc)[FM][FN], unsigned char* buf0, unsigned char* buf1, int wave,
                                  float alpha, F out) {
    static_assert(sizeof(T) == 2 && FN % 2 == 0, "");
    constexpr int PITCH = FM * 32 + 16, ROWS = FN * 8;  // (half of the rows at a time)
    const int lane = lane_id();
    unsigned char* own = (wave < WAVES / 2 ? buf0 : buf1) + wave % (WAVES / 2) * ROWS * PITCH;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int j = 0; j < FN / 2; ++j)
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                Vec<T, 4> o;
#pragma unroll
                for (int r = 0; r < 4; ++r) o[r] = T(acc[i][half * (FN / 2) + j][r] * alpha);
                *reinterpret_cast<Vec<T, 4>*>(own + (j * 16 + (lane & 15)) * PITCH + i * 32 + (lane >> 4) * 8) = o;
            }
        constexpr int ACROSS = FM * 2;  // packs of a row
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int t = 0; t < ROWS * ACROSS / kWave; ++t) {
            const int n = (t * kWave + lane) / ACROSS, c = (t * kWave + lane) % ACROSS;
            const Vec<T, 8> v = *reinterpret_cast<const Vec<T, 8>*>(own + n * PITCH + c * 16);
            out(half * ROWS + n, c * 8, v);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

}  // namespace spsyrk
