// Products of tiles on the matrix cores, D[m][n] = sum over k of A(m, k) B(n, k): staged through LDS by loads that write it directly, several
// stages deep.  Shared by the gated transition and the orthogonalisation.
//
// Three kinds of operands: bfloat16; float32 (32x32x2 float32 instructions); float16 pairs, where a value is hi + lo, each rounded to nearest
// (an error of 2^-23 of the value at most, together), and a product hi hi + hi lo + lo hi: what it leaves out, lo lo, is 2^-22 of it at most and of either sign.
// In memory sixteen values of a pair's hi part are followed by their lo parts, so that a row is as contiguous as one of 4-byte values.
// An operand lies in memory with k contiguous, [m][k], or "turned", [k][m]; the reads from LDS turn it back.
//
// v_mfma_f32_32x32x16: A (32 x 16): lane l holds row l % 32, columns 8 (l / 32) .. + 7; B likewise with its columns; D: lane l holds column
// l % 32, register v holds row 8 (v / 4) + 4 (l / 32) + v % 4.  The tiles are given as A := our B, B := our A, so that a lane holds one row m
// and four consecutive n at a time.  v_mfma_f32_32x32x2: lane l holds row l % 32, column l / 32; which k a column stands for is free as long as both
// operands agree, so a lane's sixteen bytes feed four instructions.
#pragma once

#include "ff_common.h"

#include <atomic>

namespace ff {
namespace tile {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short i16x4;
typedef __attribute__((address_space(3))) i16x4* lds_i16x4;

static inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
static inline int64_t round_up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }

__device__ __forceinline__ uint32_t pack2(float a, float b) {      // a -> low half
    bf16x2 t;
    t[0] = (__bf16)a;
    t[1] = (__bf16)b;
    return __builtin_bit_cast(uint32_t, t);
}

// ---- eight neighbours, at any alignment of their elements (gfx950 reads and writes vectors there) ----
typedef __attribute__((__vector_size__(16), aligned(2))) uint32_t Words;
typedef __attribute__((address_space(1))) Words GlobalWords;
__device__ __forceinline__ void load8(const bf16_t* p, float (&v)[8]) {
    const Words w = *(const GlobalWords*)p;
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = __uint_as_float(q & 1 ? w[q / 2] & 0xffff0000u : w[q / 2] << 16);
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
    const Words w[2] = {((const GlobalWords*)p)[0], ((const GlobalWords*)p)[1]};
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = __uint_as_float(w[q / 4][q % 4]);
}
__device__ __forceinline__ void store8(bf16_t* p, const float (&v)[8]) {
    *(GlobalWords*)p = Words{pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])};
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
        ((GlobalWords*)p)[h] = Words{__float_as_uint(v[4 * h]), __float_as_uint(v[4 * h + 1]), __float_as_uint(v[4 * h + 2]), __float_as_uint(v[4 * h + 3])};
}
// n of the eight (a caller's row may end inside them)
template <typename T> __device__ __forceinline__ void load_some(const T* p, int n, float (&v)[8]) {
    if (n >= 8) return load8(p, v);
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = q < n ? to_f32<T>(((const __attribute__((address_space(1))) T*)p)[q]) : 0.f;
}
template <typename T> __device__ __forceinline__ void store_some(T* p, int n, const float (&v)[8]) {
    if (n >= 8) return store8(p, v);
#pragma unroll
    for (int q = 0; q < 8; ++q)
        if (q < n) ((__attribute__((address_space(1))) T*)p)[q] = from_f32<T>(v[q]);
}

// kStep values of k make one round of matrix instructions.
struct Bf16 {
    static constexpr int kSize = 2, kPlanes = 1, kStep = 16;     // bytes of a value in memory
    struct Frag { uint4 u[1]; };
    static __device__ __forceinline__ f32x16 mma(const Frag& b, const Frag& a, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, b.u[0]), __builtin_bit_cast(bf16x8, a.u[0]), c, 0, 0, 0);
    }
};
struct F32 {
    static constexpr int kSize = 4, kPlanes = 1, kStep = 8;
    struct Frag { uint4 u[1]; };
    static __device__ __forceinline__ f32x16 mma(const Frag& b, const Frag& a, f32x16 c) {
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(b.u[0].x), __uint_as_float(a.u[0].x), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(b.u[0].y), __uint_as_float(a.u[0].y), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(b.u[0].z), __uint_as_float(a.u[0].z), c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(b.u[0].w), __uint_as_float(a.u[0].w), c, 0, 0, 0);
    }
};
struct Pair {
    static constexpr int kSize = 4, kPlanes = 2, kStep = 16;
    struct Frag { uint4 u[2]; };
    static __device__ __forceinline__ f32x16 mma(const Frag& b, const Frag& a, f32x16 c) {
        const f16x8 bh = __builtin_bit_cast(f16x8, b.u[0]), bl = __builtin_bit_cast(f16x8, b.u[1]);
        const f16x8 ah = __builtin_bit_cast(f16x8, a.u[0]), al = __builtin_bit_cast(f16x8, a.u[1]);
        c = __builtin_amdgcn_mfma_f32_32x32x16_f16(bl, ah, c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x16_f16(bh, al, c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(bh, ah, c, 0, 0, 0);
    }
};

// All wavefronts of a block have written to LDS what they were to write, and read what they were to read.  (__syncthreads() also waits for stores to memory to be
// acknowledged: one to two microseconds at every turn of a tile's end.)
__device__ __forceinline__ void barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// One operand in memory.  Not turned: row m at p + m pitch, `rows` of them, `bytes` of each may be read (all of its k, padded with zeros to a
// multiple of kStep).  Turned: row k at p + k pitch, `rows` of them (all k, likewise), `bytes` of each (all m).  Bytes are a multiple of 16, p and pitch
// 16-byte aligned.  What lies past an end is read from the last row or the last sixteen bytes: a caller stores no m or n that is not there.
// Blocked (the A side, bfloat16): k in blocks of 32 rows, m in blocks of 32 columns of 2 KiB each, one beside the other: four groups of eight columns, in group g
// sixteen bytes for each of 32 rows, row r at place r ^ 4 g.  A wavefront that has 32 rows stores a kilobyte at a time, a stage is copied as it lies, and the turned
// reads find four rows of four groups in banks of their own.  pitch: bytes from 32 rows to the next; bytes: as much; rows: a multiple of 32.
struct Operand {
    const void* p;
    int64_t pitch;        // bytes
    int64_t rows;
    int32_t bytes;
};

// WK: wavefronts that share a tile's k, round by round; their sums are joined in LDS in a fixed order, and the first ones hold them.
template <class Op_, int BM_, int BN_, int BK_, int STAGES_, int WM_, int WN_, int NA_, int NB_, int TA_, unsigned TB_, int WK_ = 1>
struct Core {
    typedef Op_ Op;
    typedef typename Op::Frag Frag;
    static constexpr int BM = BM_, BN = BN_, BK = BK_, STAGES = STAGES_, WM = WM_, WN = WN_, NA = NA_, NB = NB_;
    static constexpr int TA = TA_;                                 // A is turned (1) or blocked (2)
    static_assert(TA < 2 || (Op_::kStep == 16 && Op_::kPlanes == 1 && BK_ == 32), "blocks of 32 rows");
    static constexpr unsigned TB = TB_;                            // bit b: operand b of the B side is turned
    static constexpr int WK = WK_;
    static constexpr int kWaves = WM * WN * WK, kThreads = 64 * kWaves;
    static constexpr int MT = BM / WM / 32, NT = BN / WN / 32;
    static constexpr int kBytesA = BM * BK * Op::kSize, kBytesB = BN * BK * Op::kSize, kStage = NA * kBytesA + NB * kBytesB;
    static constexpr int kLoads = kStage / 16 / kThreads;          // of a wavefront, for one stage
    static_assert(kBytesA % (16 * kThreads) == 0 && kBytesB % (16 * kThreads) == 0, "the wavefronts count the same loads");
    static_assert(BK % (2 * WK * Op::kStep) == 0 || WK == 1, "the wavefronts of a tile have two rounds of a stage each, or more");
    static_assert(MT >= 1 && NT >= 1 && BK % Op::kStep == 0, "tile");

    // LDS images: rows of W slots of sixteen bytes; a row's slots are exchanged by a rule on the row, so that what one cycle reads (256 bytes) lies in
    // banks of its own: sixteen bytes of sixteen rows, or, turned, of 32 columns' values in four rows (of a pair's, two pieces 64 bytes apart).
    template <int T, int W> static __device__ __forceinline__ int swizzle(int row) {
        if constexpr (!T) return W >= 16 ? row & 15 : W == 8 ? row >> 1 & 7 : W == 4 ? row >> 2 & 3 : 0;
        else if constexpr (W < (Op::kStep == 8 ? 16 : 8)) return 0;      // (tiles of 32: four rows of 64 bytes lie in banks of their own as they are)
        else if constexpr (Op::kStep == 8) return row << 1 & 8;
        else if constexpr (Op::kPlanes == 2) return (row & 1) << 1 | (row & 2) << 2;
        else return W >= 16 ? 4 * (row & 3) : 4 * (row >> 1 & 1);
    }

    // The loads of one operand's part of a stage.  A lane's address is min(x, limit) + y from a uniform base that moves with k: x, which alone can pass an end, and
    // y are the same for all stages.
    template <int T, int R> struct Loader {
        static constexpr int W = (T ? R : BK) * Op::kSize / 16, LR = T ? BK : R, N = LR * W / kThreads;
        uint32_t x[N], y[N];
        __device__ __forceinline__ Loader(const Operand& o, int64_t r0) {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int u = j * kThreads + (int)threadIdx.x, row = u / W, chunk = ((u % W) ^ swizzle<T, W>(row)) * 16;
                if constexpr (T == 2) {
                    x[j] = (uint32_t)u * 16u;
                    y[j] = 0;
                } else if constexpr (T == 1) {
                    const int c = (int)r0 * Op::kSize + chunk, last = o.bytes - 16;
                    x[j] = (uint32_t)row * (uint32_t)o.pitch;
                    y[j] = (uint32_t)(c < last ? c : last);
                } else {
                    const int left = (int)(o.rows - r0 < R ? o.rows - r0 : R) - 1;
                    x[j] = (uint32_t)chunk;
                    y[j] = (uint32_t)(row < left ? row : left) * (uint32_t)o.pitch;
                }
            }
        }
        __device__ __forceinline__ void issue(const Operand& o, int64_t r0, int64_t k0, unsigned lds) const {
            const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
            const char* base = (const char*)o.p + (T == 2 ? k0 / 32 * o.pitch + r0 * 64 : T ? k0 * o.pitch : r0 * o.pitch + k0 * Op::kSize);
            const uint32_t limit = T == 2 ? (uint32_t)(o.bytes - (int)r0 * 64 - 16) : T ? (uint32_t)((o.rows - k0 < LR ? o.rows - k0 : LR) - 1) * (uint32_t)o.pitch : (uint32_t)(o.bytes - 16 - (int)k0 * Op::kSize);
#pragma unroll
            for (int j = 0; j < N; ++j) load16_to_lds(base, (x[j] < limit ? x[j] : limit) + y[j], lds + (j * kThreads + wave * 64) * 16);
        }
    };

    // the lane's piece of plane p of 32 rows (from `row0`) in round s
    template <int T, int R>
    static __device__ __forceinline__ uint4 piece(const unsigned char* image, int p, int row0, int s, int lane) {
        constexpr int W = (T ? R : BK) * Op::kSize / 16;
        const int hf = lane >> 5;
        if constexpr (T == 2) {
            const int i = lane & 15, group = (row0 + (lane & 16)) / 8 + (i >> 1 & 1);
            uint2 h[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int k = 16 * s + 8 * hf + 4 * t + (i >> 2);
                h[t] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)(image + group * 512 + ((k ^ 4 * (group & 3)) << 4) + (i & 1) * 8)));
            }
            return make_uint4(h[0].x, h[0].y, h[1].x, h[1].y);
        } else if constexpr (!T) {
            const int row = row0 + (lane & 31), chunk = 2 * (Op::kPlanes * s + p) + hf;
            return *reinterpret_cast<const uint4*>(image + row * (W * 16) + ((chunk ^ swizzle<false, W>(row)) << 4));
        } else if constexpr (Op::kStep == 16) {
            // of sixteen lanes, lane i asks for four columns 4 (i % 4) .. of row i / 4, and lane l receives column l of the four rows
            const int i = lane & 15, chunk = (row0 + (lane & 16)) / 8 * Op::kPlanes + 2 * p + (i >> 1 & 1);
            uint2 h[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int k = 16 * s + 8 * hf + 4 * t + (i >> 2);
                const unsigned char* q = image + k * (W * 16) + ((chunk ^ swizzle<true, W>(k)) << 4) + (i & 1) * 8;
                h[t] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)q));
            }
            return make_uint4(h[0].x, h[0].y, h[1].x, h[1].y);
        } else {
            uint32_t v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = 8 * s + 4 * hf + j, col = row0 + (lane & 31);
                v[j] = *reinterpret_cast<const uint32_t*>(image + k * (W * 16) + (((col >> 2) ^ swizzle<true, W>(k)) << 4) + (col & 3) * 4);
            }
            return make_uint4(v[0], v[1], v[2], v[3]);
        }
    }
    template <int T, int R>
    static __device__ __forceinline__ Frag frag(const unsigned char* image, int row0, int s, int lane) {
        Frag f;
#pragma unroll
        for (int p = 0; p < Op::kPlanes; ++p) f.u[p] = piece<T, R>(image, p, row0, s, lane);
        return f;
    }

    // the loads of all operands (those of one side that lie alike have pitches and sizes alike too, and differ in their bases only)
    struct Loads {
        Loader<TA, BM> a;
        Loader<(TB & 1) != 0, BN> b;
        Loader<(TB >> (NB - 1) & 1) != 0, BN> last;
        __device__ __forceinline__ Loads(const Operand* oa, const Operand* ob, int64_t m0, int64_t n0) : a(oa[0], m0), b(ob[0], n0), last(ob[NB - 1], n0) {}
        __device__ __forceinline__ void issue(const Operand* oa, const Operand* ob, int64_t m0, int64_t n0, int64_t k0, unsigned lds) const {
#pragma unroll
            for (int i = 0; i < NA; ++i) a.issue(oa[i], m0, k0, lds + i * kBytesA);
#pragma unroll
            for (int i = 0; i < NB - 1; ++i) b.issue(ob[i], n0, k0, lds + NA * kBytesA + i * kBytesB);
            last.issue(ob[NB - 1], n0, k0, lds + NA * kBytesA + (NB - 1) * kBytesB);
        }
    };

    struct Frags {
        Frag a[NA][MT], b[NB][NT];
    };
    template <int B = 0> static __device__ __forceinline__ void read_b(Frags& f, const unsigned char* image, int wn, int s, int lane) {
        if constexpr (B < NB) {
#pragma unroll
            for (int n = 0; n < NT; ++n) f.b[B][n] = frag<(TB >> B & 1) != 0, BN>(image, (wn * NT + n) * 32, s, lane);
            read_b<B + 1>(f, image + kBytesB, wn, s, lane);
        }
    }
    static __device__ __forceinline__ void read(Frags& f, const unsigned char* image, int wm, int wn, int s, int lane) {
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
            for (int m = 0; m < MT; ++m) f.a[i][m] = frag<TA, BM>(image + i * kBytesA, (wm * MT + m) * 32, s, lane);
        read_b(f, image + NA * kBytesA, wn, s, lane);
    }
    static __device__ __forceinline__ void multiply(f32x16 (&acc)[NB][MT][NT], const Frags& f) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n) acc[b][m][n] = Op::mma(f.b[b][n], f.a[NA == 1 || b + 1 < NB ? 0 : 1][m], acc[b][m][n]);      // (a second A side belongs to the last product)
    }

    static __device__ __forceinline__ void clear(f32x16 (&acc)[NB][MT][NT]) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int v = 0; v < 16; ++v) acc[b][m][n][v] = 0.f;
    }

    // adds the products over k = from .. to (multiples of kStep) of the tile at (m0, n0); smem: kLds bytes that every thread is done with
    static __device__ __forceinline__ void run(f32x16 (&acc)[NB][MT][NT], const Operand* a, const Operand* b, int64_t m0, int64_t n0, int64_t from, int64_t to,
                                               unsigned char* smem) {
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
        const int wk = WK == 1 ? 0 : wave / (WM * WN), wm = wave / WN % WM, wn = wave % WN;
        const unsigned lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
        if (from >= to) return;
        constexpr int R = BK / Op::kStep / WK;                   // rounds of a wavefront: WK s + wk
        const int stages = (int)((to - from + BK - 1) / BK), whole = (int)((to - from) / BK);
        const Loads loads(a, b, m0, n0);
#pragma unroll
        for (int i = 0; i < STAGES - 1; ++i)
            if (i < stages) loads.issue(a, b, m0, n0, from + i * BK, lds + i * kStage);
        // Operands of the next round are read while a round's products run, so a stage has to be there one turn early.
        Frags f[2];
        arrive(stages - 1 < STAGES - 2 ? stages - 1 : STAGES - 2);
        read(f[0], smem, wm, wn, wk, lane);
        int buf = 0, t = 0;
        const auto turn = [&](Frags& now, Frags& then) {
            // the next stage is there, and nobody reads the one before any more, in whose place the loads of the one STAGES - 1 ahead go
            if (t + STAGES - 2 < stages) arrive<STAGES - 3>();
            else arrive(stages - t - 2);
            if (t + STAGES - 1 < stages) loads.issue(a, b, m0, n0, from + (int64_t)(t + STAGES - 1) * BK, lds + (buf == 0 ? STAGES - 1 : buf - 1) * kStage);
            const int next = buf + 1 == STAGES ? 0 : buf + 1;
            const unsigned char *image = smem + buf * kStage, *image_next = smem + next * kStage;
#pragma unroll
            for (int s = 0; s < R; ++s) {
                Frags &mine = s & 1 ? then : now, &other = s & 1 ? now : then;
                if (s + 1 < R) read(other, image, wm, wn, WK * (s + 1) + wk, lane);
                else read(other, image_next, wm, wn, wk, lane);            // (of the last stage's successor: what lies there, for no product)
                __builtin_amdgcn_sched_barrier(0);                         // the reads before the products, or they would be waited for right behind them
                multiply(acc, mine);
                __builtin_amdgcn_sched_barrier(0);
            }
            buf = next;
            ++t;
        };
        if constexpr (R & 1) {
            while (t + 1 < whole) {
                turn(f[0], f[1]);
                turn(f[1], f[0]);
            }
            if (t < whole) {
                turn(f[0], f[1]);
                f[0] = f[1];
            }
        } else
            while (t < whole) turn(f[0], f[1]);
        const int rest = (int)((to - from) - (int64_t)whole * BK) / Op::kStep;
        for (int s = wk; s < rest; s += WK) {
            multiply(acc, f[0]);
            if (s + WK < rest) read(f[0], smem + buf * kStage, wm, wn, s + WK, lane);
        }
        barrier();
    }
    // the sums of the wavefronts that share k, in the first of them; smem as for run
    static __device__ __forceinline__ void join(f32x16 (&acc)[NB][MT][NT], unsigned char* smem) {
        if constexpr (WK > 1) {
            static_assert((WK - 1) * WM * WN * NB * MT * NT * 4096 <= STAGES * kStage, "room");
            const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63, wk = wave / (WM * WN), tile = wave % (WM * WN);
            const auto at = [&](int k, int b, int m, int n, int g) { return (float4*)smem + ((((((k - 1) * WM * WN + tile) * NB + b) * MT + m) * NT + n) * 4 + g) * 64 + lane; };
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int g = 0; g < 4; ++g)
                            if (wk > 0) *at(wk, b, m, n, g) = make_float4(acc[b][m][n][4 * g], acc[b][m][n][4 * g + 1], acc[b][m][n][4 * g + 2], acc[b][m][n][4 * g + 3]);
            barrier();
            if (wk == 0)
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int g = 0; g < 4; ++g)
#pragma unroll
                                for (int k = 1; k < WK; ++k) {
                                    const float4 v = *at(k, b, m, n, g);
                                    acc[b][m][n][4 * g] += v.x;
                                    acc[b][m][n][4 * g + 1] += v.y;
                                    acc[b][m][n][4 * g + 2] += v.z;
                                    acc[b][m][n][4 * g + 3] += v.w;
                                }
            barrier();
        }
    }
    // waits until all but the loads of the youngest N stages have arrived, for every wavefront, and for its own reads
    template <int N> static __device__ __forceinline__ void arrive() {
        static_assert(STAGES >= 3 && (STAGES - 2) * kLoads < 64, "the counter");
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N * kLoads) : "memory");
    }
    template <int N = STAGES - 2> static __device__ __forceinline__ void arrive(int n) {          // at the ends, where fewer are under way
        if constexpr (N > 0) {
            if (n >= N) arrive<N>();
            else arrive<N - 1>(n);
        } else
            arrive<0>();
    }

    // Results leave through LDS, where a lane finds eight neighbours of a row: straight from the accumulators a store would reach sixteen bytes of each of 32 rows,
    // and the stores of a tile would take longer than its products.
    // A part of the tile at a time, 32 rows (columns) of each wavefront, so that it takes half the memory.
    static constexpr int kPitch = BN + 4, kPitchTurned = BM + 4;        // floats; sixteen bytes more than a row, so that the rows of one cycle lie in banks of their own
    static constexpr int kOutRows = 128 * WM * kPitch, kOutColumns = 128 * WN * kPitchTurned;
    static constexpr int kOut = kOutRows > kOutColumns ? kOutRows : kOutColumns;
    static constexpr int kLds = STAGES * kStage > kOut ? STAGES * kStage : kOut;

    // body(m, n, v, old): eight results v in row m, columns n .. n + 7, and what fetch(m, n) has read for them.  The reads of four turns are under way together (a
    // load behind another turn's store would wait for it to be issued: they may be the same memory as far as the compiler knows).  smem: kLds bytes that every
    // thread is done with, before and after
    template <typename Fetch, typename F> static __device__ __forceinline__ void rows(const f32x16 (&acc)[MT][NT], int64_t m0, int64_t n0, unsigned char* smem, Fetch fetch, F body) {
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
        float* out = (float*)smem + (wave / WN % WM * 32 + (lane & 31)) * kPitch + (wave % WN * NT) * 32 + 4 * (lane >> 5);
        const bool mine = WK == 1 || wave < WM * WN;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    if (mine) *(float4*)(out + j * 32 + 8 * g) = make_float4(acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]);
            leave<32 * WM, BM / WM, BN, kPitch>(smem, m0 + 32 * i, n0, fetch, body);
        }
    }
    // the same turned: row n, columns m .. m + 7
    template <typename Fetch, typename F> static __device__ __forceinline__ void columns(const f32x16 (&acc)[MT][NT], int64_t m0, int64_t n0, unsigned char* smem, Fetch fetch, F body) {
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
        static_assert(WK == 1, "whole tiles");
        float* out = (float*)smem + (wave % WN * 32 + 4 * (lane >> 5)) * kPitchTurned + (wave / WN * MT) * 32 + (lane & 31);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) out[(8 * (v / 4) + v % 4) * kPitchTurned + i * 32] = acc[i][j][v];
            leave<32 * WN, BN / WN, BM, kPitchTurned>(smem, n0 + 32 * j, m0, fetch, body);
        }
    }
    // R rows of which each 32 lie APART after the 32 before
    template <int R, int APART, int C, int PITCH, typename Fetch, typename F>
    static __device__ __forceinline__ void leave(const unsigned char* smem, int64_t r0, int64_t c0, Fetch fetch, F body) {
        constexpr int kPieces = R * (C / 8), kTurns = (kPieces + kThreads - 1) / kThreads, kGroup = kTurns < 4 ? kTurns : 4;
        static_assert((kPieces % kThreads == 0 || kTurns == 1) && kTurns % kGroup == 0, "turns");
        typedef decltype(fetch(r0, c0)) Old;
#pragma unroll 1
        for (int t0 = 0; t0 < kTurns; t0 += kGroup) {
            Old old[kGroup];
#pragma unroll
            for (int t = 0; t < kGroup; ++t) {
                const int u = (t0 + t) * kThreads + (int)threadIdx.x, r = u / (C / 8);
                if (kPieces < kThreads && u >= kPieces) break;
                old[t] = fetch(r0 + r / 32 * APART + r % 32, c0 + u % (C / 8) * 8);
            }
            if (t0 == 0) barrier();
#pragma unroll
            for (int t = 0; t < kGroup; ++t) {
                const int u = (t0 + t) * kThreads + (int)threadIdx.x, r = u / (C / 8), c = u % (C / 8) * 8;
                if (kPieces < kThreads && u >= kPieces) break;
                const float4 a = *(const float4*)((const float*)smem + r * PITCH + c), b = *(const float4*)((const float*)smem + r * PITCH + c + 4);
                float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
                body(r0 + r / 32 * APART + r % 32, c0 + c, v, old[t]);
            }
        }
        barrier();
    }
    struct Nothing {};
    static __device__ __forceinline__ Nothing none(int64_t, int64_t) { return {}; }
};

// once for each device and each kernel that needs more than 64 KiB (a device beyond 64: at each call)
template <auto KERNEL> static ff_status allow_lds(const char* what) {
    static std::atomic<uint64_t> done{0};
    int device = 0;
    (void)hipGetDevice(&device);
    const uint64_t bit = device < 64 ? (uint64_t)1 << device : 0;
    if (done.load(std::memory_order_relaxed) & bit) return FF_OK;
    const hipError_t error = hipFuncSetAttribute(reinterpret_cast<const void*>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    if (error != hipSuccess) return fail(FF_EHIP, "%s: dynamic LDS limit: %s", what, hipGetErrorString(error));
    done.fetch_or(bit, std::memory_order_relaxed);
    return FF_OK;
}

// Blocks of the same rows of A run one after another on one XCD (block i starts on XCD i % 8), whose L2 then holds them, while B is small enough for all.
struct TilePlace {
    int64_t m;
    int n;
};
__device__ __forceinline__ TilePlace place_of(uint32_t block, uint32_t mtiles, uint32_t ntiles) {
    const uint32_t full = mtiles / 8 * 8 * ntiles;
    if (block >= full) {
        const uint32_t rest = block - full;
        return {(int64_t)(mtiles / 8 * 8 + rest / ntiles), (int)(rest % ntiles)};
    }
    const uint32_t xcd = block & 7u, local = block >> 3;
    return {(int64_t)(local / ntiles * 8 + xcd), (int)(local % ntiles)};
}

}  // namespace tile
}  // namespace ff
