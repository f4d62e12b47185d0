// The gated transition with its rows in registers (bfloat16, up to 256 channels): a wavefront keeps 32 rows of x, and the hidden layer of
// 32 channels at a time lives and dies between two products.
//
// Everything is worked on transposed, so that a result's layout is the next product's operand: a^T [f x rows] = Wa x^T leaves a lane with one row and sixteen
// hidden channels, which is what h^T needs as the right operand of y^T = Wo h^T.  The matrix instruction leaves channels 8 g + 4 half + q (g, q = 0 .. 3) with a half
// of the wavefront; place(r) = 16 (r / 4 % 2) + 4 (r / 8) + r % 4 is the channel that row r of a tile is given, which makes a lane's sixteen values neighbours.
//
// The weights of 32 hidden channels (Wa and Wb [32][c], Wo [c][32]) come through LDS, two stages deep, rows in the order of place().
#pragma once

#include "ff_tile.h"

namespace ff {
namespace rows {

using tile::bf16x8;
using tile::f32x16;
using tile::pack2;

__device__ __forceinline__ int place(int r) { return 16 * (r >> 2 & 1) + 4 * (r >> 3) + (r & 3); }

__device__ __forceinline__ f32x16 mma(uint4 a, uint4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// KC: channels / 32, 1 or even (slots are exchanged within eight or sixteen)
template <int KC, int WAVES> struct Weights {
    static_assert(KC == 1 || KC % 2 == 0, "slots");
    static constexpr int kThreads = 64 * WAVES;
    static constexpr int W = KC * 4;                              // slots of sixteen bytes of a row of Wa
    static constexpr int kIn = 32 * W * 16, kOut = KC * 32 * 64;  // bytes of Wa's (Wb's) part of a stage, of Wo's
    static constexpr int kStage = 2 * kIn + kOut;
    static constexpr int kLds = 2 * kStage;

    // the slot that holds piece `chunk` of a row: the sixteen rows that one cycle reads, and four rows of 64 bytes that a turned read takes, lie in banks of their own
    static __device__ __forceinline__ int slot_in(int row, int chunk) {
        if constexpr (W % 16 == 0) return chunk ^ ((row & 3) << 2 | (row >> 2 & 3));
        if constexpr (W % 8 == 0) return chunk ^ ((row >> 1 & 1) << 2 | (row >> 2 & 3));
        return chunk ^ (row >> 2 & 3);
    }
    static __device__ __forceinline__ int slot_out(int row, int chunk) { return chunk ^ (row >> 2 & 3); }

    // The loads of a stage.  Wa's and Wb's (Wo's) part is kPieces wavefront-wide loads, dealt to the wavefronts in turn; a lane's addresses relative to the stage's start
    // are the same for all stages, and with rows of 256 bytes those of a wavefront's loads differ by whole rows alone.
    static constexpr int kPieces = kIn / 1024, kEach = (kPieces + WAVES - 1) / WAVES, kKept = W == 16 ? 1 : kEach;
    struct Loads {
        uint32_t in[kKept], out[kKept];
        __device__ __forceinline__ explicit Loads(int pitch_o) {
            const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
#pragma unroll
            for (int j = 0; j < kKept; ++j) {
                const int u = (j * WAVES + wave) * 64 + lane, r = u / W, o = u / 4;
                in[j] = (uint32_t)(place(r) * (KC * 64) + slot_in(r, u % W) * 16);           // (an exclusive or is its own inverse)
                out[j] = (uint32_t)(((o & ~31) + place(o & 31)) * pitch_o + slot_out(o, u % 4) * 16);
            }
        }
        // hidden channels f0 .. f0 + 31; pitch in bytes
        __device__ __forceinline__ void issue(const char* wa, const char* wb, const char* wo, int64_t f0, int pitch_o, unsigned lds) const {
            const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
            const char *a = wa + f0 * (KC * 64), *b = wb + f0 * (KC * 64), *o = wo + f0 * 2;
            static_assert(W != 16 || WAVES == 4, "four wavefronts' loads are sixteen rows of Wa: place() of the next sixteen is eight further; of Wo 64 rows");
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                if (kPieces % WAVES != 0 && j * WAVES + wave >= kPieces) break;
                const int kept = j < kKept ? j : 0, more = j - kept;
                const unsigned to = lds + (j * WAVES + wave) * 1024;
                load16_to_lds(a + more * 8 * (KC * 64), in[kept], to);
                load16_to_lds(b + more * 8 * (KC * 64), in[kept], to + kIn);
                load16_to_lds(o + (int64_t)more * 64 * pitch_o, out[kept], to + 2 * kIn);
            }
        }
    };

    // ---- operands: a lane's address is one of four numbers below, an exclusive or with what a step changes of the slot, and a constant
    static constexpr int kMask = W % 16 == 0 ? 15 : W % 8 == 0 ? 7 : 3;           // of a slot, what is exchanged
    struct Lane {
        int in, out, in_turned, out_turned;
        __device__ __forceinline__ explicit Lane(int lane) {
            const int r = lane & 31, hf = lane >> 5, i = lane & 15, rb = (lane >> 2 & 4) + (i & 3), chunk = 2 * (rb & 1) + (rb >> 2), half = (rb >> 1 & 1) * 8;
            in = r * (W * 16) + slot_in(r, hf) * 16;
            out = r * 64 + slot_out(r, 2 * hf) * 16;
            in_turned = (4 * hf + (i >> 2)) * (W * 16) + slot_in(4 * hf + (i >> 2), chunk) * 16 + half;
            out_turned = (16 * hf + (i >> 2)) * 64 + chunk * 16 + half;
        }
    };
    // rows of Wa or Wb as left operand, channels 16 s + 8 half ..
    static __device__ __forceinline__ uint4 in(const unsigned char* part, const Lane& l, int s) {
        return *reinterpret_cast<const uint4*>(part + (l.in ^ (2 * s & kMask) << 4) + (2 * s & ~kMask) * 16);
    }
    // rows of Wo (32 ct ..), hidden channels 16 half + 8 t ..
    static __device__ __forceinline__ uint4 out(const unsigned char* part, const Lane& l, int ct, int t) {
        return *reinterpret_cast<const uint4*>(part + (l.out ^ t << 4) + ct * 2048);
    }
    // Turned: four rows of 64 contiguous bytes a read, their columns in the order of place(); of sixteen lanes, lane i asks for four columns of row i / 4.
    static __device__ __forceinline__ uint4 turned(const unsigned char* p0, const unsigned char* p1) {
        const uint2 a = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tile::lds_i16x4)p0));
        const uint2 b = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tile::lds_i16x4)p1));
        return make_uint4(a.x, a.y, b.x, b.y);
    }
    // hidden channels as rows (in the order of place()), channels 16 s + 8 half .. of Wo as k: rows 32 (s / 2) + 16 half + 4 (s % 2) .., and eight further
    static __device__ __forceinline__ uint4 out_turned(const unsigned char* part, const Lane& l, int s) {
        const unsigned char* p = part + (32 * (s >> 1) + 4 * (s & 1)) * 64;
        return turned(p + (l.out_turned ^ (s & 1) << 4), p + (l.out_turned ^ (2 + (s & 1)) << 4) + 512);
    }
    // channels 32 ct .. of Wa or Wb as rows (in the order of place()), hidden channels 16 half + 8 t .. as k: rows 16 t + 4 half .., and eight further
    static __device__ __forceinline__ uint4 in_turned(const unsigned char* part, const Lane& l, int ct, int t) {
        const unsigned char* p = part + t * 16 * (W * 16) + (4 * ct & ~kMask) * 16;
        return turned(p + (l.in_turned ^ (4 * ct & kMask) << 4), p + (l.in_turned ^ ((4 * ct & kMask) ^ 2) << 4) + 8 * (W * 16));
    }
};

// N steps whose operands are read AHEAD steps before they are used: left to itself the compiler reads each right in front of its product and waits
template <int N, int AHEAD, typename Read, typename Use> __device__ __forceinline__ void ahead(Read read, Use use) {
    decltype(read(0)) f[AHEAD + 1];
#pragma unroll
    for (int n = 0; n < AHEAD && n < N; ++n) f[n] = read(n);
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (n + AHEAD < N) f[(n + AHEAD) % (AHEAD + 1)] = read(n + AHEAD);
        __builtin_amdgcn_sched_barrier(0);
        use(n, f[n % (AHEAD + 1)]);
        __builtin_amdgcn_sched_barrier(0);
    }
}
struct One { uint4 a; };
struct Two { uint4 a, b; };
struct Three { uint4 a, b, c; };

// a row's sixteen channels 16 s + 8 half .. of x as right operands, zeros past the end and in rows that are none
template <int KC> __device__ __forceinline__ void load_row(uint4 (&v)[2 * KC], const bf16_t* x, int64_t row, bool live, int c, bool whole, int lane) {
    const bf16_t* p = x + row * c + 8 * (lane >> 5);
#pragma unroll
    for (int s = 0; s < 2 * KC; ++s) {
        v[s] = make_uint4(0, 0, 0, 0);
        if (!live) continue;
        if (whole) v[s] = *reinterpret_cast<const uint4*>(p + 16 * s);
        else {
            alignas(16) bf16_t e[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) e[q] = 16 * s + 8 * (lane >> 5) + q < c ? p[16 * s + q] : (bf16_t)0;
            v[s] = *reinterpret_cast<const uint4*>(e);
        }
    }
}

// A wavefront's 32 x 32 values (sixteen neighbours of a row a lane) as a block of tile::Operand's third kind
__device__ __forceinline__ void store_block(char* p, const uint32_t (&w)[8], int lane) {
    const int r = lane & 31, g = lane >> 5 << 1;
    *(uint4*)(p + g * 512 + (r ^ 4 * g) * 16) = make_uint4(w[0], w[1], w[2], w[3]);
    *(uint4*)(p + (g + 1) * 512 + (r ^ 4 * (g + 1)) * 16) = make_uint4(w[4], w[5], w[6], w[7]);
}
// sixteen neighbours, as bfloat16, from p on (sixteen-byte aligned)
__device__ __forceinline__ void store16(bf16_t* p, const uint32_t (&w)[8]) {
    *(uint4*)p = make_uint4(w[0], w[1], w[2], w[3]);
    *(uint4*)(p + 8) = make_uint4(w[4], w[5], w[6], w[7]);
}

}  // namespace rows
}  // namespace ff
