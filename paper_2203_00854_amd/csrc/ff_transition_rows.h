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

    // hidden channels f0 .. f0 + 31; pitches in bytes
    static __device__ __forceinline__ void load(const char* wa, const char* wb, const char* wo, int64_t f0, int pitch_o, unsigned lds) {
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
        const char *a = wa + f0 * (KC * 64), *b = wb + f0 * (KC * 64), *o = wo + f0 * 2;
        constexpr int kPieces = kIn / 1024;                       // wavefront-wide loads of a part (kIn == kOut)
#pragma unroll
        for (int j = 0; j < (3 * kPieces + WAVES - 1) / WAVES; ++j) {
            const int i = j * WAVES + wave;
            if (3 * kPieces % WAVES != 0 && i >= 3 * kPieces) break;
            const int part = kPieces % WAVES == 0 ? j / (kPieces / WAVES) : i / kPieces, u = i % kPieces * 64 + lane;
            if (part < 2) {
                const int row = u / W, chunk = slot_in(row, u % W);            // (an exclusive or is its own inverse)
                load16_to_lds(part ? b : a, (uint32_t)(place(row) * (KC * 64) + chunk * 16), lds + i * 1024);
            } else {
                const int row = u / 4, chunk = slot_out(row, u % 4);
                load16_to_lds(o, (uint32_t)(((row & ~31) + place(row & 31)) * pitch_o + chunk * 16), lds + i * 1024);
            }
        }
    }
    // rows of Wa or Wb as left operand, channels 16 s + 8 half ..
    static __device__ __forceinline__ uint4 in(const unsigned char* part, int s, int lane) {
        const int row = lane & 31;
        return *reinterpret_cast<const uint4*>(part + row * (W * 16) + (slot_in(row, 2 * s + (lane >> 5)) << 4));
    }
    // rows of Wo (32 ct ..), hidden channels 16 half + 8 t ..
    static __device__ __forceinline__ uint4 out(const unsigned char* part, int ct, int t, int lane) {
        const int row = 32 * ct + (lane & 31);
        return *reinterpret_cast<const uint4*>(part + row * 64 + (slot_out(row, 2 * (lane >> 5) + t) << 4));
    }

    // ---- turned: four rows of 64 contiguous bytes a read, their columns in the order of place(); of sixteen lanes, lane i asks for four columns of row i / 4
    static __device__ __forceinline__ uint4 turned(const unsigned char* p0, const unsigned char* p1) {
        const uint2 a = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tile::lds_i16x4)p0));
        const uint2 b = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tile::lds_i16x4)p1));
        return make_uint4(a.x, a.y, b.x, b.y);
    }
    // hidden channels as rows (in the order of place()), channels 16 s + 8 half .. of Wo as k
    static __device__ __forceinline__ uint4 out_turned(const unsigned char* part, int s, int lane) {
        const int i = lane & 15, rb = (lane >> 2 & 4) + (i & 3), chunk = 2 * (rb & 1) + (rb >> 2), row = 32 * (s >> 1) + 16 * (lane >> 5) + 4 * (s & 1) + (i >> 2);
        const unsigned char* p = part + (rb >> 1 & 1) * 8;
        return turned(p + row * 64 + slot_out(row, chunk) * 16, p + (row + 8) * 64 + slot_out(row + 8, chunk) * 16);
    }
    // channels 32 ct .. of Wa or Wb as rows (in the order of place()), hidden channels 16 half + 8 t .. as k
    static __device__ __forceinline__ uint4 in_turned(const unsigned char* part, int ct, int t, int lane) {
        const int i = lane & 15, rb = (lane >> 2 & 4) + (i & 3), chunk = 4 * ct + 2 * (rb & 1) + (rb >> 2), row = 16 * t + 4 * (lane >> 5) + (i >> 2);
        const unsigned char* p = part + (rb >> 1 & 1) * 8;
        return turned(p + row * (W * 16) + slot_in(row, chunk) * 16, p + (row + 8) * (W * 16) + slot_in(row + 8, chunk) * 16);
    }
};

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
