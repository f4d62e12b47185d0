// The gated transition, y = (act(x Wa^T) * (x Wb^T)) Wo^T, and its gradients.
#include "ff_transition_rows.h"

#include <algorithm>

namespace ff {

using tile::align256;
using tile::Bf16;
using tile::Core;
using tile::f32x16;
using tile::F32;
using tile::Operand;
using tile::round_up;

namespace {

constexpr int kPad = 16;                       // rows and columns of the products' inner dimensions are padded to this with zeros
constexpr int64_t kMostRows = 1 << 30;          // of a launch: two threads a row, 2^32 threads a grid
constexpr int64_t kHiddenBytes = 512 << 20;    // of one hidden tensor (of tokens, where they are wider) of a chunk of rows: more rows keep the units busier (701 x 701 x 128, f 512: 979 us in chunks of 64 MiB, 881 in one)

template <typename T> struct OpOf;
template <> struct OpOf<float> { typedef F32 type; };
template <> struct OpOf<bf16_t> { typedef Bf16 type; };

// ---- activations -------------------------------------------------------------------------
// In float32 with the library's functions; for bfloat16 results the sigmoid by the machine's exponential and reciprocal: off by (1.5 |a| + 5) 2^-24 of it (log2 e and the product with
// it are rounded, which the exponential multiplies by |a|; a step for it, half a one for the sum, a step for the reciprocal), against the results' 2^-8
template <bool FAST> __device__ __forceinline__ float sigmoid_of(float a) {
    if constexpr (FAST) return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * a));
    return 1.f / (1.f + expf(-a));
}
template <int ACT, bool FAST> __device__ __forceinline__ float gate_of(float a) {
    if constexpr (ACT == FF_GELU) return a * (0.5f * erfcf(-0.70710678118654752f * a));
    const float s = sigmoid_of<FAST>(a);
    return ACT == FF_SIGMOID ? s : a * s;
}
template <int ACT, bool FAST> __device__ __forceinline__ float gate_of(float a, float& slope) {
    if constexpr (ACT == FF_GELU) {
        const float phi = 0.5f * erfcf(-0.70710678118654752f * a);
        slope = phi + a * (0.39894228040143268f * expf(-0.5f * a * a));
        return a * phi;
    }
    const float s = sigmoid_of<FAST>(a);
    if constexpr (ACT == FF_SIGMOID) {
        slope = s * (1.f - s);
        return s;
    }
    slope = s * (1.f + a * (1.f - s));
    return a * s;
}

// ---- packing -------------------------------------------------------------------------------
// Copies whose rows and columns are padded with zeros, masked rows zero: what is not aligned to sixteen bytes, or has odd sizes, or rows whose values
// must not reach sums over rows.  A thread writes sixteen bytes.
struct PackJob {
    const void* src;
    void* dst;
    const float* mask;
    int64_t rows, rows_out;
    int32_t cols, cols_out;
    uint32_t blocks;
};
struct PackArgs { PackJob job[5]; };
template <typename T> __global__ __launch_bounds__(256) void k_tr_pack(PackArgs a) {
    constexpr int V = 16 / sizeof(T);
    uint32_t block = blockIdx.x;
    int j = 0;
    while (j < 4 && block >= a.job[j].blocks) block -= a.job[j++].blocks;
    const PackJob& p = a.job[j];
    const int64_t i = (int64_t)block * 256 + threadIdx.x;
    const int per = p.cols_out / V;
    const int64_t r = i / per;
    const int c = (int)(i % per) * V;
    if (r >= p.rows_out) return;
    const bool live = r < p.rows && !(p.mask && p.mask[r] == 0.f);
    const T* src = (const T*)p.src + r * p.cols;
    alignas(16) T v[V];
#pragma unroll
    for (int q = 0; q < V; ++q) v[q] = live && c + q < p.cols ? src[c + q] : T(0);
    *(uint4*)((T*)p.dst + r * p.cols_out + c) = *(const uint4*)v;
}

struct Eight { float v[8]; };
// what is past the end of a row, or in a row that is none, is held as zero
__device__ __forceinline__ void keep(float (&v)[8], int64_t n) {
    if (n >= 8) return;
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = q < n ? v[q] : 0.f;
}

// ---- hidden layer --------------------------------------------------------------------------
struct HiddenArgs {
    Operand x, w[2];
    void* h;
    int64_t rows, rows_out;       // of this chunk; of h
    int32_t f, k, pitch;          // hidden channels; channels of x, padded; values of a row of h
    uint32_t mtiles, ntiles;
};
// Both projections share the tile of x; their product with the activation leaves alone.  Channels and rows past the end are zeros.  Bound by the matrix
// instructions: float32 9920 x 173 with 692 hidden channels 61 us, the matrix units 0.66 busy (eleven stages of 16 k: a third is the way in and out of a tile); in
// bfloat16 with tiles of 256 x 128, 16384 x 512 with 2048, forward 134 us, 770 TFLOP/s of both kernels.
template <class C, typename T, int ACT> __global__ __launch_bounds__(C::kThreads, C::kThreads == 512 ? 2 : C::BM == 64 ? 4 : C::BM == 32 ? 1 : 2) void k_tr_hidden(HiddenArgs a) {
    extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
    const tile::TilePlace at = tile::place_of(blockIdx.x, a.mtiles, a.ntiles);
    f32x16 acc[2][C::MT][C::NT];
    C::clear(acc);
    C::run(acc, &a.x, a.w, at.m * C::BM, (int64_t)at.n * C::BN, 0, a.k, smem);
    C::join(acc, smem);
#pragma unroll
    for (int i = 0; i < C::MT; ++i)
#pragma unroll
        for (int j = 0; j < C::NT; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[0][i][j][v] = gate_of<ACT, sizeof(T) == 2>(acc[0][i][j][v]) * acc[1][i][j][v];
    C::rows(acc[0], at.m * C::BM, (int64_t)at.n * C::BN, smem, C::none, [&](int64_t m, int64_t n, float (&v)[8], typename C::Nothing) {
        if (m >= a.rows_out || n >= a.pitch) return;
        keep(v, m < a.rows ? a.f - n : 0);
        tile::store8((T*)a.h + m * a.pitch + n, v);
    });
}

// ---- output --------------------------------------------------------------------------------
struct OutArgs {
    Operand a[2], b[2];
    int32_t parts;                // products that are added up
    int32_t k, cols;
    int64_t rows;
    const void* residual;
    const float* mask;
    void* out;
    uint32_t mtiles, ntiles;
};
// out = (residual +) sum of the products; a masked row's sum counts as zero, whatever it is.  Bound as above: the same float32 case 33 us.
template <class C, typename T> __global__ __launch_bounds__(C::kThreads, C::kThreads == 512 ? 2 : C::BM == 64 ? 4 : C::BM == 32 ? 1 : 2) void k_tr_out(OutArgs a) {
    extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
    const tile::TilePlace at = tile::place_of(blockIdx.x, a.mtiles, a.ntiles);
    f32x16 acc[1][C::MT][C::NT];
    C::clear(acc);
    for (int p = 0; p < a.parts; ++p) C::run(acc, a.a + p, a.b + p, at.m * C::BM, (int64_t)at.n * C::BN, 0, a.k, smem);
    C::join(acc, smem);
    const auto fetch = [&](int64_t m, int64_t n) {
        Eight e;
#pragma unroll
        for (int q = 0; q < 8; ++q) e.v[q] = 0.f;
        if (a.residual && m < a.rows && n < a.cols) tile::load_some((const T*)a.residual + m * a.cols + n, a.cols - (int)n, e.v);
        return e;
    };
    C::rows(acc[0], at.m * C::BM, (int64_t)at.n * C::BN, smem, fetch, [&](int64_t m, int64_t n, float (&v)[8], Eight r) {
        if (m >= a.rows || n >= a.cols) return;
        const bool live = !(a.mask && a.mask[m] == 0.f);
#pragma unroll
        for (int q = 0; q < 8; ++q) r.v[q] += live ? v[q] : 0.f;
        tile::store_some((T*)a.out + m * a.cols + n, a.cols - (int)n, r.v);
    });
}

// ---- the whole forward pass with rows in registers -------------------------------------------
// The hidden layer would be 4 times the bytes of x (f = 4 c, and twice that, written and read): it stays in registers.  A block has 128 rows, four wavefronts, and streams the weights, which
// L2 holds, through LDS; 32 hidden channels are 3 c / 16 matrix instructions a wavefront between two barriers, three blocks a unit at up to 128 channels fill each other's
// gaps.  Bound by the matrix units and the exponentials between them: 2048 x 2048 x 128 with 512 hidden channels and residual 1.73 ms, 950 TFLOP/s (through memory 4.9 ms), of 3.2 GB that
// take 0.63; 128 x 256 x 256 with 1024 60 us, 853 TFLOP/s: 256 blocks, one a unit, whose last turns nothing fills.
struct RowsArgs {
    const bf16_t *x, *residual;
    const char *w_a, *w_b, *w_o;
    const float* mask;
    bf16_t* y;
    int64_t rows;
    int32_t f, c, pitch_o;        // hidden channels, padded to 32; channels; bytes of a row of Wo
    int32_t whole;                // rows of x (residual, y) are 32 KC channels and 16-byte aligned
};
template <int KC, int ACT> __global__ __launch_bounds__(256, KC <= 4 ? 3 : KC <= 6 ? 2 : 1) void k_tr_rows(RowsArgs a) {
    typedef rows::Weights<KC, 4> W;
    extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63, hf = lane >> 5;
    const unsigned lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    const typename W::Loads loads(a.pitch_o);
    loads.issue(a.w_a, a.w_b, a.w_o, 0, a.pitch_o, lds);
    const int64_t row = (int64_t)blockIdx.x * 128 + wave * 32 + (lane & 31);
    const typename W::Lane at(lane);
    const bool there = row < a.rows, live = there && !(a.mask && a.mask[row] == 0.f);
    uint4 x[2 * KC];
    rows::load_row<KC>(x, a.x, row, live, a.c, a.whole, lane);
    f32x16 y[KC];
#pragma unroll
    for (int i = 0; i < KC; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) y[i][v] = 0.f;
    int buf = 0;
    for (int f0 = 0; f0 < a.f; f0 += 32, buf ^= 1) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();                                       // the stage is there, and nobody reads the other one any more
        if (f0 + 32 < a.f) loads.issue(a.w_a, a.w_b, a.w_o, f0 + 32, a.pitch_o, lds + (buf ^ 1) * W::kStage);
        const unsigned char* part = smem + buf * W::kStage;
        f32x16 p, q;
#pragma unroll
        for (int v = 0; v < 16; ++v) p[v] = q[v] = 0.f;
        rows::ahead<2 * KC, KC <= 4 ? 2 : 3>([&](int s) { return rows::Two{W::in(part, at, s), W::in(part + W::kIn, at, s)}; },
                                [&](int s, const rows::Two& w) {
                                    p = rows::mma(w.a, x[s], p);
                                    q = rows::mma(w.b, x[s], q);
                                });
        uint32_t h[8];
#pragma unroll
        for (int v = 0; v < 8; ++v) h[v] = tile::pack2(gate_of<ACT, true>(p[2 * v]) * q[2 * v], gate_of<ACT, true>(p[2 * v + 1]) * q[2 * v + 1]);
        rows::ahead<2 * KC, KC <= 4 ? 4 : 5>([&](int n) { return rows::One{W::out(part + 2 * W::kIn, at, n % KC, n / KC)}; },
                                [&](int n, const rows::One& w) {
                                    const int t = n / KC * 4;
                                    y[n % KC] = rows::mma(w.a, make_uint4(h[t], h[t + 1], h[t + 2], h[t + 3]), y[n % KC]);
                                });
    }
    if (!there) return;
    const int64_t to = row * a.c + 16 * hf;
#pragma unroll
    for (int i = 0; i < KC; ++i) {
        if (a.whole) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float v[8];
                uint4 r = make_uint4(0, 0, 0, 0);
                if (a.residual) r = *reinterpret_cast<const uint4*>(a.residual + to + 32 * i + 8 * u);
                const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = (live ? y[i][8 * u + e] : 0.f) + __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
                *reinterpret_cast<uint4*>(a.y + to + 32 * i + 8 * u) = make_uint4(tile::pack2(v[0], v[1]), tile::pack2(v[2], v[3]), tile::pack2(v[4], v[5]), tile::pack2(v[6], v[7]));
            }
        } else
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (32 * i + 16 * hf + e < a.c)
                    a.y[to + 32 * i + e] = f32_to_bf16((live ? y[i][e] : 0.f) + (a.residual ? bf16_to_f32(a.residual[to + 32 * i + e]) : 0.f));
    }
}

// ---- gradients of the hidden layer -----------------------------------------------------------
struct GradArgs {
    Operand a[2], b[3];           // x, dy; Wa, Wb, Wo
    void *da, *db, *h;
    int64_t rows, rows_out;
    int32_t f, k, pitch;
    uint32_t mtiles, ntiles;
};
// a, b and dh = dy Wo of a tile in one loop over the channels; da = dh b act'(a), db = dh act(a) and h, rounded to the tensors' type, are what the
// products with the weights and with x and dy read.  Three accumulators a tile: 18000 x 173 with 692 hidden channels in float32 161 us, the matrix units 0.66 busy.
template <class C, typename T, int ACT> __global__ __launch_bounds__(C::kThreads, C::kThreads == 512 || C::BM == 64 ? 2 : C::BM == 32 ? 1 : 2) void k_tr_grad(GradArgs a) {
    extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
    const tile::TilePlace at = tile::place_of(blockIdx.x, a.mtiles, a.ntiles);
    f32x16 acc[3][C::MT][C::NT];
    C::clear(acc);
    C::run(acc, a.a, a.b, at.m * C::BM, (int64_t)at.n * C::BN, 0, a.k, smem);
    C::join(acc, smem);
#pragma unroll
    for (int i = 0; i < C::MT; ++i)
#pragma unroll
        for (int j = 0; j < C::NT; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                float slope;
                const float gate = gate_of<ACT, sizeof(T) == 2>(acc[0][i][j][v], slope), b = acc[1][i][j][v], dh = acc[2][i][j][v];
                acc[0][i][j][v] = dh * b * slope;
                acc[1][i][j][v] = dh * gate;
                acc[2][i][j][v] = gate * b;
            }
    void* const out[3] = {a.da, a.db, a.h};
#pragma unroll
    for (int t = 0; t < 3; ++t)
        C::rows(acc[t], at.m * C::BM, (int64_t)at.n * C::BN, smem, C::none, [&](int64_t m, int64_t n, float (&v)[8], typename C::Nothing) {
            if (m >= a.rows_out || n >= a.pitch) return;
            keep(v, m < a.rows ? a.f - n : 0);
            tile::store8((T*)out[t] + m * a.pitch + n, v);
        });
}

// The same with rows in registers (bfloat16, up to 256 channels), and dx with them: a^T, b^T and dh^T = Wo^T dy^T of 32 hidden channels leave a lane with sixteen neighbours
// of each, from which da, db and h are stored and dx^T += Wa^T da^T + Wb^T db^T goes on.  The weights' other sides are read turned from the same stage.
// Its stores, 6 f bytes a row, and two wavefronts a SIMD, which the registers of x, dy and dx allow: 701 x 701 x 128 with 512 hidden channels 585 us, 2.1 GB at 3.6 TB/s of the 5.0 that a
// copy reaches and the matrix units 0.36 busy, so neither is full.  Without the stores the weights' gradients would need a, b and dh once more, 6 of 16 parts of the work.
struct GradRowsArgs {
    const bf16_t *x, *dy;
    const char *w_a, *w_b, *w_o;
    const float* mask;
    char *da, *db, *h;            // blocked, 64 f bytes for each 32 rows
    bf16_t* dx;
    bf16_t *x_copy, *dy_copy;     // NULL, or [rows_out][32 KC]: rows and channels that are none are zeros there
    int64_t rows, rows_out;       // rows_out: a multiple of 32
    int32_t f, c, pitch_o;        // as in RowsArgs
    int32_t whole;
};
template <int KC, int ACT> __global__ __launch_bounds__(256, KC <= 4 ? 2 : 1) void k_tr_grad_rows(GradRowsArgs a) {
    typedef rows::Weights<KC, 4> W;
    extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63, hf = lane >> 5;
    const unsigned lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    const typename W::Loads loads(a.pitch_o);
    loads.issue(a.w_a, a.w_b, a.w_o, 0, a.pitch_o, lds);
    const int64_t row = (int64_t)blockIdx.x * 128 + wave * 32 + (lane & 31);
    const bool live = row < a.rows && !(a.mask && a.mask[row] == 0.f);
    const typename W::Lane place(lane);
    const bool held = (int64_t)blockIdx.x * 128 + wave * 32 < a.rows_out;                // the wavefront's 32 rows have a place in da, db and h
    uint4 x[2 * KC], dy[2 * KC];
    rows::load_row<KC>(x, a.x, row, live, a.c, a.whole, lane);
    rows::load_row<KC>(dy, a.dy, row, live, a.c, a.whole, lane);
    if (a.x_copy && held) {
        const int64_t at = row * (32 * KC) + 8 * hf;
#pragma unroll
        for (int s = 0; s < 2 * KC; ++s) {
            *(uint4*)(a.x_copy + at + 16 * s) = x[s];
            *(uint4*)(a.dy_copy + at + 16 * s) = dy[s];
        }
    }
    f32x16 dx[KC];
#pragma unroll
    for (int i = 0; i < KC; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) dx[i][v] = 0.f;
    int buf = 0;
    for (int f0 = 0; f0 < a.f; f0 += 32, buf ^= 1) {
        // The stage is there, and nobody reads the other one any more.  Behind its loads a wavefront has issued the six stores of the turn before, which are not waited for
        // (operations of this kind end in their order; a wavefront without a row that is held has issued none).
        if (f0 > 0 && held) asm volatile("s_waitcnt vmcnt(6)" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        tile::barrier();
        if (f0 + 32 < a.f) loads.issue(a.w_a, a.w_b, a.w_o, f0 + 32, a.pitch_o, lds + (buf ^ 1) * W::kStage);
        const unsigned char* part = smem + buf * W::kStage;
        f32x16 p, q, r;
#pragma unroll
        for (int v = 0; v < 16; ++v) p[v] = q[v] = r[v] = 0.f;
        rows::ahead<2 * KC, 2>([&](int s) { return rows::Three{W::in(part, place, s), W::in(part + W::kIn, place, s), W::out_turned(part + 2 * W::kIn, place, s)}; },
                               [&](int s, const rows::Three& w) {
                                   p = rows::mma(w.a, x[s], p);
                                   q = rows::mma(w.b, x[s], q);
                                   r = rows::mma(w.c, dy[s], r);
                               });
        uint32_t da[8], db[8], h[8];
#pragma unroll
        for (int v = 0; v < 8; ++v) {
            float w[3][2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float slope;
                const float gate = gate_of<ACT, true>(p[2 * v + e], slope);
                w[0][e] = r[2 * v + e] * q[2 * v + e] * slope;
                w[1][e] = r[2 * v + e] * gate;
                w[2][e] = gate * q[2 * v + e];
            }
            da[v] = tile::pack2(w[0][0], w[0][1]);
            db[v] = tile::pack2(w[1][0], w[1][1]);
            h[v] = tile::pack2(w[2][0], w[2][1]);
        }
        if (held) {
            const int64_t at = (row >> 5) * a.f * 64 + f0 * 64;
            rows::store_block(a.da + at, da, lane);
            rows::store_block(a.db + at, db, lane);
            rows::store_block(a.h + at, h, lane);
        }
        // (channels change faster than the four parts of k: an accumulator rests between two of its own)
        rows::ahead<4 * KC, 4>([&](int n) { return rows::One{W::in_turned(n / KC & 1 ? part + W::kIn : part, place, n % KC, n / KC >> 1)}; },
                               [&](int n, const rows::One& w) {
                                   const int t = (n / KC >> 1) * 4;
                                   dx[n % KC] = rows::mma(w.a, n / KC & 1 ? make_uint4(db[t], db[t + 1], db[t + 2], db[t + 3]) : make_uint4(da[t], da[t + 1], da[t + 2], da[t + 3]), dx[n % KC]);
                               });
    }
    if (row >= a.rows) return;
    const int64_t at = row * a.c + 16 * hf;
#pragma unroll
    for (int i = 0; i < KC; ++i) {
        if (a.whole) {
            uint32_t w[8];
#pragma unroll
            for (int v = 0; v < 8; ++v) w[v] = tile::pack2(dx[i][2 * v], dx[i][2 * v + 1]);
            rows::store16(a.dx + at + 32 * i, w);
        } else
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (32 * i + 16 * hf + e < a.c) a.dx[at + 32 * i + e] = f32_to_bf16(dx[i][e]);
    }
}

// ---- gradients of the weights ------------------------------------------------------------------
struct WeightArgs {
    Operand a[3], b[3];           // da, db, h; x, x, dy
    float* partial;               // [splits][3][fp][cp]; the last is that of Wo turned
    int64_t rows;                 // padded to kPad
    int64_t per_split;            // rows of a split
    int32_t fp, cp;
    uint32_t ftiles, ctiles;
    int32_t add;                  // to what an earlier chunk left
};
// Sums over rows: both operands lie with the rows as k.  The rows are split over blocks, whose sums are joined in a fixed order.  Where rows are many da, db and h
// are read once by tiles of 256 x 128: 701 x 701 x 128 with 512 hidden channels 407 us for 1.7 GB, 4.3 TB/s, the matrix units 0.27 busy; 128 x 256 x 256 with 1024 67 us and 16 for the join of 20 parts, 61 MB of
// sums that the 240 blocks' accumulators are.  Float32, 18000 x 173: 163 us, the matrix units 0.71 busy.
template <class C> __global__ __launch_bounds__(C::kThreads) void k_tr_weights(WeightArgs a) {
    extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
    // each XCD (block i starts on XCD i % 8) has a run of neighbouring items: tiles of the same rows, which its L2 then holds
    // (18000 x 173 in float32 196 MB from HBM instead of 675, 128 x 256 x 256 233 instead of 393: the latter's whole backward pass 198 -> 192 us, 701 x 701 x 128 887 -> 873)
    const uint32_t tiles = a.ftiles * a.ctiles, block = blockIdx.y * gridDim.x + blockIdx.x, all = gridDim.x * gridDim.y, xcd = block & 7u;
    const uint32_t item = xcd * (all >> 3) + (xcd < (all & 7u) ? xcd : all & 7u) + (block >> 3), split = item / gridDim.x, rest = item % gridDim.x, which = rest / tiles, t = rest % tiles;
    const int64_t m0 = (int64_t)(t / a.ctiles) * C::BM, n0 = (int64_t)(t % a.ctiles) * C::BN;
    const int64_t from = split * a.per_split, to = from + a.per_split < a.rows ? from + a.per_split : a.rows;
    f32x16 acc[1][C::MT][C::NT];
    C::clear(acc);
    C::run(acc, a.a + which, a.b + which, m0, n0, from, to, smem);
    float* out = a.partial + ((int64_t)split * 3 + which) * a.fp * a.cp;
    const int32_t rows = a.fp, cols = a.cp;
    const auto fetch = [&](int64_t m, int64_t n) {
        Eight e;
#pragma unroll
        for (int q = 0; q < 8; ++q) e.v[q] = 0.f;
        if (a.add && m < rows && n < cols) tile::load8(out + m * cols + n, e.v);
        return e;
    };
    C::rows(acc[0], m0, n0, smem, fetch, [&](int64_t m, int64_t n, float (&v)[8], const Eight& was) {
        if (m >= rows || n >= cols) return;
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] += was.v[q];
        tile::store8(out + m * cols + n, v);
    });
}

struct JoinArgs {
    const float* partial;
    void* dw[3];
    int32_t f, c, fp, cp, splits, accumulate;
};
// The gradients of a 32 x 32 part of the weights, their parts added up in order; that of Wo is turned in LDS.
template <typename G> __global__ __launch_bounds__(256) void k_tr_join(JoinArgs a) {
    __shared__ float turned[32][33];
    const int which = blockIdx.z;
    const int64_t size = (int64_t)a.fp * a.cp;
    const int f0 = blockIdx.y * 32, c0 = blockIdx.x * 32, lane = threadIdx.x & 31;
    G* const out = (G*)a.dw[which];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int f = f0 + ((int)threadIdx.x >> 5) + 8 * k, c = c0 + lane;
        const bool there = f < a.f && c < a.c;
        float sum = 0.f;
        const float* p = a.partial + which * size + (int64_t)f * a.cp + c;
        if (there)
#pragma unroll 4
            for (int s = 0; s < a.splits; ++s) sum += p[s * 3 * size];
        if (which == 2) turned[(threadIdx.x >> 5) + 8 * k][lane] = sum;
        else if (there) {
            G* o = out + (int64_t)f * a.c + c;
            *o = from_f32<G>(a.accumulate ? to_f32<G>(*o) + sum : sum);
        }
    }
    if (which != 2) return;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int c = c0 + ((int)threadIdx.x >> 5) + 8 * k, f = f0 + lane;
        if (f >= a.f || c >= a.c) continue;
        const float sum = turned[lane][(threadIdx.x >> 5) + 8 * k];
        G* o = out + (int64_t)c * a.f + f;
        *o = from_f32<G>(a.accumulate ? to_f32<G>(*o) + sum : sum);
    }
}

// Channels / 32 that the kernels with rows in registers are built for: the next one that holds c (0: none, or the tiled kernels are faster).  They
// take a block of 128 rows a unit of its own through all hidden channels, so few rows leave units empty.  Measured, in us: rows in registers 0.18 (backward
// 0.45) for 32 hidden channels and 32 channels, for every 256 blocks; tiled 6 (15) for the launches and 400 TFLOP/s.
int rows_tiles(const ff_transition_desc& d, bool backward) {
    const int need = (d.c + 31) / 32, kc = d.dtype != FF_BF16 || need > 8 ? 0 : need == 1 ? 1 : (need + 1) / 2 * 2;
    const double turns = (double)((d.rows + 32767) / 32768) * ((d.f + 31) / 32) * kc, flop = (double)d.rows * d.c * d.f * (backward ? 10 : 6);
    return turns * (backward ? 0.45 : 0.18) <= (backward ? 15. : 6.) + flop / 4e8 ? kc : 0;
}
// ---- the calls -------------------------------------------------------------------------------
struct Sizes {
    int esz;
    int64_t cp, fp, chunk;         // padded channels; rows worked on at a time, a multiple of 128
    size_t weight;                 // bytes of a packed weight
    size_t tokens, hidden;         // bytes of a chunk's packed x and of its hidden tensor
    bool wide;                     // tiles of 256 in the weights' gradients
    int splits;
    int64_t per_split;
    size_t partial;
};
Sizes sizes_of(const ff_transition_desc& d, bool backward) {
    Sizes s;
    s.esz = d.dtype == FF_F32 ? 4 : 2;
    const int kc = rows_tiles(d, backward);
    s.cp = kc ? kc * 32 : round_up(d.c, kPad);
    s.fp = round_up(d.f, kc ? 32 : kPad);
    const int64_t most = std::max<int64_t>(128, kHiddenBytes / (std::max(s.fp, s.cp) * s.esz) / 128 * 128);
    s.chunk = std::min(most, round_up(std::max<int64_t>(d.rows, 1), 128));
    s.weight = align256((size_t)s.fp * s.cp * s.esz);
    s.tokens = align256((size_t)s.chunk * s.cp * s.esz);
    s.hidden = align256((size_t)s.chunk * s.fp * s.esz);
    // as many splits of the rows as give a block (of small tiles two or four) for each of 256 compute units, of 256 rows at least
    s.wide = d.dtype == FF_BF16 && d.f >= 256;
    const int least = d.dtype == FF_F32 ? 64 : 128, bm = s.wide ? 256 : least, bn = s.wide && d.c > 128 ? 256 : least, blocks = s.wide ? 256 : d.dtype == FF_F32 ? 1024 : 512;
    const int64_t tiles = 3 * ((d.f + bm - 1) / bm) * ((d.c + bn - 1) / bn);
    const int64_t want = std::max<int64_t>(1, std::min(blocks / tiles, s.chunk / 256));
    s.per_split = round_up((s.chunk + want - 1) / want, 128);
    s.splits = (int)((s.chunk + s.per_split - 1) / s.per_split);
    s.partial = align256((size_t)s.splits * 3 * s.fp * s.cp * 4);
    return s;
}

bool aligned(const void* p) { return ((uintptr_t)p & 15u) == 0; }

template <class C, auto KERNEL, typename Args> ff_status launch(int kind, const char* what, dim3 grid, const Args& args, hipStream_t stream) {
    Timed t(kind, stream);
    const ff_status st = tile::allow_lds<KERNEL>(what);
    if (st != FF_OK) return st;
    hipLaunchKernelGGL(KERNEL, grid, dim3(C::kThreads), C::kLds, stream, args);
    return check_launch(what);
}

PackJob pack_job(const void* src, void* dst, const float* mask, int64_t rows, int64_t rows_out, int cols, int64_t cols_out, int esz) {
    return {src, dst, mask, rows, rows_out, cols, (int32_t)cols_out, (uint32_t)((rows_out * (cols_out * esz / 16) + 255) / 256)};
}
template <typename T> ff_status pack(const PackJob* jobs, int n, hipStream_t stream) {
    PackArgs a{};
    uint32_t blocks = 0;
    for (int i = 0; i < n; ++i) {
        a.job[i] = jobs[i];
        blocks += jobs[i].blocks;
    }
    for (int i = n; i < 5; ++i) a.job[i] = jobs[n - 1];             // (never reached: no block is left for them)
    Timed t(KK_TR_PACK, stream);
    hipLaunchKernelGGL((k_tr_pack<T>), dim3(blocks), dim3(256), 0, stream, a);
    return check_launch("ff_gated_transition: packing");
}

Operand operand(const void* p, int64_t pitch, int64_t rows, int64_t cols, int esz) {
    return {p, pitch * esz, rows, (int32_t)(cols * esz)};
}

// the weights as the products read them: themselves, or padded copies in ws
struct Weights {
    Operand a, b, o;
    ff_status status;
};
template <typename T> Weights weights_of(const ff_transition_desc& d, const Sizes& s, const void* w_a, const void* w_b, const void* w_o, char*& ws, hipStream_t stream) {
    Weights w{};
    char* copies = ws;
    ws += 3 * s.weight;
    const bool as_is = d.c == s.cp && d.f == s.fp && aligned(w_a) && aligned(w_b) && aligned(w_o);
    const void* from[3] = {w_a, w_b, w_o};
    if (!as_is) {
        PackJob jobs[3];
        for (int i = 0; i < 3; ++i) {
            void* dst = copies + i * s.weight;
            jobs[i] = i < 2 ? pack_job(from[i], dst, nullptr, d.f, s.fp, d.c, s.cp, s.esz) : pack_job(from[i], dst, nullptr, d.c, s.cp, d.f, s.fp, s.esz);
            from[i] = dst;
        }
        w.status = pack<T>(jobs, 3, stream);
    }
    w.a = operand(from[0], s.cp, s.fp, s.cp, s.esz);
    w.b = operand(from[1], s.cp, s.fp, s.cp, s.esz);
    w.o = operand(from[2], s.fp, s.cp, s.fp, s.esz);
    return w;
}

template <int KC> ff_status launch_rows(int act, const RowsArgs& a, hipStream_t stream) {
    typedef rows::Weights<KC, 4> W;
    const dim3 grid((uint32_t)((a.rows + 127) / 128));
    const char* what = "ff_gated_transition_forward";
    return act == FF_SILU   ? launch<W, k_tr_rows<KC, FF_SILU>>(KK_TR_ROWS, what, grid, a, stream)
           : act == FF_GELU ? launch<W, k_tr_rows<KC, FF_GELU>>(KK_TR_ROWS, what, grid, a, stream)
                            : launch<W, k_tr_rows<KC, FF_SIGMOID>>(KK_TR_ROWS, what, grid, a, stream);
}
ff_status forward_rows(const ff_transition_desc& d, int kc, const void* x, const void* w_a, const void* w_b, const void* w_o, const void* residual, const float* mask,
                       void* y, void* ws_, hipStream_t stream) {
    const int64_t cp = kc * 32, fp = round_up(d.f, 32);
    const void* from[3] = {w_a, w_b, w_o};
    if (d.c != cp || d.f != fp || !aligned(w_a) || !aligned(w_b) || !aligned(w_o)) {
        PackJob jobs[3];
        char* ws = (char*)ws_;
        for (int i = 0; i < 3; ++i) {
            jobs[i] = i < 2 ? pack_job(from[i], ws, nullptr, d.f, fp, d.c, cp, 2) : pack_job(from[i], ws, nullptr, d.c, cp, d.f, fp, 2);
            from[i] = ws;
            ws += align256((size_t)(fp * cp * 2));
        }
        const ff_status st = pack<bf16_t>(jobs, 3, stream);
        if (st != FF_OK) return st;
    }
    const bool whole = d.c == cp && aligned(x) && aligned(residual) && aligned(y);
    for (int64_t r0 = 0; r0 < d.rows; r0 += kMostRows) {
        const auto at = [&](const void* t) { return t ? (const bf16_t*)t + r0 * d.c : nullptr; };
        const RowsArgs a{at(x), at(residual), (const char*)from[0], (const char*)from[1], (const char*)from[2], mask ? mask + r0 : nullptr, (bf16_t*)at(y), std::min(kMostRows, d.rows - r0),
                         (int32_t)fp, d.c, (int32_t)(fp * 2), whole};
        const ff_status st = kc == 1   ? launch_rows<1>(d.act, a, stream)
                             : kc == 2 ? launch_rows<2>(d.act, a, stream)
                             : kc == 4 ? launch_rows<4>(d.act, a, stream)
                             : kc == 6 ? launch_rows<6>(d.act, a, stream)
                                       : launch_rows<8>(d.act, a, stream);
        if (st != FF_OK) return st;
    }
    return FF_OK;
}

// ---- tiled products: the kernel of each tile size, and the choice among them -----------------------
// Large tiles ask less of L2 (128 x 128 in bfloat16 needs 65 bytes a clock and unit, of 64 there are), small ones fill the units: the largest that gives 200 blocks.
template <class C, auto SILU, auto GELU, auto SIGMOID, typename Args> ff_status run_act(int kind, const char* what, Args a, int64_t m, int64_t n, int act, hipStream_t stream) {
    a.mtiles = (uint32_t)((m + C::BM - 1) / C::BM);
    a.ntiles = (uint32_t)((n + C::BN - 1) / C::BN);
    const dim3 grid(a.mtiles * a.ntiles);
    return act == FF_SILU ? launch<C, SILU>(kind, what, grid, a, stream) : act == FF_GELU ? launch<C, GELU>(kind, what, grid, a, stream) : launch<C, SIGMOID>(kind, what, grid, a, stream);
}
template <typename T> struct Hidden {
    typedef T Type;
    typedef typename OpOf<T>::type Op;
    typedef Core<Op, 32, 32, 256 / sizeof(T), 4, 1, 1, 1, 2, 0, 0u, 4> Least;
    typedef Core<Op, 64, 64, 64 / sizeof(T), 4, 2, 2, 1, 2, 0, 0u> Small;
    typedef Core<Bf16, 128, 64, 32, 4, 2, 2, 1, 2, 0, 0u> Medium;
    typedef Core<Bf16, 256, 128, 32, 4, 4, 2, 1, 2, 0, 0u> Large;
    template <class C> static ff_status run(const HiddenArgs& a, int64_t m, int64_t n, int act, hipStream_t stream) {
        return run_act<C, k_tr_hidden<C, T, FF_SILU>, k_tr_hidden<C, T, FF_GELU>, k_tr_hidden<C, T, FF_SIGMOID>>(KK_TR_HIDDEN, "ff_gated_transition_forward", a, m, n, act, stream);
    }
};
template <typename T, unsigned TB> struct Out {
    typedef T Type;
    typedef typename OpOf<T>::type Op;
    typedef Core<Op, 32, 32, 256 / sizeof(T), 4, 1, 1, 1, 1, 0, TB, 4> Least;
    typedef Core<Op, 64, 64, 64 / sizeof(T), 4, 2, 2, 1, 1, 0, TB> Small;
    typedef Core<Bf16, 128, 128, 32, 4, 2, 2, 1, 1, 0, TB> Medium;
    typedef Core<Bf16, 256, 128, 32, 4, 4, 2, 1, 1, 0, TB> Large;
    template <class C> static ff_status run(OutArgs a, int64_t m, int64_t n, int, hipStream_t stream) {
        a.mtiles = (uint32_t)((m + C::BM - 1) / C::BM);
        a.ntiles = (uint32_t)((n + C::BN - 1) / C::BN);
        return launch<C, k_tr_out<C, T>>(KK_TR_OUT, "ff_gated_transition", dim3(a.mtiles * a.ntiles), a, stream);
    }
};
template <typename T> struct Grad {
    typedef T Type;
    typedef typename OpOf<T>::type Op;
    typedef Core<Op, 32, 32, 256 / sizeof(T), 3, 1, 1, 2, 3, 0, 4u, 4> Least;
    typedef Core<Op, 64, 64, 64 / sizeof(T), 3, 2, 2, 2, 3, 0, 4u> Small;
    typedef Core<Bf16, 128, 64, 32, 3, 2, 2, 2, 3, 0, 4u> Medium;
    typedef Core<Bf16, 128, 128, 32, 3, 4, 2, 2, 3, 0, 4u> Large;
    template <class C> static ff_status run(const GradArgs& a, int64_t m, int64_t n, int act, hipStream_t stream) {
        return run_act<C, k_tr_grad<C, T, FF_SILU>, k_tr_grad<C, T, FF_GELU>, k_tr_grad<C, T, FF_SIGMOID>>(KK_TR_GRAD, "ff_gated_transition_backward", a, m, n, act, stream);
    }
};
// Tiles of 64 by 64 that are few leave most units empty: four times as many of 32 by 32, k shared by four wavefronts, up to this many.  Float32, 16 rows of 384 channels with 1536
// hidden ones 55 -> 19 us, 400 rows 60 -> 32, with more of them 36; bfloat16, 16 rows of 1024 with 4096 37 -> 15, 100 rows 40 -> 20, 400 rows 46 -> 31.
constexpr int64_t kFewTiles = 128;
template <class C> bool enough(int64_t m, int64_t n) { return (m + C::BM - 1) / C::BM * ((n + C::BN - 1) / C::BN) >= 200; }
template <class K, typename Args> ff_status tiled(int64_t m, int64_t n, const Args& a, int act, hipStream_t stream) {
    // (float32 products are bound by their instructions, 64 cycles each: small tiles cost nothing)
    if constexpr (sizeof(typename K::Type) == 2) {
        if (enough<typename K::Large>(m, n)) return K::template run<typename K::Large>(a, m, n, act, stream);
        if (enough<typename K::Medium>(m, n)) return K::template run<typename K::Medium>(a, m, n, act, stream);
    }
    if ((m + 63) / 64 * ((n + 63) / 64) <= kFewTiles) return K::template run<typename K::Least>(a, m, n, act, stream);
    return K::template run<typename K::Small>(a, m, n, act, stream);
}

template <typename T> ff_status forward(const ff_transition_desc& d, const void* x, const void* w_a, const void* w_b, const void* w_o, const void* residual,
                                        const float* mask, void* y, void* ws_, hipStream_t stream) {
    const Sizes s = sizes_of(d, false);
    char* ws = (char*)ws_;
    const Weights w = weights_of<T>(d, s, w_a, w_b, w_o, ws, stream);
    if (w.status != FF_OK) return w.status;
    char* const tokens = ws;
    char* const hidden = tokens + s.tokens;
    const bool as_is = d.c % kPad == 0 && aligned(x);
    for (int64_t r0 = 0; r0 < d.rows; r0 += s.chunk) {
        const int64_t rows = std::min(s.chunk, d.rows - r0);
        const T* xr = (const T*)x + r0 * d.c;
        if (!as_is) {
            const PackJob job = pack_job(xr, tokens, nullptr, rows, rows, d.c, s.cp, s.esz);
            const ff_status st = pack<T>(&job, 1, stream);
            if (st != FF_OK) return st;
        }
        const HiddenArgs ha{operand(as_is ? (const void*)xr : tokens, s.cp, rows, s.cp, s.esz), {w.a, w.b}, hidden, rows, rows, d.f, (int32_t)s.cp, (int32_t)s.fp, 0, 0};
        ff_status st = tiled<Hidden<T>>(rows, s.fp, ha, d.act, stream);
        if (st != FF_OK) return st;
        OutArgs oa{};
        oa.a[0] = operand(hidden, s.fp, rows, s.fp, s.esz);
        oa.b[0] = w.o;
        oa.parts = 1;
        oa.k = (int32_t)s.fp;
        oa.cols = d.c;
        oa.rows = rows;
        oa.residual = residual ? (const T*)residual + r0 * d.c : nullptr;
        oa.mask = mask ? mask + r0 : nullptr;
        oa.out = (T*)y + r0 * d.c;
        st = tiled<Out<T, 0u>>(rows, d.c, oa, 0, stream);
        if (st != FF_OK) return st;
    }
    return FF_OK;
}

template <int KC> ff_status launch_grad_rows(int act, const GradRowsArgs& a, hipStream_t stream) {
    typedef rows::Weights<KC, 4> W;
    const dim3 grid((uint32_t)((a.rows_out + 127) / 128));
    const char* what = "ff_gated_transition_backward";
    return act == FF_SILU   ? launch<W, k_tr_grad_rows<KC, FF_SILU>>(KK_TR_GRAD, what, grid, a, stream)
           : act == FF_GELU ? launch<W, k_tr_grad_rows<KC, FF_GELU>>(KK_TR_GRAD, what, grid, a, stream)
                            : launch<W, k_tr_grad_rows<KC, FF_SIGMOID>>(KK_TR_GRAD, what, grid, a, stream);
}

// tiles of the weights' gradients: wide ones where there are enough hidden channels
struct Blocked {
    typedef Core<Bf16, 256, 256, 32, 4, 2, 4, 1, 1, 2, 1u> Square;
    typedef Core<Bf16, 256, 128, 32, 4, 4, 2, 1, 1, 2, 1u> Tall;
    typedef Core<Bf16, 128, 128, 32, 4, 2, 2, 1, 1, 2, 1u> Small;
};
template <typename T> struct Turned {
    typedef Core<typename OpOf<T>::type, sizeof(T) == 4 ? 64 : 128, sizeof(T) == 4 ? 64 : 128, 64 / sizeof(T), 4, 2, 2, 1, 1, 1, 1u> Small;
    typedef Core<Bf16, 256, 256, 32, 4, 2, 4, 1, 1, 1, 1u> Square;
};
template <class C> ff_status weights(WeightArgs a, int splits, hipStream_t stream) {
    a.ftiles = (uint32_t)((a.fp + C::BM - 1) / C::BM);
    a.ctiles = (uint32_t)((a.cp + C::BN - 1) / C::BN);
    return launch<C, k_tr_weights<C>>(KK_TR_WEIGHTS, "ff_gated_transition_backward", dim3(3 * a.ftiles * a.ctiles, splits), a, stream);
}

template <typename T> ff_status backward(const ff_transition_desc& d, const void* x, const void* w_a, const void* w_b, const void* w_o, const void* dy,
                                         const float* mask, void* dx, void* const (&dw)[3], int grad_dtype, bool accumulate, void* ws_, hipStream_t stream) {
    const Sizes s = sizes_of(d, true);
    char* ws = (char*)ws_;
    const Weights w = weights_of<T>(d, s, w_a, w_b, w_o, ws, stream);
    if (w.status != FF_OK) return w.status;
    char* const tokens[2] = {ws, ws + s.tokens};
    ws += 2 * s.tokens;
    char* const hidden[3] = {ws, ws + s.hidden, ws + 2 * s.hidden};
    float* const partial = (float*)(ws + 3 * s.hidden);
    const int kc = rows_tiles(d, true);
    const bool as_is = (kc ? d.c == s.cp : d.c % kPad == 0) && aligned(x) && aligned(dy);
    ff_status st = FF_OK;
    for (int64_t r0 = 0; r0 < d.rows; r0 += s.chunk) {
        const int64_t rows = std::min(s.chunk, d.rows - r0), padded = round_up(rows, kc ? 32 : kPad);
        const void* in[2] = {(const T*)x + r0 * d.c, (const T*)dy + r0 * d.c};
        const float* const live = mask ? mask + r0 : nullptr;
        const bool copies = !as_is || mask;
        if (kc) {
            if constexpr (sizeof(T) == 2) {
                const GradRowsArgs ga{(const bf16_t*)in[0], (const bf16_t*)in[1], (const char*)w.a.p, (const char*)w.b.p, (const char*)w.o.p, live, hidden[0], hidden[1],
                                      hidden[2], (bf16_t*)dx + r0 * d.c, copies ? (bf16_t*)tokens[0] : nullptr, (bf16_t*)tokens[1], rows, padded, (int32_t)s.fp, d.c,
                                      (int32_t)(s.fp * 2), as_is && aligned(dx)};
                st = kc == 1 ? launch_grad_rows<1>(d.act, ga, stream) : kc == 2 ? launch_grad_rows<2>(d.act, ga, stream) : kc == 4 ? launch_grad_rows<4>(d.act, ga, stream)
                     : kc == 6 ? launch_grad_rows<6>(d.act, ga, stream) : launch_grad_rows<8>(d.act, ga, stream);
            }
        } else {
            if (copies) {
                PackJob jobs[2];
                for (int i = 0; i < 2; ++i) jobs[i] = pack_job(in[i], tokens[i], live, rows, rows, d.c, s.cp, s.esz);
                st = pack<T>(jobs, 2, stream);
                if (st != FF_OK) return st;
            }
            const GradArgs ga{{operand(copies ? tokens[0] : in[0], s.cp, rows, s.cp, s.esz), operand(copies ? tokens[1] : in[1], s.cp, rows, s.cp, s.esz)}, {w.a, w.b, w.o},
                              hidden[0], hidden[1], hidden[2], rows, padded, d.f, (int32_t)s.cp, (int32_t)s.fp, 0, 0};
            st = tiled<Grad<T>>(padded, s.fp, ga, d.act, stream);
        }
        if (st != FF_OK) return st;
        const Operand ox = operand(copies ? tokens[0] : in[0], s.cp, rows, s.cp, s.esz), ody = operand(copies ? tokens[1] : in[1], s.cp, rows, s.cp, s.esz);
        Operand oh[3];
        for (int i = 0; i < 3; ++i) oh[i] = kc ? Operand{hidden[i], s.fp * 64, padded, (int32_t)(s.fp * 64)} : operand(hidden[i], s.fp, padded, s.fp, s.esz);
        WeightArgs wa{{oh[0], oh[1], oh[2]}, {ox, ox, ody}, partial, padded, s.per_split, (int32_t)s.fp, (int32_t)s.cp, 0, 0, r0 > 0};
        if (kc) st = s.wide ? d.c > 128 ? weights<Blocked::Square>(wa, s.splits, stream) : weights<Blocked::Tall>(wa, s.splits, stream) : weights<Blocked::Small>(wa, s.splits, stream);
        else st = s.wide ? weights<typename Turned<T>::Square>(wa, s.splits, stream) : weights<typename Turned<T>::Small>(wa, s.splits, stream);
        if (st != FF_OK || kc) {
            if (st != FF_OK) return st;
            continue;
        }
        OutArgs oa{};
        oa.a[0] = oh[0];
        oa.a[1] = oh[1];
        oa.b[0] = w.a;
        oa.b[1] = w.b;
        oa.parts = 2;
        oa.k = (int32_t)s.fp;
        oa.cols = d.c;
        oa.rows = rows;
        oa.out = (T*)dx + r0 * d.c;
        st = tiled<Out<T, 1u>>(rows, d.c, oa, 0, stream);
        if (st != FF_OK) return st;
    }
    JoinArgs ja{partial, {dw[0], dw[1], dw[2]}, d.f, d.c, (int32_t)s.fp, (int32_t)s.cp, d.rows ? s.splits : 0, accumulate};
    const dim3 grid((uint32_t)((d.c + 31) / 32), (uint32_t)((d.f + 31) / 32), 3);
    Timed t(KK_TR_JOIN, stream);
    if (grad_dtype == FF_F32) hipLaunchKernelGGL((k_tr_join<float>), grid, dim3(256), 0, stream, ja);
    else hipLaunchKernelGGL((k_tr_join<bf16_t>), grid, dim3(256), 0, stream, ja);
    return check_launch("ff_gated_transition_backward");
}

}  // namespace

size_t transition_forward_workspace(const ff_transition_desc& d) {
    if (const int kc = rows_tiles(d, false)) return std::max<size_t>(256, 3 * align256((size_t)(round_up(d.f, 32) * kc * 64)));
    const Sizes s = sizes_of(d, false);
    return 3 * s.weight + s.tokens + s.hidden;
}
size_t transition_backward_workspace(const ff_transition_desc& d) {
    const Sizes s = sizes_of(d, true);
    return 3 * s.weight + 2 * s.tokens + 3 * s.hidden + s.partial;
}
ff_status transition_forward_run(const ff_transition_desc& d, const void* x, const void* w_a, const void* w_b, const void* w_o, const void* residual,
                                 const float* mask, void* y, void* ws, hipStream_t stream) {
    if (const int kc = rows_tiles(d, false)) return forward_rows(d, kc, x, w_a, w_b, w_o, residual, mask, y, ws, stream);
    return d.dtype == FF_F32 ? forward<float>(d, x, w_a, w_b, w_o, residual, mask, y, ws, stream)
                             : forward<bf16_t>(d, x, w_a, w_b, w_o, residual, mask, y, ws, stream);
}
ff_status transition_backward_run(const ff_transition_desc& d, const void* x, const void* w_a, const void* w_b, const void* w_o, const void* dy,
                                  const float* mask, void* dx, void* dw_a, void* dw_b, void* dw_o, int grad_dtype, bool accumulate, void* ws, hipStream_t stream) {
    void* const dw[3] = {dw_a, dw_b, dw_o};
    return d.dtype == FF_F32 ? backward<float>(d, x, w_a, w_b, w_o, dy, mask, dx, dw, grad_dtype, accumulate, ws, stream)
                             : backward<bf16_t>(d, x, w_a, w_b, w_o, dy, mask, dx, dw, grad_dtype, accumulate, ws, stream);
}

}  // namespace ff
