// Orthogonalising updates by Newton-Schulz products, and the Muon step over the matrices of a model.
//
//   X = G / (|G| + eps);  per step, with n the shorter side:  A = X X^T (X^T X where a matrix is tall);  X = a X + (b A + c A^2) X  (X (...))
//
// Three launches a step for all matrices together: A; B = b A + c A^2; X = a X + B X.  What is added behind a product is added in float32: with a I inside B the rounding of B's
// diagonal, another one in each row, would carry the large singular directions into the small ones, which the next steps make larger (2048 x 2048: an
// error of 3.5e-6 in norm instead of 2.3e-6, and more beside more exact sums; b I inside an operand of B's product does the same).  Values are held as float16 pairs: 23
// significant bits, and three matrix instructions for a product where float32 ones would take sixteen times the time of one.  A and B are held times kScale, so that magnitudes to
// 255 have a place and the smallest are 2^-32 apart.  X is held times a power of two of its own in each step, from a bound of its norm: an update far below eps is a
// small X, of which a fixed factor would leave few bits or none (at 10^-5 eps, times 256: an error of 2e-3), and large matrices have small values.  With the usual coefficients singular
// values are at most 1 at the start and below 1.3 after any number of steps.  A tall matrix is worked on as it lies: its operands are read turned.
#include "ff_tile.h"

#include <math.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <new>
#include <vector>

namespace ff {

using tile::align256;
using tile::Core;
using tile::f32x16;
using tile::Operand;
using tile::Pair;
using tile::round_up;

namespace {

constexpr float kRoot = 16.f, kScale = kRoot * kRoot, kUnscale = 1.f / kScale;
constexpr int kPad = 16;
constexpr int64_t kHead = 256;                   // bytes in front of a matrix's workspace: the factor of X in each step, 64 floats
constexpr int kMostBlocks = 1 << 22;             // of a launch: 2^32 threads a grid
constexpr int kXcds = 8;                         // block i starts on XCD i % 8: places are laid out so that a matrix stays with one, whose L2 its tiles share
constexpr int kPiece = 4096;                     // values that a block of the element-wise kernels holds
constexpr int kFewSmall = 64;                    // small matrices beside large ones: so few are tiles more in the large ones' launches instead of a launch of 25 us behind them
constexpr int64_t kBatch = 1 << 30;              // workspace of the matrices that are worked on together, unless one alone needs more

// One matrix, as the kernels see it.
struct Matrix {
    const void* g;
    void* p;                                     // what the last step writes
    float* master;
    float* m;
    int64_t ws;                                  // bytes into the workspace: the factors of X; X, X of the next step, A and B as pairs
    int32_t rows, cols;
    int32_t piece0, pieces;                      // among the batch's
    float decay;
    int32_t pad;
    __host__ __device__ bool tall() const { return rows > cols; }
    __host__ __device__ int64_t rp() const { return (rows + kPad - 1) / kPad * kPad; }
    __host__ __device__ int64_t cp() const { return (cols + kPad - 1) / kPad * kPad; }
    __host__ __device__ int64_t np() const { return tall() ? cp() : rp(); }
    __host__ __device__ int64_t bytes_x() const { return rp() * cp() * 4; }
    __host__ __device__ int64_t bytes_a() const { return np() * np() * 4; }
    __host__ __device__ int64_t x(int which) const { return ws + kHead + which * bytes_x(); }
    __host__ __device__ int64_t a(int which) const { return ws + kHead + 2 * bytes_x() + which * bytes_a(); }
    __host__ __device__ int64_t bytes() const { return kHead + 2 * (bytes_x() + bytes_a()); }
};
struct Place {
    int32_t matrix, at;                          // matrix < 0: none
};

// Where the kernels find matrices and places: in a plan, or, for matrices of one shape that lie one after another, by counting.
struct Table {
    const Matrix* matrices;                      // NULL: `one`, its g and p moved on by in_step and out_step bytes, its ws by ws_step
    const Place* places;
    Matrix one;
    int64_t in_step, out_step, ws_step;
    int32_t count, each;                         // matrices; places of a matrix
};
__device__ __forceinline__ Matrix matrix_of(const Table& t, int32_t i) {
    if (t.matrices) return t.matrices[i];
    Matrix m = t.one;
    m.g = (const char*)m.g + i * t.in_step;
    m.p = (char*)m.p + i * t.out_step;
    m.ws += i * t.ws_step;
    m.piece0 = i * m.pieces;
    return m;
}
__device__ __forceinline__ Place place_at(const Table& t, uint32_t block) {
    if (t.matrices) return t.places[block];
    const uint32_t each = (uint32_t)t.each;
    if (t.count < kXcds) {                                     // few matrices: runs of tiles
        const uint32_t all = (uint32_t)t.count * each, run = (all + kXcds - 1) / kXcds, at = block % kXcds * run + block / kXcds;
        return {at < all ? (int32_t)(at / each) : -1, (int32_t)(at % each)};
    }
    const int32_t m = (int32_t)(block / kXcds / each * kXcds + block % kXcds);
    return {m < t.count ? m : -1, (int32_t)(block / kXcds % each)};
}
uint32_t places_of(int32_t count, int32_t each) {
    const uint32_t all = (uint32_t)count * (uint32_t)each;
    return count < kXcds ? (all + kXcds - 1) / kXcds * kXcds : (uint32_t)((count + kXcds - 1) / kXcds * kXcds) * (uint32_t)each;
}

// ---- pairs ---------------------------------------------------------------------------------
typedef __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16 f16x2;
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;
// two values, the first in the lower halves
__device__ __forceinline__ void split(float a, float b, uint32_t& hi, uint32_t& lo) {
    const f16x2 h = __builtin_convertvector((f32x2{a, b}), f16x2);
    hi = __builtin_bit_cast(uint32_t, h);
    lo = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a - (float)h[0], b - (float)h[1]}), f16x2));
}
__device__ __forceinline__ float join(uint32_t hi, uint32_t lo) {
    return (float)__builtin_bit_cast(_Float16, (uint16_t)hi) + (float)__builtin_bit_cast(_Float16, (uint16_t)lo);
}
// eight values of a row from value i of a matrix on (rows are multiples of sixteen values): their hi parts, and 32 bytes further their lo parts
__device__ __forceinline__ int64_t pairs_at(int64_t i) { return (i >> 4) * 64 + (i & 8) * 2; }
__device__ __forceinline__ void store_pairs(char* p, const float (&v)[8]) {
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) split(v[2 * q], v[2 * q + 1], hi[q], lo[q]);
    *(uint4*)p = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    *(uint4*)(p + 32) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
}
struct Pairs { uint4 hi, lo; };
__device__ __forceinline__ Pairs load_pairs(const char* p) { return {*(const uint4*)p, *(const uint4*)(p + 32)}; }
__device__ __forceinline__ float value_of(const Pairs& p, int q) {
    const uint32_t h[4] = {p.hi.x, p.hi.y, p.hi.z, p.hi.w}, l[4] = {p.lo.x, p.lo.y, p.lo.z, p.lo.w};
    return q & 1 ? join(h[q / 2] >> 16, l[q / 2] >> 16) : join(h[q / 2] & 0xffffu, l[q / 2] & 0xffffu);
}

// ---- momentum and norm ---------------------------------------------------------------------
struct StepArgs {
    float lr, beta, rest, max_norm;
    double eps;
    float a, b, c;
    float top_at[2], top[2];                     // where |a t + b t^3 + c t^5| has its maxima, and how high they are
    int32_t nesterov, rms;
};
// X has a norm, and values, of at most `bound`: the power of two that brings them below 2^14, of float16's 2^16.  (256 at least: a bound passes 255 with coefficients that let X
// grow, perhaps without X.  2^120 at most, so that its inverse and what is multiplied with it are float32 values of full precision.)
__device__ __forceinline__ float factor_of(float bound) {
    const int e = 140 - (int)(__float_as_uint(bound) >> 23 & 255u);
    return __uint_as_float((uint32_t)(127 + (e < 8 ? 8 : e > 120 ? 120 : e)) << 23);
}
constexpr float kRoom = 1.f + 1.f / 256.f;       // for roundings of the bound and of X
// of X = G by, by = 1 / (norm + eps).  A matrix of zeros is its own X, whatever eps is: 1 / 0, or the inverse of an eps below 2^-1024, is infinite and 0 times it NaN, which would reach
// the weights of a matrix that has no gradient yet.
__device__ __forceinline__ float first_bound(double norm, double eps, double& by) {
    by = norm == 0. ? 0. : 1. / (norm + eps);
    return (float)(norm * by) * kRoom;
}
__device__ __forceinline__ float next_bound(float bound, const StepArgs& a) {
    const float q = bound * bound;
    float v = fabsf(bound * (a.a + q * (a.b + q * a.c)));
#pragma unroll
    for (int i = 0; i < 2; ++i) v = a.top_at[i] < bound && v < a.top[i] ? a.top[i] : v;
    return v * kRoom;
}
__device__ __forceinline__ float clip_of(const float* norm, float max_norm, bool& skip) {
    if (!norm) return 1.f;
    const float n = *norm;
    skip = !(n <= 3.402823466e38f);
    const float c = max_norm / (n + 1e-6f);
    return c < 1.f ? c : 1.f;
}

// eight values at padded place i (a row's pad is none of them)
struct Spot {
    int64_t r, at;
    int c, n;
};
__device__ __forceinline__ Spot spot_of(const Matrix& x, int64_t i) {
    Spot s;
    const int64_t cp = x.cp();
    s.r = i / cp;
    s.c = (int)(i - s.r * cp);
    const int left = x.cols - s.c;
    s.n = s.r < x.rows ? (left < 0 ? 0 : left < 8 ? left : 8) : 0;
    s.at = s.r * x.cols + s.c;
    return s;
}
// the update that is orthogonalised, of the new momentum and the gradient
__device__ __forceinline__ float update_of(float m, float g, const StepArgs& a) { return a.nesterov ? a.beta * m + a.rest * g : m; }

// m = beta m + (1 - beta) k g, and the sum of squares of the update, in float64.  MUON false: of g itself.  Bound by HBM: 48 blocks' 79 M values
// in matrices beyond 128 x 128, bfloat16 gradients, 135 us for 770 MB, 5.7 TB/s.
template <typename G, bool MUON> __global__ __launch_bounds__(256) void k_muon_momentum(Table t, StepArgs a, const float* norm, double* partial) {
    const Place at = place_at(t, blockIdx.x);
    if (at.matrix < 0) return;
    const Matrix x = matrix_of(t, at.matrix);
    bool skip = false;
    const float k = MUON ? clip_of(norm, a.max_norm, skip) : 1.f;
    const int64_t end = x.rp() * x.cp(), first = (int64_t)at.at * kPiece;
    double sum = 0.;
    for (int64_t i = first + threadIdx.x * 8; i < first + kPiece && i < end; i += 256 * 8) {
        const Spot s = spot_of(x, i);
        float g[8], m[8];
        tile::load_some((const G*)x.g + s.at, s.n, g);
        if constexpr (MUON) {
            tile::load_some((const float*)x.m + s.at, s.n, m);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                g[q] *= k;
                m[q] = a.beta * m[q] + a.rest * g[q];
                g[q] = update_of(m[q], g[q], a);
            }
            if (!skip) tile::store_some(x.m + s.at, s.n, m);
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) sum += q < s.n ? (double)g[q] * g[q] : 0.;
    }
    __shared__ double sums[256];
    sums[threadIdx.x] = sum;
    __syncthreads();
    for (int n = 128; n > 0; n >>= 1) {
        if ((int)threadIdx.x < n) sums[threadIdx.x] += sums[threadIdx.x + n];
        __syncthreads();
    }
    if (threadIdx.x == 0) partial[x.piece0 + at.at] = sums[0];
}

__device__ __forceinline__ float* factors_of(const Matrix& x, char* ws) { return (float*)(ws + x.ws); }

// X = update / (norm + eps) as pairs, its padding zeros, and its factors.  Bound by HBM likewise: 159 us for 770 MB.  (The update is formed again: it would be another 4 bytes a value.)
template <typename G, bool MUON> __global__ __launch_bounds__(256) void k_ns_start(Table t, StepArgs a, const float* norm, const double* partial, char* ws, int steps) {
    const Place at = place_at(t, blockIdx.x);
    if (at.matrix < 0) return;
    const Matrix x = matrix_of(t, at.matrix);
    bool skip = false;
    const float k = MUON ? clip_of(norm, a.max_norm, skip) : 1.f;
    if (skip) return;
    __shared__ double sums[256];
    double sum = 0.;
    for (int i = threadIdx.x; i < x.pieces; i += 256) sum += partial[x.piece0 + i];
    sums[threadIdx.x] = sum;
    __syncthreads();
    for (int n = 128; n > 0; n >>= 1) {
        if ((int)threadIdx.x < n) sums[threadIdx.x] += sums[threadIdx.x + n];
        __syncthreads();
    }
    double by;
    float bound = first_bound(sqrt(sums[0]), a.eps, by);
    const double inv = by * factor_of(bound);
    if (at.at == 0 && threadIdx.x == 0)
        for (int s = 0; s < steps; ++s, bound = next_bound(bound, a)) factors_of(x, ws)[s] = factor_of(bound);
    const int64_t end = x.rp() * x.cp(), first = (int64_t)at.at * kPiece;
    char* out = ws + x.x(0);
    for (int64_t i = first + threadIdx.x * 8; i < first + kPiece && i < end; i += 256 * 8) {
        const Spot s = spot_of(x, i);
        float g[8], m[8];
        tile::load_some((const G*)x.g + s.at, s.n, g);
        if constexpr (MUON) {
            tile::load_some((const float*)x.m + s.at, s.n, m);                            // (the new one)
#pragma unroll
            for (int q = 0; q < 8; ++q) g[q] = update_of(m[q], g[q] * k, a);
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) g[q] = q < s.n ? (float)(g[q] * inv) : 0.f;
        store_pairs(out + pairs_at(i), g);
    }
}

// ---- the products --------------------------------------------------------------------------
template <int TILE_, int BK, int STAGES, int BLOCKS> struct Cores {
    static constexpr int TILE = TILE_;
    typedef Core<Pair, TILE, TILE, BK, STAGES, 2, 2, 1, 1, 0, 0u> Straight;        // rows by rows
    typedef Core<Pair, TILE, TILE, BK, STAGES, 2, 2, 1, 1, 1, 1u> Turned;          // columns by columns
    typedef Core<Pair, TILE, TILE, BK, STAGES, 2, 2, 1, 1, 0, 1u> Mixed;           // rows by columns
    static constexpr int kBlocks = BLOCKS;                                         // on a compute unit
    static constexpr size_t kLds = std::max({Straight::kLds, Turned::kLds, Mixed::kLds});
};
// Three stages of 16 k leave room for three blocks on a compute unit, whose ends then overlap with the others' products.  Where a launch has fewer blocks than there are
// units a block stands alone with what a stage costs it, a barrier and the reads behind it, so that stages of 32 k are better (orthogonalising 4096 x 1024: eight of 16 k
// 434 us, five of 32 383, four 374; of 64 k for the smaller tiles 390: all while the ends read no A and no X; 391 now).  Fewer blocks still, and tiles of 64 fill four times the units.
typedef Cores<128, 16, 3, 3> Many;
typedef Cores<128, 32, 4, 1> Some;
typedef Cores<64, 32, 4, 2> Few;

__device__ __forceinline__ Operand operand_x(const Matrix& x, const char* ws, int which) {
    return {ws + x.x(which), x.cp() * 4, x.rp(), (int32_t)(x.cp() * 4)};
}
__device__ __forceinline__ Operand operand_a(const Matrix& x, const char* ws, int which) {
    return {ws + x.a(which), x.np() * 4, x.np(), (int32_t)(x.np() * 4)};
}
// tile t of the lower triangle, row by row
__device__ __forceinline__ void triangle(int t, int& i, int& j) {
    i = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
    while (i * (i + 1) / 2 > t) --i;
    while ((i + 1) * (i + 2) / 2 <= t) ++i;
    j = t - i * (i + 1) / 2;
}
// eight values of A, row m from column n on (a multiple of eight)
__device__ __forceinline__ void store_gram(char* a, int64_t np, int64_t m, int64_t n, const float (&v)[8]) {
    if (m < np && n < np) store_pairs(a + pairs_at(m * np + n), v);
}

// A.  SPLIT: sums over a part of k each, for k_ns_join.  48 blocks: 126 us for 2016 tiles, the matrix units 0.38 busy, 480 MB through HBM at 3.7 TB/s: k is 256 long for most tiles, so a third is
// the way in and out.  4096 x 1024: 136 tiles of 64 in three parts each 25 us and 5 for the join.
template <class C, bool SPLIT> __global__ __launch_bounds__(256, C::kBlocks) void k_ns_gram(Table t, char* ws, int step, float* parts) {
    typedef typename C::Straight Straight;
    constexpr int kTile = C::TILE;
    extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
    const Place at = place_at(t, blockIdx.x);
    if (at.matrix < 0) return;
    const Matrix x = matrix_of(t, at.matrix);
    int i, j;
    triangle(at.at, i, j);
    const Operand o = operand_x(x, ws, step & 1);
    const float factor = factors_of(x, ws)[step];
    f32x16 acc[1][Straight::MT][Straight::NT];
    Straight::clear(acc);
    const int64_t all = x.tall() ? x.rp() : x.cp(), each = SPLIT ? (all / kPad + gridDim.y - 1) / gridDim.y * kPad : all, from = SPLIT ? blockIdx.y * each : 0;
    const int64_t to = from + each < all ? from + each : all;
    if (x.tall()) C::Turned::run(acc, &o, &o, (int64_t)i * kTile, (int64_t)j * kTile, from, to, smem);
    else Straight::run(acc, &o, &o, (int64_t)i * kTile, (int64_t)j * kTile, from, to, smem);
    if constexpr (SPLIT) {
        float* out = parts + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kTile * kTile;
        Straight::rows(acc[0], 0, 0, smem, Straight::none, [&](int64_t m, int64_t n, float (&v)[8], typename Straight::Nothing) { tile::store8(out + m * kTile + n, v); });
    } else {
        const float by = kRoot / factor;                           // its square is kScale over that of X's factor (and no float32 value where that is large)
        const auto store = [&](int64_t m, int64_t n, float (&v)[8], typename Straight::Nothing) {
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] = v[q] * by * by;
            store_gram(ws + x.a(0), x.np(), m, n, v);
        };
        Straight::rows(acc[0], (int64_t)i * kTile, (int64_t)j * kTile, smem, Straight::none, store);
        if (i != j) Straight::columns(acc[0], (int64_t)i * kTile, (int64_t)j * kTile, smem, Straight::none, store);
    }
}

// A of its parts, added up in their order; a block has 32 rows of a tile
__global__ __launch_bounds__(256) void k_ns_join(Table t, char* ws, int step, const float* parts, int splits) {
    constexpr int kTile = Few::TILE, kBand = 32, kPitch = kBand + 1;
    __shared__ float band[kTile * kPitch];
    const Place at = place_at(t, blockIdx.x);
    if (at.matrix < 0) return;
    const Matrix x = matrix_of(t, at.matrix);
    int i, j;
    triangle(at.at, i, j);
    const int64_t np = x.np(), m0 = (int64_t)i * kTile + blockIdx.y * kBand, n0 = (int64_t)j * kTile;
    char* to = ws + x.a(0);
    const int64_t next = (int64_t)gridDim.x * kTile * kTile;
    const float by = kRoot / factors_of(x, ws)[step];
    const float* from = parts + ((int64_t)blockIdx.x * kTile + blockIdx.y * kBand) * kTile;
    for (int u = threadIdx.x; u < kBand * kTile / 8; u += 256) {
        const int r = u / (kTile / 8), c = u % (kTile / 8) * 8;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, more[8];
#pragma unroll 4
        for (int s = 0; s < splits; ++s) {
            tile::load8(from + s * next + u * 8, more);
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] += more[q];
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) band[(c + q) * kPitch + r] = v[q] = v[q] * by * by;
        store_gram(to, np, m0 + r, n0 + c, v);
    }
    if (i == j) return;
    tile::barrier();
    for (int u = threadIdx.x; u < kTile * kBand / 8; u += 256) {
        const int r = u / (kBand / 8), c = u % (kBand / 8) * 8;
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = band[r * kPitch + c + q];
        store_gram(to, np, n0 + r, m0 + c, v);
    }
}

// B = b A + c A^2.  48 blocks 107 us for 490 MB; 4096 x 1024 15 us, 32 stages of 32 k in a row by half the units.
template <class C> __global__ __launch_bounds__(256, C::kBlocks) void k_ns_poly(Table t, char* ws, StepArgs a) {
    typedef typename C::Straight Straight;
    constexpr int kTile = C::TILE;
    extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
    const Place at = place_at(t, blockIdx.x);
    if (at.matrix < 0) return;
    const Matrix x = matrix_of(t, at.matrix);
    int i, j;
    triangle(at.at, i, j);
    const Operand oa = operand_a(x, ws, 0);
    f32x16 acc[1][Straight::MT][Straight::NT];
    Straight::clear(acc);
    const int64_t np = x.np();
    Straight::run(acc, &oa, &oa, (int64_t)i * kTile, (int64_t)j * kTile, 0, np, smem);
    char* out = ws + x.a(1);
    const char* was = ws + x.a(0);
    const auto fetch = [&](int64_t m, int64_t n) { return m < np && n < np ? load_pairs(was + pairs_at(m * np + n)) : Pairs{}; };
    const auto store = [&](int64_t m, int64_t n, float (&v)[8], const Pairs& old) {
        if (m >= np || n >= np) return;
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = a.b * value_of(old, q) + (a.c * kUnscale) * v[q];
        store_pairs(out + pairs_at(m * np + n), v);
    };
    Straight::rows(acc[0], (int64_t)i * kTile, (int64_t)j * kTile, smem, fetch, store);
    if (i != j) Straight::columns(acc[0], (int64_t)i * kTile, (int64_t)j * kTile, smem, fetch, store);
}

enum Last { kMore = 0, kOut = 1, kWeights = 2 };
__device__ __forceinline__ float size_of(const Matrix& x, const StepArgs& a) {
    const int32_t longer = x.rows > x.cols ? x.rows : x.cols;
    return a.lr * (a.rms ? 0.2f * sqrtf((float)longer) : sqrtf((float)longer / (float)x.cols));
}
// `left` values (of eight) of the result at place `at` of the matrix
template <int LAST, typename P> __device__ __forceinline__ void finish(const Matrix& x, const StepArgs& a, float size, int64_t at, int left, const float (&v)[8]) {
    P* p = (P*)x.p + at;
    if constexpr (LAST == kOut) tile::store_some(p, left, v);
    else {
        const float decay = a.lr * x.decay;
        float w[8];
        if (x.master) tile::load_some((const float*)x.master + at, left, w);
        else tile::load_some((const P*)p, left, w);
#pragma unroll
        for (int q = 0; q < 8; ++q) w[q] -= decay * w[q] + size * v[q];
        if (x.master) tile::store_some(x.master + at, left, w);
        tile::store_some(p, left, w);
    }
}
// X = a X + B X (a X + X B where a matrix is tall); the last step's goes to the caller: as it is, or into the weights.  48 blocks 223 us for 1.05 GB, of which 270 MB are X once more for the end (the last, with
// weights and masters, 299 for 1.51 GB);
// 4096 x 1024 36 us, 256 tiles, one a unit, 23 of them matrix instructions at the rate of a large product.
template <int LAST, typename P, class C> __global__ __launch_bounds__(256, C::kBlocks) void k_ns_apply(Table t, char* ws, int step, StepArgs a, const float* norm) {
    typedef typename C::Straight Straight;
    constexpr int kTile = C::TILE;
    extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
    const Place at = place_at(t, blockIdx.x);
    if (at.matrix < 0) return;
    const Matrix x = matrix_of(t, at.matrix);
    if (LAST == kWeights) {
        bool skip = false;
        (void)clip_of(norm, a.max_norm, skip);
        if (skip) return;
    }
    const int64_t rp = x.rp(), cp = x.cp();
    const int ntiles = (int)((cp + kTile - 1) / kTile), i = at.at / ntiles, j = at.at % ntiles;
    const Operand ox = operand_x(x, ws, step & 1), ob = operand_a(x, ws, 1);
    const float factor = factors_of(x, ws)[step], next = LAST == kMore ? factors_of(x, ws)[step + 1] : 1.f;
    f32x16 acc[1][Straight::MT][Straight::NT];
    Straight::clear(acc);
    if (x.tall()) Straight::run(acc, &ox, &ob, (int64_t)i * kTile, (int64_t)j * kTile, 0, cp, smem);
    else C::Mixed::run(acc, &ob, &ox, (int64_t)i * kTile, (int64_t)j * kTile, 0, rp, smem);
    char* to = ws + x.x(~step & 1);
    const float size = size_of(x, a), by = next / factor;
    const char* was = ws + x.x(step & 1);
    const auto fetch = [&](int64_t m, int64_t n) { return m < rp && n < cp ? load_pairs(was + pairs_at(m * cp + n)) : Pairs{}; };
    Straight::rows(acc[0], (int64_t)i * kTile, (int64_t)j * kTile, smem, fetch, [&](int64_t m, int64_t n, float (&v)[8], const Pairs& old) {
        if (m >= rp || n >= cp) return;
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = (a.a * value_of(old, q) + kUnscale * v[q]) * by;
        if constexpr (LAST == kMore) store_pairs(to + pairs_at(m * cp + n), v);
        else {
            const int left = x.cols - (int)n;
            if (m >= x.rows || left <= 0) return;
            finish<LAST, P>(x, a, size, m * x.cols + n, left, v);
        }
    });
}

// ---- small matrices: everything in one block ---------------------------------------------------
// A matrix of at most SIZE x SIZE stays in LDS from its momentum to its weights: X and A (then B in A's place) as pairs in rows of SIZE values, a product's
// results in registers between two barriers.  A wavefront has one 32 x 32 tile of the result (SIZE 64), or two beside each other (SIZE 128).
// Bound by the chain of 3 steps dependent products, each a barrier, reads from LDS, 3 k / 16 matrix instructions in a row and the rounding into pairs: one 128 x 64 31 us (2.0 a product),
// where the other path needs seventeen launches; 1200 matrices of up to 128 x 128 on 256 units 420 us, the matrix units 0.29 busy.
template <int SIZE> struct Small {
    static constexpr int kWaves = SIZE == 128 ? 8 : 4, kThreads = 64 * kWaves, kUnits = SIZE == 128 ? 2 : 1;
    static constexpr int W = SIZE / 4, kImage = SIZE * SIZE * 4, kLds = 2 * kImage;
    // sixteen bytes of row `row`: eight values from column c, a multiple of eight, of the hi part (p = 0) or the lo part.  Rows that one cycle reads together, straight or turned, lie in banks of their own.
    static __device__ __forceinline__ int at(int row, int c, int p) { return row * (W * 16) + (((c >> 4) * 4 + p * 2 + (c >> 3 & 1)) ^ ((row & 1) << 1 | (row & 2) << 2 | (row >> 2 & 1) | (row & 8) >> 1)) * 16; }

    // 32 rows (straight) or columns (turned) from `first`, k = 16 s ..: a lane's address is a number of its own, an exclusive or with what s, the part and the half of a
    // turned read change of the slot, and a constant.
    template <bool T> static __device__ __forceinline__ int lane_of(int first, int lane) {
        const int hf = lane >> 5, i = lane & 15;
        if constexpr (!T) return at(first + (lane & 31), 8 * hf, 0);
        return at(8 * hf + (i >> 2), first + (lane & 16) + 8 * (i >> 1 & 1), 0) + (i & 1) * 8;
    }
    template <bool T> static __device__ __forceinline__ Pair::Frag frag(const unsigned char* image, int of, int s) {
        Pair::Frag f;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            if constexpr (!T) f.u[p] = *(const uint4*)(image + (of ^ ((4 * s + 2 * p & 15) << 4)) + (4 * s & ~15) * 16);
            else {
                uint2 h[2];
#pragma unroll
                for (int t = 0; t < 2; ++t) h[t] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tile::lds_i16x4)(image + (of ^ (2 * p ^ t) << 4) + (16 * s + 4 * t) * (W * 16))));
                f.u[p] = make_uint4(h[0].x, h[0].y, h[1].x, h[1].y);
            }
        }
        return f;
    }
    // the four values that a lane holds as results 4 g .. 4 g + 3 of tile u, of the hi part (p = 0) or the lo part; of = at(m0 + lane % 32, n0, 0) + 8 (lane / 32), n0 a multiple of 32 (of 64 for two tiles)
    static __device__ __forceinline__ int result_at(int of, int u, int g, int p) {
        return (of ^ ((8 * u + 4 * (g >> 1) + 2 * p + (g & 1) & 15) << 4)) + (8 * u & ~15) * 16;
    }
    template <int TILES> struct Frags {
        Pair::Frag a, b[TILES];
    };
    template <int P> static __device__ __forceinline__ f32x16 part(const Pair::Frag& b, const Pair::Frag& a, f32x16 c) {       // lo hi, hi lo, hi hi
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(tile::f16x8, b.u[P == 0]), __builtin_bit_cast(tile::f16x8, a.u[P == 1]), c, 0, 0, 0);
    }
    // TILES tiles of the product of two images over k (a multiple of sixteen); operands are read a round ahead.  An instruction waits for the one before on its
    // accumulator: two tiles take turns, of one the cross terms have an accumulator of their own.
    template <bool TA, bool TB, int TILES>
    static __device__ __forceinline__ void product(f32x16 (&acc)[kUnits], const unsigned char* a, const unsigned char* b, int m0, int n0, int k, int lane) {
        f32x16 c[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int v = 0; v < 16; ++v) c[u][v] = 0.f;
        const int oa = lane_of<TA>(m0, lane), ob = lane_of<TB>(n0, lane), ob2 = TILES == 2 ? lane_of<TB>(n0 + 32, lane) : 0, rounds = k / 16;
        Frags<TILES> f[2];
        const auto read = [&](Frags<TILES>& f, int s) {
            f.a = frag<TA>(a, oa, s);
            f.b[0] = frag<TB>(b, ob, s);
            if constexpr (TILES == 2) f.b[1] = frag<TB>(b, ob2, s);
        };
        const auto turn = [&](int s, Frags<TILES>& now, Frags<TILES>& then) {
            read(then, s + 1 < rounds ? s + 1 : s);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (TILES == 2) {
                c[0] = part<0>(now.b[0], now.a, c[0]);
                c[1] = part<0>(now.b[1], now.a, c[1]);
                c[0] = part<1>(now.b[0], now.a, c[0]);
                c[1] = part<1>(now.b[1], now.a, c[1]);
                c[0] = part<2>(now.b[0], now.a, c[0]);
                c[1] = part<2>(now.b[1], now.a, c[1]);
            } else {
                c[1] = part<0>(now.b[0], now.a, c[1]);
                c[0] = part<2>(now.b[0], now.a, c[0]);
                c[1] = part<1>(now.b[0], now.a, c[1]);
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        read(f[0], 0);
        int s = 0;
        for (; s + 1 < rounds; s += 2) {
            turn(s, f[0], f[1]);
            turn(s + 1, f[1], f[0]);
        }
        if (s < rounds) turn(s, f[0], f[1]);
        if constexpr (TILES == 1) acc[0] = c[0] + c[1];
        else {
            acc[0] = c[0];
            acc[1] = c[1];
        }
    }
    // the wavefront's tiles, none to kUnits
    template <bool TA, bool TB>
    static __device__ __forceinline__ void product(f32x16 (&acc)[kUnits], const unsigned char* a, const unsigned char* b, int m0, int n0, int tiles, int k, int lane) {
        if constexpr (kUnits == 2) {
            if (tiles == 2) return product<TA, TB, 2>(acc, a, b, m0, n0, k, lane);
        }
        if (tiles == 1) product<TA, TB, 1>(acc, a, b, m0, n0, k, lane);
    }
    // what store() has written there
    static __device__ __forceinline__ void load(f32x16 (&acc)[kUnits], const unsigned char* from, int m0, int n0, int tiles, int rows, int cols, int lane) {
        if (m0 + (lane & 31) >= rows) return;
        const int of = at(m0 + (lane & 31), n0, 0) + 8 * (lane >> 5);
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
            if (u < tiles)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    if (n0 + 32 * u + 8 * g >= cols) continue;
                    const uint2 hi = *(const uint2*)(from + result_at(of, u, g, 0)), lo = *(const uint2*)(from + result_at(of, u, g, 1));
                    const uint32_t h[2] = {hi.x, hi.y}, l[2] = {lo.x, lo.y};
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[u][4 * g + q] = q & 1 ? join(h[q / 2] >> 16, l[q / 2] >> 16) : join(h[q / 2] & 0xffffu, l[q / 2] & 0xffffu);
                }
    }
    // rows and columns below the given numbers
    static __device__ __forceinline__ void store(const f32x16 (&acc)[kUnits], unsigned char* to, int m0, int n0, int tiles, int rows, int cols, int lane) {
        if (m0 + (lane & 31) >= rows) return;
        const int of = at(m0 + (lane & 31), n0, 0) + 8 * (lane >> 5);
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
            if (u < tiles)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    if (n0 + 32 * u + 8 * g >= cols) continue;
                    uint32_t hi[2], lo[2];
#pragma unroll
                    for (int q = 0; q < 2; ++q) split(acc[u][4 * g + 2 * q], acc[u][4 * g + 2 * q + 1], hi[q], lo[q]);
                    *(uint2*)(to + result_at(of, u, g, 0)) = make_uint2(hi[0], hi[1]);
                    *(uint2*)(to + result_at(of, u, g, 1)) = make_uint2(lo[0], lo[1]);
                }
    }
};

template <int SIZE, int LAST, typename G, typename P> __global__ __launch_bounds__(Small<SIZE>::kThreads) void k_ns_small(Table t, int first, int steps, StepArgs a, const float* norm) {
    typedef Small<SIZE> S;
    constexpr bool MUON = LAST == kWeights;
    extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
    unsigned char *const xs = smem, *const as = smem + S::kImage;
    const Matrix x = matrix_of(t, first + (int)blockIdx.x);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    bool skip = false;
    const float k = MUON ? clip_of(norm, a.max_norm, skip) : 1.f;
    if (skip) return;
    const int rp = (int)x.rp(), cp = (int)x.cp(), np = (int)x.np();
    // the update, in registers, and the sum of its squares
    constexpr int kTurns = SIZE * SIZE / 8 / S::kThreads;
    float g[kTurns][8];
    double sum = 0.;
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const int64_t place = (int64_t)(i * S::kThreads + (int)threadIdx.x) * 8;
        if (place >= (int64_t)rp * cp) continue;
        const Spot s = spot_of(x, place);
        tile::load_some((const G*)x.g + s.at, s.n, g[i]);
        if constexpr (MUON) {
            float m[8];
            tile::load_some((const float*)x.m + s.at, s.n, m);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                g[i][q] *= k;
                m[q] = a.beta * m[q] + a.rest * g[i][q];
                g[i][q] = update_of(m[q], g[i][q], a);
            }
            tile::store_some(x.m + s.at, s.n, m);
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            g[i][q] = q < s.n ? g[i][q] : 0.f;
            sum += (double)g[i][q] * g[i][q];
        }
    }
    double* sums = (double*)smem;
    sums[threadIdx.x] = sum;
    __syncthreads();
    for (int n = S::kThreads / 2; n > 0; n >>= 1) {
        if ((int)threadIdx.x < n) sums[threadIdx.x] += sums[threadIdx.x + n];
        __syncthreads();
    }
    double per;
    float bound = first_bound(sqrt(sums[0]), a.eps, per), factor = factor_of(bound);
    const double inv = per * factor;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const int place = (i * S::kThreads + (int)threadIdx.x) * 8;
        if (place >= rp * cp) continue;
        const int r = place / cp, c = place % cp;
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) split((float)(g[i][2 * q] * inv), (float)(g[i][2 * q + 1] * inv), hi[q], lo[q]);
        *(uint4*)(xs + S::at(r, c, 0)) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        *(uint4*)(xs + S::at(r, c, 1)) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
    // Three products a step, one piece of code: A of X; B = b A + c A^2, into A's place; X = a X + B X.  A wavefront has the same tiles of A and of B, and keeps
    // its A; and its tiles of X.
    tile::barrier();
    struct Tiles {
        int rows, cols, m0, n0, count;
    };
    const auto tiles_of = [&](int rows, int cols) {
        const int across = (cols + 31) / 32, down = (rows + 31) / 32, each = across * down > S::kWaves ? S::kUnits : 1, groups = (across + each - 1) / each;
        const int m0 = wave / groups * 32, n0 = wave % groups * each * 32;
        return Tiles{rows, cols, m0, n0, wave < groups * down ? (across - n0 / 32 < each ? across - n0 / 32 : each) : 0};
    };
    const Tiles square = tiles_of(np, np), whole = tiles_of(rp, cp);
    f32x16 acc[S::kUnits] = {}, held[S::kUnits] = {}, kept[S::kUnits] = {};          // kept: X before it is rounded
    S::load(kept, xs, whole.m0, whole.n0, whole.count, rp, cp, lane);
#pragma unroll 1
    for (int phase = 0, left = 3 * steps; left > 0; --left) {
        const bool last = phase == 2, tall = x.tall();
        const Tiles mine = last ? whole : square;
        if (phase == 0 && tall) S::template product<true, true>(acc, xs, xs, mine.m0, mine.n0, mine.count, rp, lane);
        else if (last && !tall) S::template product<false, true>(acc, as, xs, mine.m0, mine.n0, mine.count, rp, lane);
        else S::template product<false, false>(acc, phase == 1 ? as : xs, phase == 0 ? xs : as, mine.m0, mine.n0, mine.count, phase == 1 ? np : cp, lane);
        float by = kRoot / factor;                              // as in k_ns_gram
        if (last) {
            bound = next_bound(bound, a);
            const float next = factor_of(bound);
            by = next / factor;
            factor = next;
        }
#pragma unroll
        for (int u = 0; u < S::kUnits; ++u) {
            if (phase == 1) acc[u] = a.b * held[u] + (a.c * kUnscale) * acc[u];
            else if (last) kept[u] = acc[u] = (a.a * kept[u] + kUnscale * acc[u]) * by;
            else held[u] = acc[u] = acc[u] * by * by;
        }
        if (phase > 0) tile::barrier();                        // all have read what is overwritten (A's place holds B at first, which nobody reads any more)
        S::store(acc, last ? xs : as, mine.m0, mine.n0, mine.count, mine.rows, mine.cols, lane);
        tile::barrier();
        phase = last ? 0 : phase + 1;
    }
    const float size = size_of(x, a), by = 1.f / factor;
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const int place = (i * S::kThreads + (int)threadIdx.x) * 8;
        if (place >= rp * cp) continue;
        const Spot s = spot_of(x, place);
        if (s.n == 0) continue;
        const Pairs p{*(const uint4*)(xs + S::at((int)s.r, s.c, 0)), *(const uint4*)(xs + S::at((int)s.r, s.c, 1))};
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = by * value_of(p, q);
        finish<LAST, P>(x, a, size, s.at, s.n, v);
    }
}

// ---- launches --------------------------------------------------------------------------------
struct Batch {
    int64_t ws;                                   // bytes of workspace of its matrices
    int32_t piece0, pieces, tri0, tris, app0, apps;        // places of the three kinds, in the plan's lists
    int32_t splits, tri_tile, app_tile, pad;         // parts of k in the Gram matrices, 1 = whole; tiles of 64 or 128
};
int pieces_of(const Matrix& m) { return (int)((m.rp() * m.cp() + kPiece - 1) / kPiece); }
int tris_of(const Matrix& m, int tile) {
    const int n = (int)((m.np() + tile - 1) / tile);
    return n * (n + 1) / 2;
}
int apps_of(const Matrix& m, int tile) { return (int)((m.rp() + tile - 1) / tile * ((m.cp() + tile - 1) / tile)); }
// the tiles of a launch that would have this many blocks with the large ones
int tile_for(int64_t large) { return large < 192 ? 64 : 128; }
int small_of(const Matrix& m) { return std::max(m.rows, m.cols) <= 64 ? 64 : std::max(m.rows, m.cols) <= 128 ? 128 : 0; }
// Few Gram tiles of a long k: k is split, in parts of 512 and more (the join costs as much as 512 of k).
int splits_of(int tile, int64_t tris, int64_t longest) {
    const int64_t s = std::min<int64_t>({8, 512 / std::max<int64_t>(tris, 1), longest / 512});
    return tile == 64 && s >= 3 ? (int)s : 1;
}
int64_t parts_bytes(int64_t tris, int splits) { return splits > 1 ? tris * splits * Few::TILE * Few::TILE * 4 : 0; }

template <auto KERNEL, typename... A> ff_status go(int kind, dim3 blocks, int threads, size_t lds, hipStream_t stream, const char* what, A... args) {
    Timed t(kind, stream);
    if (lds) {
        const ff_status st = tile::allow_lds<KERNEL>(what);
        if (st != FF_OK) return st;
    }
    hipLaunchKernelGGL(KERNEL, blocks, dim3(threads), lds, stream, args...);
    return check_launch(what);
}

// All steps of one batch.  Tables for the three kinds of places differ in `places` (of a plan) or `each`.
struct Tables {
    Table piece, tri, app;
    uint32_t pieces, tris, apps;
    int splits, tri_tile, app_tile;
    double* partial;
    float* parts;
};
// the polynomial and its maxima: the roots t^2 of a + 3 b t^2 + 5 c t^4
void polynomial(StepArgs& s, double a, double b, double c) {
    s.a = (float)a;
    s.b = (float)b;
    s.c = (float)c;
    const double half = 3 * b / 2, disc = half * half - 5 * c * a, root = half < 0 ? half - sqrt(std::max(disc, 0.)) : half + sqrt(std::max(disc, 0.));
    const double q[2] = {root != 0 ? -a / root : 0, c != 0 ? -root / (5 * c) : 0};
    for (int i = 0; i < 2; ++i) {
        const bool there = disc >= 0 && q[i] > 0;
        s.top_at[i] = there ? (float)sqrt(q[i]) : INFINITY;
        s.top[i] = there ? (float)fabs(sqrt(q[i]) * (a + q[i] * (b + q[i] * c))) : 0.f;
    }
}
template <int LAST> constexpr const char* kWhat = LAST == kWeights ? "ff_muon_step" : "ff_orthogonalise";

template <class C, int LAST, typename P> ff_status apply(const Tables& t, int step, const StepArgs& a, const float* norm, char* ws, hipStream_t stream) {
    return go<k_ns_apply<LAST, P, C>>(KK_NS_APPLY, t.apps, 256, C::kLds, stream, kWhat<LAST>, t.app, ws, step, a, norm);
}
template <int LAST, typename P> ff_status apply(const Tables& t, int step, const StepArgs& a, const float* norm, char* ws, hipStream_t stream) {
    return t.app_tile == 64 ? apply<Few, LAST, P>(t, step, a, norm, ws, stream)
           : t.apps > 256   ? apply<Many, LAST, P>(t, step, a, norm, ws, stream)
                            : apply<Some, LAST, P>(t, step, a, norm, ws, stream);
}
// A of X, B of A
template <class C> ff_status gram(const Tables& t, int step, const StepArgs& a, char* ws, hipStream_t stream, const char* what) {
    ff_status st;
    const auto whole = [&] { return go<k_ns_gram<C, false>>(KK_NS_GRAM, t.tris, 256, C::kLds, stream, what, t.tri, ws, step, (float*)nullptr); };
    if constexpr (C::TILE == 64) {
        if (t.splits > 1) {
            st = go<k_ns_gram<C, true>>(KK_NS_GRAM, dim3(t.tris, t.splits), 256, C::kLds, stream, what, t.tri, ws, step, t.parts);
            if (st == FF_OK) st = go<k_ns_join>(KK_NS_GRAM, dim3(t.tris, 2), 256, 0, stream, what, t.tri, ws, step, (const float*)t.parts, t.splits);
        } else
            st = whole();
    } else
        st = whole();
    return st != FF_OK ? st : go<k_ns_poly<C>>(KK_NS_POLY, t.tris, 256, C::kLds, stream, what, t.tri, ws, a);
}
template <typename G, typename P, int LAST> ff_status steps_of(const Tables& t, const StepArgs& a, int steps, const float* norm, char* ws, hipStream_t stream) {
    constexpr bool MUON = LAST == kWeights;
    const char* what = kWhat<LAST>;
    ff_status st = go<k_muon_momentum<G, MUON>>(KK_MUON_MOMENTUM, t.pieces, 256, 0, stream, what, t.piece, a, norm, t.partial);
    if (st == FF_OK) st = go<k_ns_start<G, MUON>>(KK_NS_START, t.pieces, 256, 0, stream, what, t.piece, a, norm, (const double*)t.partial, ws, steps);
    for (int s = 0; s < steps && st == FF_OK; ++s) {
        st = t.tri_tile == 64 ? gram<Few>(t, s, a, ws, stream, what) : t.tris > 256 ? gram<Many>(t, s, a, ws, stream, what) : gram<Some>(t, s, a, ws, stream, what);
        if (st == FF_OK) st = s + 1 < steps ? apply<kMore, float>(t, s, a, norm, ws, stream) : apply<LAST, P>(t, s, a, norm, ws, stream);
    }
    return st;
}
// `count` matrices of a size from `first` on, a block each
template <typename G, typename P, int LAST> ff_status small(const Table& t, int size, int first, int count, const StepArgs& a, int steps, const float* norm, hipStream_t stream) {
    for (; count > 0; first += kMostBlocks, count -= kMostBlocks) {
        const int n = std::min(count, kMostBlocks);
        const ff_status st = size == 64 ? go<k_ns_small<64, LAST, G, P>>(KK_NS_SMALL, n, Small<64>::kThreads, Small<64>::kLds, stream, kWhat<LAST>, t, first, steps, a, norm)
                                        : go<k_ns_small<128, LAST, G, P>>(KK_NS_SMALL, n, Small<128>::kThreads, Small<128>::kLds, stream, kWhat<LAST>, t, first, steps, a, norm);
        if (st != FF_OK) return st;
    }
    return FF_OK;
}

// ---- a plan: header, batches, matrices, places -------------------------------------------------
struct Header {
    uint32_t tag;
    int32_t matrices, batches, pieces, tris, apps;
    int32_t small, smaller;                       // matrices of at most 128 x 128 and, behind them, of at most 64 x 64, the last of all
    int64_t ws;                                   // the largest batch's
    int64_t bytes;                                // of the plan
};
static_assert(sizeof(Header) % 16 == 0 && sizeof(Matrix) % 16 == 0 && sizeof(Batch) % 8 == 0, "the plan's records");
uint32_t tag_of(const ff_muon_desc& d) { return 0x4d000000u | d.param_dtype << 8 | d.grad_dtype; }

struct Layout {
    int64_t batches, matrices, piece, tri, app, bytes;
};
Layout layout_of(const Header& h) {
    Layout l;
    l.batches = sizeof(Header);
    l.matrices = round_up(l.batches + (int64_t)sizeof(Batch) * h.batches, 16);
    l.piece = l.matrices + (int64_t)sizeof(Matrix) * h.matrices;
    l.tri = l.piece + (int64_t)sizeof(Place) * h.pieces;
    l.app = l.tri + (int64_t)sizeof(Place) * h.tris;
    l.bytes = round_up(l.app + (int64_t)sizeof(Place) * h.apps, 16);
    return l;
}

Matrix matrix_from(const ff_muon_tensor& t) {
    Matrix m{};
    m.g = t.g;
    m.p = t.p;
    m.master = t.master;
    m.m = t.m;
    m.rows = t.rows;
    m.cols = t.cols;
    m.decay = t.weight_decay;
    m.pieces = pieces_of(m);
    return m;
}
// Places of matrices first .. last - 1 in an order that keeps a matrix (a run of its tiles, where few matrices have many) on one XCD and loads all eight alike
template <typename Count, typename Weight>
void spread(const std::vector<Matrix>& matrices, int first, int last, Count count, Weight weight, std::vector<Place>& out) {
    int64_t total = 0;
    for (int i = first; i < last; ++i) total += count(matrices[i]);
    const int run = (int)((total + 4 * kXcds - 1) / (4 * kXcds));
    std::vector<Place> queue[kXcds];
    int64_t load[kXcds] = {};
    for (int i = first; i < last; ++i) {
        const int n = count(matrices[i]);
        for (int at = 0; at < n; at += run) {
            const int q = (int)(std::min_element(load, load + kXcds) - load), end = std::min(n, at + run);
            load[q] += (end - at) * weight(matrices[i]);
            for (int k = at; k < end; ++k) queue[q].push_back({i, k});
        }
    }
    size_t longest = 0;
    for (const auto& q : queue) longest = std::max(longest, q.size());
    for (size_t k = 0; k < longest; ++k)
        for (const auto& q : queue) out.push_back(k < q.size() ? q[k] : Place{-1, 0});
}
struct Made {
    std::vector<Matrix> matrices;
    std::vector<Batch> batches;
    std::vector<Place> piece, tri, app;
    int64_t ws = 256;
    int small = 0, smaller = 0;
};
// Large matrices first, so that small ones fill the end; a batch ends where its workspace would pass kBatch (but for small ones, which are worked on with large ones where they are few).
Made make(const ff_muon_desc& d, const ff_muon_tensor* ts) {
    Made r;
    for (int i = 0; i < d.n_tensors; ++i)
        if (ts[i].rows > 0 && ts[i].cols > 0) r.matrices.push_back(matrix_from(ts[i]));
    std::stable_sort(r.matrices.begin(), r.matrices.end(), [](const Matrix& a, const Matrix& b) { return std::max(a.rp(), a.cp()) > std::max(b.rp(), b.cp()); });
    int large = 0;
    for (const Matrix& m : r.matrices) {
        large += small_of(m) == 0;
        r.small += small_of(m) == 128;
        r.smaller += small_of(m) == 64;
    }
    if (large > 0 && r.small + r.smaller <= kFewSmall) {
        large += r.small + r.smaller;
        r.small = r.smaller = 0;
    }
    for (int first = 0; first < large;) {
        Batch b{};
        b.piece0 = (int32_t)r.piece.size();
        b.tri0 = (int32_t)r.tri.size();
        b.app0 = (int32_t)r.app.size();
        int last = first;
        int64_t tris = 0, apps = 0, few = 0, longest = 0, room = 0;
        for (; last < large && (last == first || room + r.matrices[last].bytes() <= kBatch || small_of(r.matrices[last])); ++last) {
            const Matrix& m = r.matrices[last];
            room += (int64_t)align256((size_t)m.bytes());
            tris += tris_of(m, 128);
            apps += apps_of(m, 128);
            few += tris_of(m, 64);
            longest = std::max(longest, std::max(m.rp(), m.cp()));
        }
        for (int i = first; i < last; ++i) {
            Matrix& m = r.matrices[i];
            m.ws = b.ws;
            m.piece0 = b.pieces;
            b.ws += (int64_t)align256((size_t)m.bytes());
            b.pieces += m.pieces;
            for (int32_t k = 0; k < m.pieces; ++k) r.piece.push_back({i, k});
        }
        b.tri_tile = tile_for(tris);
        b.app_tile = tile_for(apps);
        b.splits = splits_of(b.tri_tile, few, longest);
        spread(r.matrices, first, last, [&](const Matrix& m) { return tris_of(m, b.tri_tile); }, [](const Matrix& m) { return std::max(m.rp(), m.cp()) + 128; }, r.tri);
        spread(r.matrices, first, last, [&](const Matrix& m) { return apps_of(m, b.app_tile); }, [](const Matrix& m) { return m.np() + 128; }, r.app);
        b.tris = (int32_t)(r.tri.size() - b.tri0);
        b.apps = (int32_t)(r.app.size() - b.app0);
        r.ws = std::max(r.ws, b.ws + (int64_t)align256((size_t)b.pieces * 8) + parts_bytes(b.tris, b.splits));
        if (r.piece.size() > INT32_MAX / 2 || r.tri.size() > INT32_MAX / 2 || r.app.size() > INT32_MAX / 2) throw std::bad_alloc();
        r.batches.push_back(b);
        first = last;
    }
    return r;
}
Header header_of(const ff_muon_desc& d, const Made& r) {
    Header h{};
    h.tag = tag_of(d);
    h.matrices = (int32_t)r.matrices.size();
    h.batches = (int32_t)r.batches.size();
    h.pieces = (int32_t)r.piece.size();
    h.tris = (int32_t)r.tri.size();
    h.apps = (int32_t)r.app.size();
    h.small = r.small;
    h.smaller = r.smaller;
    h.ws = r.ws;
    h.bytes = layout_of(h).bytes;
    return h;
}

}  // namespace

size_t muon_plan_size(const ff_muon_desc& d, const ff_muon_tensor* ts) {
    try {
        return (size_t)header_of(d, make(d, ts)).bytes;
    } catch (const std::bad_alloc&) {
        return 0;
    }
}
// 0: done; 1: overlaps; -1: no host memory
int muon_plan_fill(const ff_muon_desc& d, const ff_muon_tensor* ts, void* plan) {
    try {
        std::vector<ff_adamw_tensor> flat((size_t)d.n_tensors);
        for (int i = 0; i < d.n_tensors; ++i) {
            flat[i] = ff_adamw_tensor{};
            flat[i].p = ts[i].p;
            flat[i].g = ts[i].g;
            flat[i].master = ts[i].master;
            flat[i].m = ts[i].m;
            flat[i].numel = (int64_t)ts[i].rows * ts[i].cols;
        }
        const ff_adamw_desc ad{d.param_dtype, d.grad_dtype, 32, d.n_tensors};
        const int overlaps = adamw_overlaps(ad, flat.data());
        if (overlaps) return overlaps;
        const Made r = make(d, ts);
        const Header h = header_of(d, r);
        const Layout l = layout_of(h);
        char* out = (char*)plan;
        memset(out, 0, (size_t)h.bytes);
        memcpy(out, &h, sizeof h);
        const auto put = [&](int64_t at, const void* from, size_t bytes) {
            if (bytes) memcpy(out + at, from, bytes);
        };
        put(l.batches, r.batches.data(), sizeof(Batch) * r.batches.size());
        put(l.matrices, r.matrices.data(), sizeof(Matrix) * r.matrices.size());
        put(l.piece, r.piece.data(), sizeof(Place) * r.piece.size());
        put(l.tri, r.tri.data(), sizeof(Place) * r.tri.size());
        put(l.app, r.app.data(), sizeof(Place) * r.app.size());
        return 0;
    } catch (const std::bad_alloc&) {
        return -1;
    }
}
bool muon_plan_whole(const ff_muon_desc& d, const void* plan_host, size_t bytes) {
    Header h;
    if (bytes < sizeof h) return false;
    memcpy(&h, plan_host, sizeof h);
    return h.tag == tag_of(d) && h.bytes == (int64_t)bytes && layout_of(h).bytes == (int64_t)bytes;
}
size_t muon_workspace(const void* plan_host) { return (size_t)((const Header*)plan_host)->ws; }

namespace {
template <typename G, typename P> ff_status muon_step(const Header& head, const void* plan_host, const char* dev, const StepArgs& a, int steps, const float* norm, char* ws, hipStream_t stream) {
    const Layout l = layout_of(head);
    Table t{};
    t.matrices = (const Matrix*)(dev + l.matrices);
    for (int i = 0; i < head.batches; ++i) {
        const Batch& b = ((const Batch*)((const char*)plan_host + l.batches))[i];
        char* const partial = ws + b.ws;
        Tables ts{t, t, t, (uint32_t)b.pieces, (uint32_t)b.tris, (uint32_t)b.apps, b.splits, b.tri_tile, b.app_tile, (double*)partial, (float*)(partial + align256((size_t)b.pieces * 8))};
        ts.piece.places = (const Place*)(dev + l.piece) + b.piece0;
        ts.tri.places = (const Place*)(dev + l.tri) + b.tri0;
        ts.app.places = (const Place*)(dev + l.app) + b.app0;
        const ff_status st = steps_of<G, P, kWeights>(ts, a, steps, norm, ws, stream);
        if (st != FF_OK) return st;
    }
    const int first = head.matrices - head.small - head.smaller;
    const ff_status st = small<G, P, kWeights>(t, 128, first, head.small, a, steps, norm, stream);
    return st != FF_OK ? st : small<G, P, kWeights>(t, 64, first + head.small, head.smaller, a, steps, norm, stream);
}
}  // namespace

ff_status muon_step_run(const ff_muon_desc& d, const void* plan_host, const void* plan, const ff_muon_hyper& h, const float* norm, void* ws, hipStream_t stream) {
    const Header& head = *(const Header*)plan_host;
    StepArgs a{};
    a.lr = (float)h.lr;
    a.beta = (float)h.beta;
    a.rest = (float)(1. - h.beta);
    a.max_norm = norm ? (float)h.max_norm : 0.f;
    a.eps = h.eps;
    polynomial(a, h.a, h.b, h.c);
    a.nesterov = h.nesterov;
    a.rms = h.scale == FF_MUON_RMS;
    const char* dev = (const char*)plan;
    if (d.param_dtype == FF_F32)
        return d.grad_dtype == FF_F32 ? muon_step<float, float>(head, plan_host, dev, a, h.steps, norm, (char*)ws, stream)
                                      : muon_step<bf16_t, float>(head, plan_host, dev, a, h.steps, norm, (char*)ws, stream);
    return d.grad_dtype == FF_F32 ? muon_step<float, bf16_t>(head, plan_host, dev, a, h.steps, norm, (char*)ws, stream)
                                  : muon_step<bf16_t, bf16_t>(head, plan_host, dev, a, h.steps, norm, (char*)ws, stream);
}

// ---- matrices of one shape -------------------------------------------------------------------
namespace {
struct Uniform {
    Matrix one;
    int64_t bytes;             // of workspace a matrix
    int32_t group;             // matrices worked on together
    int splits, tri_tile, app_tile;
    uint32_t tris;             // places of a group
};
Uniform uniform_of(const ff_orthogonalise_desc& d) {
    Uniform u{};
    u.one.rows = d.rows;
    u.one.cols = d.cols;
    u.one.pieces = pieces_of(u.one);
    u.bytes = (int64_t)align256((size_t)u.one.bytes());
    u.group = (int32_t)std::max<int64_t>(1, std::min<int64_t>(d.count, kBatch / u.bytes));
    u.tri_tile = tile_for((int64_t)u.group * tris_of(u.one, 128));
    u.app_tile = tile_for((int64_t)u.group * apps_of(u.one, 128));
    u.splits = splits_of(u.tri_tile, (int64_t)u.group * tris_of(u.one, 64), std::max(u.one.rp(), u.one.cp()));
    u.tris = places_of(u.group, tris_of(u.one, u.tri_tile));
    return u;
}
template <typename T> ff_status orthogonalise(const ff_orthogonalise_desc& d, const void* x, void* out, char* ws, hipStream_t stream) {
    const Uniform u = uniform_of(d);
    StepArgs a{};
    a.eps = d.eps;
    polynomial(a, d.a, d.b, d.c);
    Table t{};
    t.one = u.one;
    t.in_step = t.out_step = (int64_t)d.rows * d.cols * (int64_t)sizeof(T);
    t.ws_step = u.bytes;
    if (const int size = small_of(u.one)) {
        t.one.g = x;
        t.one.p = out;
        return small<T, T, kOut>(t, size, 0, d.count, a, d.steps, nullptr, stream);
    }
    char* const partial = ws + u.bytes * u.group;
    for (int32_t i = 0; i < d.count; i += u.group) {
        t.count = std::min(u.group, d.count - i);
        t.one.g = (const char*)x + i * t.in_step;
        t.one.p = (char*)out + i * t.out_step;
        Tables ts{t, t, t, 0, 0, 0, u.splits, u.tri_tile, u.app_tile, (double*)partial, (float*)(partial + align256((size_t)u.group * u.one.pieces * 8))};
        ts.pieces = places_of(t.count, ts.piece.each = u.one.pieces);
        ts.tris = places_of(t.count, ts.tri.each = tris_of(u.one, u.tri_tile));
        ts.apps = places_of(t.count, ts.app.each = apps_of(u.one, u.app_tile));
        const ff_status st = steps_of<T, T, kOut>(ts, a, d.steps, nullptr, ws, stream);
        if (st != FF_OK) return st;
    }
    return FF_OK;
}
}  // namespace
size_t orthogonalise_workspace(const ff_orthogonalise_desc& d) {
    const Uniform u = uniform_of(d);
    if (small_of(u.one)) return 256;
    return (size_t)u.bytes * u.group + align256((size_t)u.group * u.one.pieces * 8) + (size_t)parts_bytes(u.tris, u.splits);
}
ff_status orthogonalise_run(const ff_orthogonalise_desc& d, const void* x, void* out, void* ws, hipStream_t stream) {
    return d.dtype == FF_F32 ? orthogonalise<float>(d, x, out, (char*)ws, stream) : orthogonalise<bf16_t>(d, x, out, (char*)ws, stream);
}

}  // namespace ff
