// Orthogonalising updates by Newton-Schulz products, and the Muon step over the matrices of a model.
//
//   X = G / (|G| + eps);  per step, with n the shorter side:  A = X X^T (X^T X where a matrix is tall);  X = a X + (b A + c A^2) X  (X (...))
//
// Three launches a step for all matrices together: the Gram matrix, the polynomial, its product with X.  Values are held as float16 pairs of kScale times
// themselves: 24 significant bits, and three matrix instructions for a product where float32 ones would take sixteen times the time of one.  Magnitudes
// to 255 have a place, and singular values are at most 1 at the start and below 1.3 after any number of steps with the usual coefficients; 2^-33 is
// the smallest step between small values.  A tall matrix is worked on as it lies: its operands are read turned.
#include "ff_tile.h"

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

constexpr float kScale = 256.f, kUnscale = 1.f / 256.f;
constexpr int kPad = 16;
constexpr int kTile = 128;
constexpr int kPiece = 16384;                    // values that a block of the element-wise kernels holds
constexpr int64_t kBatch = 256 << 20;            // workspace of the matrices that are worked on together, unless one alone needs more

// One matrix, as the kernels see it.
struct Matrix {
    const void* g;
    void* p;                                     // what the last step writes
    float* master;
    float* m;
    int64_t ws;                                  // bytes into the workspace: X, X of the next step, A, B, as pairs
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
    __host__ __device__ int64_t x(int which) const { return ws + which * bytes_x(); }
    __host__ __device__ int64_t a(int which) const { return ws + 2 * bytes_x() + which * bytes_a(); }
    __host__ __device__ int64_t bytes() const { return 2 * bytes_x() + 2 * bytes_a(); }
};
struct Place {
    int32_t matrix, at;
};

// Where the kernels find matrices and places: in a plan, or, for matrices of one shape that lie one after another, by counting.
struct Table {
    const Matrix* matrices;                      // NULL: `one`, its g and p moved on by in_step and out_step bytes, its ws by ws_step
    const Place* places;
    Matrix one;
    int64_t in_step, out_step, ws_step;
    int32_t each;                                // places of a matrix
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
    return {(int32_t)(block / (uint32_t)t.each), (int32_t)(block % (uint32_t)t.each)};
}

// ---- pairs ---------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t half_bits(_Float16 h) { return __builtin_bit_cast(uint16_t, h); }
__device__ __forceinline__ void split(float v, uint32_t& hi, uint32_t& lo) {
    const _Float16 h = (_Float16)v;
    hi = half_bits(h);
    lo = half_bits((_Float16)(v - (float)h));
}
__device__ __forceinline__ float join(uint32_t hi, uint32_t lo) {
    return (float)__builtin_bit_cast(_Float16, (uint16_t)hi) + (float)__builtin_bit_cast(_Float16, (uint16_t)lo);
}
// eight values of a row from value i of a matrix on (rows are multiples of sixteen values): their hi parts, and 32 bytes further their lo parts
__device__ __forceinline__ int64_t pairs_at(int64_t i) { return (i >> 4) * 64 + (i & 8) * 2; }
__device__ __forceinline__ void store_pairs(char* p, const float (&v)[8]) {
    uint32_t hi[8], lo[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) split(v[q], hi[q], lo[q]);
    *(uint4*)p = make_uint4(hi[0] | hi[1] << 16, hi[2] | hi[3] << 16, hi[4] | hi[5] << 16, hi[6] | hi[7] << 16);
    *(uint4*)(p + 32) = make_uint4(lo[0] | lo[1] << 16, lo[2] | lo[3] << 16, lo[4] | lo[5] << 16, lo[6] | lo[7] << 16);
}
__device__ __forceinline__ void load_pairs(const char* p, float (&v)[8]) {
    const uint4 h4 = *(const uint4*)p, l4 = *(const uint4*)(p + 32);
    const uint32_t h[4] = {h4.x, h4.y, h4.z, h4.w}, l[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = q & 1 ? join(h[q / 2] >> 16, l[q / 2] >> 16) : join(h[q / 2] & 0xffffu, l[q / 2] & 0xffffu);
}

// ---- momentum and norm ---------------------------------------------------------------------
struct StepArgs {
    float lr, beta, rest, max_norm;
    double eps;
    float a, b, c;
    int32_t nesterov, rms;
};
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

// m = beta m + (1 - beta) k g, and the sum of squares of the update, in float64: bound by HBM.  MUON false: of g itself.
template <typename G, bool MUON> __global__ __launch_bounds__(256) void k_muon_momentum(Table t, StepArgs a, const float* norm, double* partial) {
    const Place at = place_at(t, blockIdx.x);
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

// X = update / (norm + eps) as pairs, its padding zeros
template <typename G, bool MUON> __global__ __launch_bounds__(256) void k_ns_start(Table t, StepArgs a, const float* norm, const double* partial, char* ws) {
    const Place at = place_at(t, blockIdx.x);
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
    const double inv = (double)kScale / (sqrt(sums[0]) + a.eps);
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
typedef Core<Pair, kTile, kTile, 16, 4, 2, 2, 1, 1, false, 0u> Straight;      // rows by rows
typedef Core<Pair, kTile, kTile, 16, 4, 2, 2, 1, 1, true, 1u> Turned;         // columns by columns
typedef Core<Pair, kTile, kTile, 16, 4, 2, 2, 1, 1, false, 1u> Mixed;         // rows by columns

constexpr size_t kTileLds = std::max({Straight::kLds, Turned::kLds, Mixed::kLds});

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
// a tile of a symmetric matrix and its mirror image; value(m, n, v) turns sums into what is held
template <class C, typename F>
__device__ __forceinline__ void store_symmetric(f32x16 (&acc)[C::MT][C::NT], char* out, int64_t np, int i, int j, unsigned char* smem, F value) {
    const auto store = [&](int64_t m, int64_t n, float (&v)[8]) {
        if (m >= np || n >= np) return;
        value(m, n, v);
        store_pairs(out + pairs_at(m * np + n), v);
    };
    C::rows(acc, (int64_t)i * kTile, (int64_t)j * kTile, smem, store);
    if (i != j) C::columns(acc, (int64_t)i * kTile, (int64_t)j * kTile, smem, store);
}

__global__ __launch_bounds__(256, 2) void k_ns_gram(Table t, char* ws, int which) {
    extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
    const Place at = place_at(t, blockIdx.x);
    const Matrix x = matrix_of(t, at.matrix);
    int i, j;
    triangle(at.at, i, j);
    const Operand o = operand_x(x, ws, which);
    f32x16 acc[1][Straight::MT][Straight::NT];
    Straight::clear(acc);
    if (x.tall()) Turned::run(acc, &o, &o, (int64_t)i * kTile, (int64_t)j * kTile, 0, x.rp(), smem);
    else Straight::run(acc, &o, &o, (int64_t)i * kTile, (int64_t)j * kTile, 0, x.cp(), smem);
    store_symmetric<Straight>(acc[0], ws + x.a(0), x.np(), i, j, smem, [&](int64_t, int64_t, float (&v)[8]) {
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] *= kUnscale;
    });
}

// B = b A + c A^2
__global__ __launch_bounds__(256, 2) void k_ns_poly(Table t, char* ws, float b, float c) {
    extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
    const Place at = place_at(t, blockIdx.x);
    const Matrix x = matrix_of(t, at.matrix);
    int i, j;
    triangle(at.at, i, j);
    const Operand o = operand_a(x, ws, 0);
    f32x16 acc[1][Straight::MT][Straight::NT];
    Straight::clear(acc);
    const int64_t np = x.np();
    Straight::run(acc, &o, &o, (int64_t)i * kTile, (int64_t)j * kTile, 0, np, smem);
    const char* a = ws + x.a(0);
    store_symmetric<Straight>(acc[0], ws + x.a(1), np, i, j, smem, [&](int64_t m, int64_t n, float (&v)[8]) {
        float was[8];
        load_pairs(a + pairs_at(m * np + n), was);
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = b * was[q] + (c * kUnscale) * v[q];
    });
}

enum Last { kMore = 0, kOut = 1, kWeights = 2 };
// X = a X + B X (X B where a matrix is tall); the last step's goes to the caller: as it is, or into the weights
template <int LAST, typename P> __global__ __launch_bounds__(256, 2) void k_ns_apply(Table t, char* ws, int which, StepArgs a, const float* norm) {
    extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
    const Place at = place_at(t, blockIdx.x);
    const Matrix x = matrix_of(t, at.matrix);
    if (LAST == kWeights) {
        bool skip = false;
        (void)clip_of(norm, a.max_norm, skip);
        if (skip) return;
    }
    const int64_t rp = x.rp(), cp = x.cp();
    const int ntiles = (int)((cp + kTile - 1) / kTile), i = at.at / ntiles, j = at.at % ntiles;
    const Operand ox = operand_x(x, ws, which), ob = operand_a(x, ws, 1);
    f32x16 acc[1][Straight::MT][Straight::NT];
    Straight::clear(acc);
    if (x.tall()) Straight::run(acc, &ox, &ob, (int64_t)i * kTile, (int64_t)j * kTile, 0, cp, smem);
    else Mixed::run(acc, &ob, &ox, (int64_t)i * kTile, (int64_t)j * kTile, 0, rp, smem);
    const char* from = ws + x.x(which);
    char* to = ws + x.x(which ^ 1);
    const int32_t longer = x.rows > x.cols ? x.rows : x.cols;
    const float size = a.lr * (a.rms ? 0.2f * sqrtf((float)longer) : sqrtf((float)longer / (float)x.cols)), decay = a.lr * x.decay;
    Straight::rows(acc[0], (int64_t)i * kTile, (int64_t)j * kTile, smem, [&](int64_t m, int64_t n, float (&v)[8]) {
        if (m >= rp || n >= cp) return;
        float was[8];
        load_pairs(from + pairs_at(m * cp + n), was);
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = a.a * was[q] + kUnscale * v[q];
        if constexpr (LAST == kMore) store_pairs(to + pairs_at(m * cp + n), v);
        else {
            const int left = x.cols - (int)n;
            if (m >= x.rows || left <= 0) return;
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] *= kUnscale;
            P* p = (P*)x.p + m * x.cols + n;
            if constexpr (LAST == kOut) tile::store_some(p, left, v);
            else {
                float w[8];
                float* master = x.master + m * x.cols + n;
                if (x.master) tile::load_some((const float*)master, left, w);
                else tile::load_some((const P*)p, left, w);
#pragma unroll
                for (int q = 0; q < 8; ++q) w[q] -= decay * w[q] + size * v[q];
                if (x.master) tile::store_some(master, left, w);
                tile::store_some(p, left, w);
            }
        }
    });
}

// ---- launches --------------------------------------------------------------------------------
struct Batch {
    int64_t ws;                                   // bytes of workspace of its matrices
    int32_t piece0, pieces, tri0, tris, app0, apps;        // places of the three kinds, in the plan's lists
};
int pieces_of(const Matrix& m) { return (int)((m.rp() * m.cp() + kPiece - 1) / kPiece); }
int tris_of(const Matrix& m) {
    const int n = (int)((m.np() + kTile - 1) / kTile);
    return n * (n + 1) / 2;
}
int apps_of(const Matrix& m) { return (int)((m.rp() + kTile - 1) / kTile * ((m.cp() + kTile - 1) / kTile)); }

template <auto KERNEL, typename... A> ff_status go(int kind, uint32_t blocks, size_t lds, hipStream_t stream, const char* what, A... args) {
    Timed t(kind, stream);
    if (lds) tile::allow_lds<KERNEL>();
    hipLaunchKernelGGL(KERNEL, dim3(blocks), dim3(256), lds, stream, args...);
    return check_launch(what);
}

// All steps of one batch.  Tables for the three kinds of places differ in `places` (of a plan) or `each`.
struct Tables {
    Table piece, tri, app;
    uint32_t pieces, tris, apps;
};
template <typename G, typename P, int LAST> ff_status steps_of(const Tables& t, const StepArgs& a, int steps, const float* norm, double* partial, char* ws, hipStream_t stream) {
    constexpr bool MUON = LAST == kWeights;
    const char* what = MUON ? "ff_muon_step" : "ff_orthogonalise";
    ff_status st = go<k_muon_momentum<G, MUON>>(KK_MUON_MOMENTUM, t.pieces, 0, stream, what, t.piece, a, norm, partial);
    if (st == FF_OK) st = go<k_ns_start<G, MUON>>(KK_NS_START, t.pieces, 0, stream, what, t.piece, a, norm, (const double*)partial, ws);
    for (int s = 0; s < steps && st == FF_OK; ++s) {
        st = go<k_ns_gram>(KK_NS_GRAM, t.tris, kTileLds, stream, what, t.tri, ws, s & 1);
        if (st == FF_OK) st = go<k_ns_poly>(KK_NS_POLY, t.tris, kTileLds, stream, what, t.tri, ws, a.b, a.c);
        if (st != FF_OK) return st;
        if (s + 1 < steps) st = go<k_ns_apply<kMore, float>>(KK_NS_APPLY, t.apps, kTileLds, stream, what, t.app, ws, s & 1, a, norm);
        else st = go<k_ns_apply<LAST, P>>(KK_NS_APPLY, t.apps, kTileLds, stream, what, t.app, ws, s & 1, a, norm);
    }
    return st;
}

// ---- a plan: header, batches, matrices, places -------------------------------------------------
struct Header {
    uint32_t tag;
    int32_t matrices, batches, pieces, tris, apps;
    int64_t ws;                                   // the largest batch's
    int64_t bytes;                                // of the plan
    int64_t values;
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
struct Made {
    std::vector<Matrix> matrices;
    std::vector<Batch> batches;
    int64_t pieces = 0, tris = 0, apps = 0, ws = 0, values = 0;
};
// Matrices of much work first, so that small ones fill the end; a batch ends where its workspace would pass kBatch.
Made make(const ff_muon_desc& d, const ff_muon_tensor* ts) {
    Made r;
    for (int i = 0; i < d.n_tensors; ++i)
        if (ts[i].rows > 0 && ts[i].cols > 0) {
            r.matrices.push_back(matrix_from(ts[i]));
            r.values += (int64_t)ts[i].rows * ts[i].cols;
        }
    std::stable_sort(r.matrices.begin(), r.matrices.end(), [](const Matrix& a, const Matrix& b) { return std::max(a.rp(), a.cp()) > std::max(b.rp(), b.cp()); });
    Batch b{};
    auto close = [&] {
        if (b.pieces) r.batches.push_back(b);
        r.ws = std::max(r.ws, b.ws + (int64_t)align256((size_t)b.pieces * 8));
        r.pieces += b.pieces;
        r.tris += b.tris;
        r.apps += b.apps;
        b = Batch{};
        b.piece0 = (int32_t)r.pieces;
        b.tri0 = (int32_t)r.tris;
        b.app0 = (int32_t)r.apps;
    };
    for (Matrix& m : r.matrices) {
        if (b.pieces && b.ws + m.bytes() > kBatch) close();
        m.ws = b.ws;
        m.piece0 = b.pieces;
        b.ws += (int64_t)align256((size_t)m.bytes());
        b.pieces += m.pieces;
        b.tris += tris_of(m);
        b.apps += apps_of(m);
        if (r.pieces + b.pieces > INT32_MAX / 2 || r.apps + b.apps > INT32_MAX / 2 || r.tris + b.tris > INT32_MAX / 2) throw std::bad_alloc();
    }
    close();
    return r;
}
Header header_of(const ff_muon_desc& d, const Made& r) {
    Header h{};
    h.tag = tag_of(d);
    h.matrices = (int32_t)r.matrices.size();
    h.batches = (int32_t)r.batches.size();
    h.pieces = (int32_t)r.pieces;
    h.tris = (int32_t)r.tris;
    h.apps = (int32_t)r.apps;
    h.ws = std::max<int64_t>(r.ws, 256);
    h.values = r.values;
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
        if (!r.matrices.empty()) {
            memcpy(out + l.batches, r.batches.data(), sizeof(Batch) * r.batches.size());
            memcpy(out + l.matrices, r.matrices.data(), sizeof(Matrix) * r.matrices.size());
        }
        Place *piece = (Place*)(out + l.piece), *tri = (Place*)(out + l.tri), *app = (Place*)(out + l.app);
        for (int32_t i = 0; i < h.matrices; ++i) {
            const Matrix& m = r.matrices[i];
            for (int32_t k = 0; k < m.pieces; ++k) *piece++ = {i, k};
            for (int32_t k = 0; k < tris_of(m); ++k) *tri++ = {i, k};
            for (int32_t k = 0; k < apps_of(m); ++k) *app++ = {i, k};
        }
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

ff_status muon_step_run(const ff_muon_desc& d, const void* plan_host, const void* plan, const ff_muon_hyper& h, const float* norm, void* ws, hipStream_t stream) {
    const Header& head = *(const Header*)plan_host;
    const Layout l = layout_of(head);
    const StepArgs a{(float)h.lr, (float)h.beta, (float)(1. - h.beta), norm ? (float)h.max_norm : 0.f, h.eps, (float)h.a, (float)h.b, (float)h.c, h.nesterov, h.scale == FF_MUON_RMS};
    const char* dev = (const char*)plan;
    for (int i = 0; i < head.batches; ++i) {
        const Batch& b = ((const Batch*)((const char*)plan_host + l.batches))[i];
        Table t{};
        t.matrices = (const Matrix*)(dev + l.matrices);
        Tables ts{t, t, t, (uint32_t)b.pieces, (uint32_t)b.tris, (uint32_t)b.apps};
        ts.piece.places = (const Place*)(dev + l.piece) + b.piece0;
        ts.tri.places = (const Place*)(dev + l.tri) + b.tri0;
        ts.app.places = (const Place*)(dev + l.app) + b.app0;
        double* partial = (double*)((char*)ws + b.ws);
        ff_status st;
        if (d.param_dtype == FF_F32) {
            st = d.grad_dtype == FF_F32 ? steps_of<float, float, kWeights>(ts, a, h.steps, norm, partial, (char*)ws, stream)
                                        : steps_of<bf16_t, float, kWeights>(ts, a, h.steps, norm, partial, (char*)ws, stream);
        } else {
            st = d.grad_dtype == FF_F32 ? steps_of<float, bf16_t, kWeights>(ts, a, h.steps, norm, partial, (char*)ws, stream)
                                        : steps_of<bf16_t, bf16_t, kWeights>(ts, a, h.steps, norm, partial, (char*)ws, stream);
        }
        if (st != FF_OK) return st;
    }
    return FF_OK;
}

// ---- matrices of one shape -------------------------------------------------------------------
namespace {
struct Uniform {
    Matrix one;
    int64_t bytes;             // of workspace a matrix
    int32_t group;             // matrices worked on together
};
Uniform uniform_of(const ff_orthogonalise_desc& d) {
    Uniform u{};
    u.one.rows = d.rows;
    u.one.cols = d.cols;
    u.one.pieces = pieces_of(u.one);
    u.bytes = (int64_t)align256((size_t)u.one.bytes());
    u.group = (int32_t)std::max<int64_t>(1, std::min<int64_t>(d.count, kBatch / u.bytes));
    return u;
}
}  // namespace
size_t orthogonalise_workspace(const ff_orthogonalise_desc& d) {
    const Uniform u = uniform_of(d);
    return (size_t)u.bytes * u.group + align256((size_t)u.group * u.one.pieces * 8);
}
ff_status orthogonalise_run(const ff_orthogonalise_desc& d, const void* x, void* out, void* ws, hipStream_t stream) {
    const Uniform u = uniform_of(d);
    StepArgs a{};
    a.eps = d.eps;
    a.a = (float)d.a;
    a.b = (float)d.b;
    a.c = (float)d.c;
    const int64_t step = (int64_t)d.rows * d.cols * (d.dtype == FF_F32 ? 4 : 2);
    for (int32_t i = 0; i < d.count; i += u.group) {
        const int32_t n = std::min(u.group, d.count - i);
        Table t{};
        t.one = u.one;
        t.one.g = (const char*)x + i * step;
        t.one.p = (char*)out + i * step;
        t.in_step = t.out_step = step;
        t.ws_step = u.bytes;
        Tables ts{t, t, t, (uint32_t)(n * u.one.pieces), (uint32_t)(n * tris_of(u.one)), (uint32_t)(n * apps_of(u.one))};
        ts.piece.each = u.one.pieces;
        ts.tri.each = tris_of(u.one);
        ts.app.each = apps_of(u.one);
        double* partial = (double*)((char*)ws + u.bytes * u.group);
        const ff_status st = d.dtype == FF_F32 ? steps_of<float, float, kOut>(ts, a, d.steps, nullptr, partial, (char*)ws, stream)
                                               : steps_of<bf16_t, bf16_t, kOut>(ts, a, d.steps, nullptr, partial, (char*)ws, stream);
        if (st != FF_OK) return st;
    }
    return FF_OK;
}

}  // namespace ff
