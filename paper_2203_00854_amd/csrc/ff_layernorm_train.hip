// Layer norm in training: forward pass with residual sum and statistics, backward pass with the gradients of gamma and beta.
//
// Both passes are bound by HBM (a dozen to two dozen vector instructions per value, where 45 lane-instructions fit into the time that six bytes
// take), so a row is read once, stays in registers, and is written once.  A team of 8 to 64 lanes of one wavefront holds a row, each
// lane up to four pieces of 16 bytes; rows of more than 256 pieces are held by a whole block.  Rows that are no whole number of pieces, and tensors at any
// offset, take the same path: pieces are loaded at the alignment of their type, and a last piece that
// would pass the row's end is moved back to end with it - its first values, which the piece before holds too, count in no sum.
#include <type_traits>

#include "ff_common.h"

namespace ff {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// a piece: V values at the alignment of one
template <typename T, int V> struct __attribute__((packed, aligned(sizeof(T)))) Pack {
    T x[V];
};
template <typename T, int V> __device__ __forceinline__ void widen(const Pack<T, V>& p, float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = to_f32<T>(p.x[i]);
}
template <typename T, int V> __device__ __forceinline__ Pack<T, V> narrow(const float (&v)[V]) {
    Pack<T, V> p;
    if constexpr (sizeof(T) == 2 && V % 2 == 0) {      // two at a time: one conversion instruction
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            const uint32_t two = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{v[i], v[i + 1]}), bf16x2));
            p.x[i] = (bf16_t)two;
            p.x[i + 1] = (bf16_t)(two >> 16);
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) p.x[i] = from_f32<T>(v[i]);
    }
    return p;
}

// ---- sums over a team ----------------------------------------------------------------------
__device__ __forceinline__ float swap16_sum(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// over the lane's team of 8, 16, 32 or 64 lanes
__device__ __forceinline__ float team_sum(float v, int lanes) {
    v = sum8(v);
    if (lanes > 8) v += dpp<kDppRor8>(v);
    if (lanes > 16) v = swap16_sum(v);
    if (lanes > 32) v = half_sum(v);
    return v;
}
// over the lanes at the same place of the wavefront's teams
__device__ __forceinline__ float across_teams(float v, int lanes) {
    if (lanes <= 8) v += dpp<kDppRor8>(v);
    if (lanes <= 16) v = swap16_sum(v);
    if (lanes <= 32) v = half_sum(v);
    return v;
}

constexpr int kForwardThreads = 256, kBackwardThreads = 512, kWideThreads = 512;

// Who works on a row: lanes of a wavefront, or (WIDE) a whole block, whose sums pass through LDS.
template <bool WIDE> struct Team {
    int lanes, place;              // members, own number among them
    float* part;                   // WIDE: a word for each wavefront, twice (sums of two successive calls do not meet)
    int turn = 0;
    __device__ __forceinline__ float sum(float v) {
        if constexpr (!WIDE) {
            return team_sum(v, lanes);
        } else {
            v = wave_sum(v);
            float* p = part + turn;
            turn ^= kWideThreads / 64;
            if ((threadIdx.x & 63) == 0) p[threadIdx.x >> 6] = v;
            __syncthreads();
            float s = (p[0] + p[1]) + (p[2] + p[3]);
            if (lanes > 256) s += (p[4] + p[5]) + (p[6] + p[7]);
            return s;
        }
    }
};

// The pieces of a row that a lane holds: ITERS of them, `lanes` pieces apart.
template <int V, int ITERS, bool RAGGED> struct Held {
    int at[ITERS];                 // first channel
    int skip[ITERS];               // values at its front that another piece holds
    bool has[ITERS];
    __device__ __forceinline__ Held(int place, int lanes, int c) {
        const int pieces = (c + V - 1) / V;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int p = place + it * lanes;
            has[it] = p < pieces;
            const int from = p * V;
            at[it] = RAGGED && has[it] && from > c - V ? c - V : from;
            skip[it] = RAGGED ? from - at[it] : 0;
        }
    }
    __device__ __forceinline__ bool counts(int it, int i) const { return !RAGGED || i >= skip[it]; }
};

template <typename T, int V, int ITERS, bool RAGGED, bool WIDE>
__global__ __launch_bounds__(WIDE ? kWideThreads : kForwardThreads) void k_ln_forward(
    const T* x, const T* residual, const T* __restrict__ gamma, const T* __restrict__ beta, T* sum, T* __restrict__ y,
    float* __restrict__ mean_out, float* __restrict__ rstd_out, int64_t rows, int c, int lanes, float eps) {
    __shared__ float part[WIDE ? 2 * kWideThreads / 64 : 1];
    typedef Pack<T, V> Pc;
    Team<WIDE> team{lanes, WIDE ? (int)threadIdx.x : (int)threadIdx.x & (lanes - 1), part};
    const Held<V, ITERS, RAGGED> held(team.place, team.lanes, c);
    float gm[ITERS][V] = {}, bt[ITERS][V] = {};
#pragma unroll
    for (int it = 0; it < ITERS; ++it)
        if (held.has[it]) {
            widen<T, V>(*(const Pc*)(gamma + held.at[it]), gm[it]);
            widen<T, V>(*(const Pc*)(beta + held.at[it]), bt[it]);
        }
    const float inv_c = 1.f / (float)c;
    const int per_block = WIDE ? 1 : (int)blockDim.x / lanes;
    const int64_t stride = (int64_t)gridDim.x * per_block;
    for (int64_t row = (int64_t)blockIdx.x * per_block + (WIDE ? 0 : threadIdx.x / lanes); row < rows; row += stride) {
        const int64_t base = row * c;
        float v[ITERS][V];
        Pc kept[ITERS];
        float s = 0.f;
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
            if (held.has[it]) kept[it] = *(const Pc*)(x + base + held.at[it]);
        if (residual) {
#pragma unroll
            for (int it = 0; it < ITERS; ++it)
                if (held.has[it]) {
                    float r[V];
                    widen<T, V>(*(const Pc*)(residual + base + held.at[it]), r);
                    widen<T, V>(kept[it], v[it]);
#pragma unroll
                    for (int i = 0; i < V; ++i) r[i] += v[it][i];
                    kept[it] = narrow<T, V>(r);
                }
        }
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
            if (held.has[it]) {
                widen<T, V>(kept[it], v[it]);
#pragma unroll
                for (int i = 0; i < V; ++i) s += held.counts(it, i) ? v[it][i] : 0.f;
            }
        const float mean = team.sum(s) * inv_c;
        float q = 0.f;
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
            if (held.has[it]) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    v[it][i] -= mean;
                    q += held.counts(it, i) ? v[it][i] * v[it][i] : 0.f;
                }
            }
        const float rstd = 1.f / sqrtf(team.sum(q) * inv_c + eps);
        if (mean_out && team.place == 0) {
            mean_out[row] = mean;
            rstd_out[row] = rstd;
        }
        // (the sum may lie where x or the residual was: every value of the row has been read when its statistics are known)
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
            if (held.has[it]) {
                if (residual) *(Pc*)(sum + base + held.at[it]) = kept[it];
                float o[V];
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] = v[it][i] * rstd * gm[it][i] + bt[it][i];
                *(Pc*)(y + base + held.at[it]) = narrow<T, V>(o);
            }
    }
}

// A block goes through its rows with the sums of dgamma and dbeta in registers (a lane's channels are the same in every row), joins them
// over its teams and wavefronts in a fixed order and leaves 2 c partial sums; with one block in all these are the result.
template <typename T, int V, int ITERS, bool RAGGED, bool WIDE>
__global__ __launch_bounds__(WIDE ? kWideThreads : kBackwardThreads) void k_ln_backward(
    const T* __restrict__ s, const T* __restrict__ gamma, const float* __restrict__ mean_in, const float* __restrict__ rstd_in, const T* dy,
    const T* dsum, T* dx, float* __restrict__ partial, float* __restrict__ dgamma, float* __restrict__ dbeta, bool accumulate, int64_t rows,
    int c, int lanes, float eps) {
    extern __shared__ float joined[];                  // every wavefront's sums of dgamma and dbeta; WIDE: what Team needs
    typedef Pack<T, V> Pc;
    Team<WIDE> team{lanes, WIDE ? (int)threadIdx.x : (int)threadIdx.x & (lanes - 1), joined};
    const Held<V, ITERS, RAGGED> held(team.place, team.lanes, c);
    float gm[ITERS][V] = {}, dg[ITERS][V] = {}, db[ITERS][V] = {};
#pragma unroll
    for (int it = 0; it < ITERS; ++it)
        if (held.has[it]) widen<T, V>(*(const Pc*)(gamma + held.at[it]), gm[it]);
    const float inv_c = 1.f / (float)c;
    const int per_block = WIDE ? 1 : (int)blockDim.x / lanes;
    const int64_t stride = (int64_t)gridDim.x * per_block;
    for (int64_t row = (int64_t)blockIdx.x * per_block + (WIDE ? 0 : threadIdx.x / lanes); row < rows; row += stride) {
        const int64_t base = row * c;
        float u[ITERS][V] = {}, d[ITERS][V] = {};
        Pc pu[ITERS], pd[ITERS], ps[ITERS];
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
            if (held.has[it]) {
                pu[it] = *(const Pc*)(s + base + held.at[it]);
                pd[it] = *(const Pc*)(dy + base + held.at[it]);
            }
        if (dsum) {
#pragma unroll
            for (int it = 0; it < ITERS; ++it)
                if (held.has[it]) ps[it] = *(const Pc*)(dsum + base + held.at[it]);
        }
        float t = 0.f;
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
            if (held.has[it]) {
                widen<T, V>(pu[it], u[it]);
                widen<T, V>(pd[it], d[it]);
            }
        float mean, rstd;
        if (mean_in) {
            mean = mean_in[row];
            rstd = rstd_in[row];
        } else {
#pragma unroll
            for (int it = 0; it < ITERS; ++it)
                if (held.has[it]) {
#pragma unroll
                    for (int i = 0; i < V; ++i) t += held.counts(it, i) ? u[it][i] : 0.f;
                }
            mean = team.sum(t) * inv_c;
            float q = 0.f;
#pragma unroll
            for (int it = 0; it < ITERS; ++it)
                if (held.has[it]) {
#pragma unroll
                    for (int i = 0; i < V; ++i) q += held.counts(it, i) ? (u[it][i] - mean) * (u[it][i] - mean) : 0.f;
                }
            rstd = 1.f / sqrtf(team.sum(q) * inv_c + eps);
        }
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
            if (held.has[it]) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    u[it][i] = (u[it][i] - mean) * rstd;
                    const float e = d[it][i];
                    d[it][i] *= gm[it][i];
                    if (held.counts(it, i)) {
                        dg[it][i] += e * u[it][i];
                        db[it][i] += e;
                        a += d[it][i];
                        b += d[it][i] * u[it][i];
                    }
                }
            }
        a = team.sum(a) * inv_c;
        b = team.sum(b) * inv_c;
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
            if (held.has[it]) {
                float o[V];
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] = rstd * (d[it][i] - a - u[it][i] * b);
                if (dsum) {
                    float r[V];
                    widen<T, V>(ps[it], r);
#pragma unroll
                    for (int i = 0; i < V; ++i) o[i] += r[i];
                }
                *(Pc*)(dx + base + held.at[it]) = narrow<T, V>(o);
            }
    }
    const bool alone = gridDim.x == 1;
    float* out = partial + (size_t)blockIdx.x * 2 * c;
    auto leave = [&](int i, float v) {                 // partial sum number i of 2 c
        if (alone) {
            float* to = i < c ? dgamma + i : dbeta + i - c;
            *to = accumulate ? *to + v : v;
        } else {
            out[i] = v;
        }
    };
    if constexpr (WIDE) {
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
            if (held.has[it])
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (held.counts(it, i)) {
                        leave(held.at[it] + i, dg[it][i]);
                        leave(c + held.at[it] + i, db[it][i]);
                    }
    } else {
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                dg[it][i] = across_teams(dg[it][i], lanes);
                db[it][i] = across_teams(db[it][i], lanes);
            }
        // each wavefront's sums by (kind, piece, value, lane), then a thread adds up a channel's over the wavefronts
        const int wave = threadIdx.x >> 6, slots = ITERS * V * lanes;
        if ((int)(threadIdx.x & 63) < lanes) {
            float* to = joined + wave * 2 * slots + team.place;
#pragma unroll
            for (int it = 0; it < ITERS; ++it)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    to[(it * V + i) * lanes] = dg[it][i];
                    to[slots + (it * V + i) * lanes] = db[it][i];
                }
        }
        __syncthreads();
        const int last = (c + V - 1) / V - 1;
        for (int ch = threadIdx.x; ch < c; ch += kBackwardThreads) {
            const int p = ch / V, i = RAGGED && p == last ? ch - (c - V) : ch % V;
            const float* from = joined + (p / lanes * V + i) * lanes + (p & (lanes - 1));
            float g = 0.f, b = 0.f;
#pragma unroll
            for (int w = 0; w < kBackwardThreads / 64; ++w) {
                g += from[w * 2 * slots];
                b += from[w * 2 * slots + slots];
            }
            leave(ch, g);
            leave(c + ch, b);
        }
    }
}

// dgamma and dbeta from the blocks' partial sums: a block takes 64 of the 2 c columns, its sixteen wavefronts every sixteenth of the partial sums each
__global__ __launch_bounds__(1024) void k_ln_join(const float* __restrict__ partial, int blocks, int c, bool accumulate,
                                                  float* __restrict__ dgamma, float* __restrict__ dbeta) {
    __shared__ float part[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = blockIdx.x * 64 + lane;
    float sum = 0.f;
    if (i < 2 * c) {
#pragma unroll 8
        for (int b = wave; b < blocks; b += 16) sum += partial[(size_t)b * 2 * c + i];
    }
    part[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || i >= 2 * c) return;
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) sum += part[w][lane];
    float* to = i < c ? dgamma + i : dbeta + i - c;
    *to = accumulate ? *to + sum : sum;
}

// ---- which kernel takes a shape ------------------------------------------------------------
// Pieces are 16 bytes (one value where the row is shorter).  A lane holds at most sixteen values: with the sums of dgamma and dbeta beside them
// more would leave two wavefronts per SIMD, or spill.  Of the ways to cover a row by lanes times pieces the one with the
// fewest idle places is taken, of equals the one with the most lanes; rows of more than 64 such lanes are a block's, of 256 threads or, beyond 512 pieces, of 512.
struct Shape {
    int v, iters, lanes;
    bool ragged, wide;
};
static Shape shape_of(int dtype, int c) {
    Shape s{dtype == FF_F32 ? 4 : 8, 1, 8, false, false};
    if (c < s.v) s.v = 1;
    const int pieces = (c + s.v - 1) / s.v;
    s.ragged = c % s.v != 0;
    const int most = s.v == 8 ? 2 : 4;
    if (pieces > 64 * most) {
        s.wide = true;
        s.lanes = pieces > 512 ? kWideThreads : 256;
        s.iters = (pieces + s.lanes - 1) / s.lanes;
        return s;
    }
    int best = 1 << 30;
    for (int lanes = 64; lanes >= 8; lanes >>= 1) {
        const int iters = (pieces + lanes - 1) / lanes;
        if (iters > most || iters * lanes >= best) continue;
        best = iters * lanes;
        s.iters = iters;
        s.lanes = lanes;
    }
    return s;
}

template <typename F> static void with_shape(const Shape& s, F go) {
    auto it = [&](auto v, auto ragged) {
        constexpr int V = decltype(v)::value;
        constexpr bool R = decltype(ragged)::value;
        auto at = [&](auto wide) {
            if (s.iters == 1) go(v, std::integral_constant<int, 1>{}, std::bool_constant<R>{}, wide);
            else if (s.iters == 2) go(v, std::integral_constant<int, 2>{}, std::bool_constant<R>{}, wide);
            else if constexpr (V == 4) {
                if (s.iters == 3) go(v, std::integral_constant<int, 3>{}, std::bool_constant<R>{}, wide);
                else go(v, std::integral_constant<int, 4>{}, std::bool_constant<R>{}, wide);
            }
        };
        if (s.wide) at(std::true_type{});
        else at(std::false_type{});
    };
    auto full = [&](auto v) {
        if (s.ragged) it(v, std::true_type{});
        else it(v, std::false_type{});
    };
    if (s.v == 8) full(std::integral_constant<int, 8>{});
    else if (s.v == 4) full(std::integral_constant<int, 4>{});
    else go(std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{}, std::false_type{}, std::false_type{});
}

static int64_t turns_of(int64_t rows, int per_block) { return (rows + per_block - 1) / per_block; }

template <typename T>
static void forward_t(const ff_norm_desc& d, const void* x, const void* residual, const void* gamma, const void* beta, void* sum, void* y,
                      float* mean, float* rstd, hipStream_t stream) {
    const Shape s = shape_of(d.dtype, d.c);
    with_shape(s, [&](auto v, auto iters, auto ragged, auto wide) {
        constexpr int V = decltype(v)::value, I = decltype(iters)::value;
        constexpr bool R = decltype(ragged)::value, W = decltype(wide)::value;
        if constexpr (V != (sizeof(T) == 4 ? 8 : 4)) {
            const int threads = W ? s.lanes : kForwardThreads;
            int64_t blocks = turns_of(d.rows, W ? 1 : threads / s.lanes);
            const int64_t cap = (int64_t)compute_units() * (W ? 4 : 16);
            if (blocks > cap) blocks = cap;
            hipLaunchKernelGGL((k_ln_forward<T, V, I, R, W>), dim3((unsigned)blocks), dim3(threads), 0, stream, (const T*)x, (const T*)residual,
                               (const T*)gamma, (const T*)beta, (T*)sum, (T*)y, mean, rstd, d.rows, d.c, s.lanes, d.ln_eps);
        }
    });
}

ff_status layernorm_forward_run(const ff_norm_desc& d, const void* x, const void* residual, const void* gamma, const void* beta, void* sum,
                                void* y, float* mean, float* rstd, hipStream_t stream) {
    Timed t(KK_LN_FORWARD, stream);
    if (d.dtype == FF_F32) forward_t<float>(d, x, residual, gamma, beta, sum, y, mean, rstd, stream);
    else forward_t<bf16_t>(d, x, residual, gamma, beta, sum, y, mean, rstd, stream);
    return check_launch("ff_layernorm_forward");
}

// Blocks of the backward pass.  A number of its own, not the device's, so that the order of the sums does not depend on the machine.
constexpr int kBackwardBlocks = 512;
static int backward_blocks(const ff_norm_desc& d, const Shape& s) {
    const int64_t turns = turns_of(d.rows, s.wide ? 1 : kBackwardThreads / s.lanes);
    if (turns <= 4) return turns > 0;                  // one block: no partial sums, no second launch
    return (int)(turns < kBackwardBlocks ? turns : kBackwardBlocks);
}

size_t layernorm_backward_workspace(const ff_norm_desc& d) {
    const size_t n = (size_t)backward_blocks(d, shape_of(d.dtype, d.c)) * 2 * d.c * sizeof(float);
    return n < 256 ? 256 : (n + 255) & ~(size_t)255;
}

template <typename T>
static void backward_t(const ff_norm_desc& d, const Shape& s, int blocks, const void* src, const void* gamma, const float* mean, const float* rstd, const void* dy,
                       const void* dsum, void* dx, float* dgamma, float* dbeta, bool accumulate, float* partial, hipStream_t stream) {
    with_shape(s, [&](auto v, auto iters, auto ragged, auto wide) {
        constexpr int V = decltype(v)::value, I = decltype(iters)::value;
        constexpr bool R = decltype(ragged)::value, W = decltype(wide)::value;
        if constexpr (V != (sizeof(T) == 4 ? 8 : 4)) {
            const size_t lds = W ? 2 * kWideThreads / 64 * sizeof(float) : (size_t)kBackwardThreads / 64 * 2 * I * V * s.lanes * sizeof(float);     // at most 64 KiB
            hipLaunchKernelGGL((k_ln_backward<T, V, I, R, W>), dim3(blocks), dim3(W ? s.lanes : kBackwardThreads), lds, stream, (const T*)src,
                               (const T*)gamma, mean, rstd, (const T*)dy, (const T*)dsum, (T*)dx, partial, dgamma, dbeta, accumulate, d.rows, d.c,
                               s.lanes, d.ln_eps);
        }
    });
}

ff_status layernorm_backward_run(const ff_norm_desc& d, const void* s, const void* gamma, const float* mean, const float* rstd,
                                 const void* dy, const void* dsum, void* dx, float* dgamma, float* dbeta, bool accumulate, void* ws,
                                 hipStream_t stream) {
    const Shape shape = shape_of(d.dtype, d.c);
    const int blocks = backward_blocks(d, shape);
    if (blocks > 0) {
        Timed t(KK_LN_BACKWARD, stream);
        if (d.dtype == FF_F32) backward_t<float>(d, shape, blocks, s, gamma, mean, rstd, dy, dsum, dx, dgamma, dbeta, accumulate, (float*)ws, stream);
        else backward_t<bf16_t>(d, shape, blocks, s, gamma, mean, rstd, dy, dsum, dx, dgamma, dbeta, accumulate, (float*)ws, stream);
    }
    if (blocks != 1) {
        Timed t(KK_LN_JOIN, stream);
        hipLaunchKernelGGL(k_ln_join, dim3((2 * d.c + 63) / 64), dim3(1024), 0, stream, (const float*)ws, blocks, d.c, accumulate, dgamma, dbeta);
    }
    return check_launch("ff_layernorm_backward");
}

}  // namespace ff
