// Layer norm in training: forward pass with residual sum and statistics, backward pass with the gradients of gamma and beta.
//
// Both passes are bound by HBM (a dozen to two dozen vector instructions per value, where 45 lane-instructions fit into the time that six bytes
// take), so a row is read once, stays in registers, and is written once.  A team of 1 to 64 lanes of one wavefront holds a row, each
// lane up to sixteen values in pieces of 16 bytes; rows of more than 1024 channels are held by a whole block.  Rows that are no whole number of pieces, and tensors at any
// offset, take the same path: pieces are loaded at the alignment of their type, and a piece that
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

// A piece of a row; STREAMED: past the caches.
template <bool STREAMED, typename T, int V> __device__ __forceinline__ Pack<T, V> fetch(const T* p) {
    if constexpr (STREAMED) {
        typedef uint32_t words __attribute__((ext_vector_type(4), aligned(2)));
        static_assert(sizeof(Pack<T, V>) == sizeof(words), "whole pieces only");
        return __builtin_bit_cast(Pack<T, V>, __builtin_nontemporal_load((const words*)p));
    } else {
        return *(const Pack<T, V>*)p;
    }
}

// ---- sums over a team ----------------------------------------------------------------------
__device__ __forceinline__ float swap16_sum(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// over the lane's team of 1, 2, 4, .. 64 lanes, of several values at once
template <typename... F> __device__ __forceinline__ void team_sum(int lanes, F&... v) {
    if (lanes > 4) {
        ((v = sum8(v)), ...);
        if (lanes > 8) ((v += dpp<kDppRor8>(v)), ...);
        if (lanes > 16) ((v = swap16_sum(v)), ...);
        if (lanes > 32) ((v = half_sum(v)), ...);
    } else {
        if (lanes > 1) ((v += dpp<kDppXor1>(v)), ...);
        if (lanes > 2) ((v += dpp<kDppXor2>(v)), ...);
    }
}
// over the lanes at the same place of the wavefront's teams (rotations of sixteen lanes: together they visit all of a row's teams), of two tables at once
template <int N, int M> __device__ __forceinline__ void across_teams(int lanes, float (&v)[N][M], float (&w)[N][M]) {
    constexpr int kRor4 = 0x124, kRor2 = 0x122, kRor1 = 0x121;
    auto each = [&](auto f) {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int m = 0; m < M; ++m) {
                v[n][m] = f(v[n][m]);
                w[n][m] = f(w[n][m]);
            }
    };
    if (lanes <= 8) each([](float x) { return x + dpp<kDppRor8>(x); });
    if (lanes <= 4) each([](float x) { return x + dpp<kRor4>(x); });
    if (lanes <= 2) each([](float x) { return x + dpp<kRor2>(x); });
    if (lanes <= 1) each([](float x) { return x + dpp<kRor1>(x); });
    if (lanes <= 16) each([](float x) { return swap16_sum(x); });
    if (lanes <= 32) each([](float x) { return half_sum(x); });
}

constexpr int kForwardThreads = 256, kWideThreads = 512;
// Threads of a backward block whose rows are held by lanes: as many as leave a lane the registers for its values (eight take 82, sixteen 150).
constexpr int backward_threads(int values) { return values <= 8 ? 1024 : 512; }

// Who works on a row: lanes of a wavefront, or (WIDE) a whole block, whose sums pass through LDS.
template <bool WIDE> struct Team {
    int lanes, place;              // members, own number among them
    float* part;                   // WIDE: two words for each of kWideThreads / 64 wavefronts, twice (sums of two successive calls do not meet)
    int turn = 0;
    __device__ __forceinline__ Team(int lanes_, float* part_) : lanes(lanes_), place(WIDE ? (int)threadIdx.x : (int)threadIdx.x & (lanes_ - 1)), part(part_) {
        if constexpr (WIDE) {
            if (threadIdx.x < 4 * kWideThreads / 64) part[threadIdx.x] = 0.f;
            __syncthreads();
        }
    }
    __device__ __forceinline__ float sum(float v) {
        if constexpr (WIDE) {
            float none = 0.f;
            sum(v, none);
        } else {
            team_sum(lanes, v);
        }
        return v;
    }
    // of two at once
    __device__ __forceinline__ void sum(float& v, float& w) {
        if constexpr (!WIDE) {
            team_sum(lanes, v, w);
        } else {
            constexpr int W = kWideThreads / 64;
            float* p = part + turn;
            turn ^= 2 * W;
            v = wave_sum(v);
            w = wave_sum(w);
            if ((threadIdx.x & 63) == 0) {
                p[threadIdx.x >> 6] = v;
                p[W + (threadIdx.x >> 6)] = w;
            }
            __syncthreads();
            v = w = 0.f;
#pragma unroll
            for (int i = 0; i < W; ++i) {              // (the words of wavefronts that a smaller block lacks are zero)
                v += p[i];
                w += p[W + i];
            }
        }
    }
};

// The pieces of a row that a lane holds: ITERS of them, `lanes` pieces apart.  Where the team's places are more than the row
// (MASKED), a piece past the end is moved back to end with the row: all lanes load and compute alike, without branches, and only
// values that no other place holds count in sums over the row.
template <int V, int ITERS, bool MASKED> struct Held {
    int at[ITERS];                 // first channel
    int skip[ITERS];               // values at its front that another place holds; V or more: all of them
    __device__ __forceinline__ Held(int place, int lanes, int c) {
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int from = (place + it * lanes) * V;
            at[it] = MASKED && from > c - V ? c - V : from;
            skip[it] = MASKED ? from - at[it] : 0;
        }
    }
    __device__ __forceinline__ float counted(int it, int i, float v) const { return !MASKED || i >= skip[it] ? v : 0.f; }
    __device__ __forceinline__ bool stores(int it) const { return !MASKED || skip[it] < V; }
};

// Two sums over a team, the second of squared distances from the mean that the first gives (in registers: no second reading, no cancellation).
// 128 x 256 x 256 bfloat16 with the residual sum 12.2 us, 2048 x 2048 x 128 368 us (5.9 TB/s).
template <typename T, int V, int ITERS, bool MASKED, bool WIDE, bool STREAMED>
__global__ __launch_bounds__(WIDE ? kWideThreads : kForwardThreads) void k_ln_forward(
    const T* x, const T* residual, const T* __restrict__ gamma, const T* __restrict__ beta, T* sum, T* __restrict__ y,
    float* __restrict__ mean_out, float* __restrict__ rstd_out, int64_t rows, int c, int lanes, int turns, float eps) {
    __shared__ float part[WIDE ? 4 * kWideThreads / 64 : 1];
    typedef Pack<T, V> Pc;
    Team<WIDE> team(lanes, part);
    const Held<V, ITERS, MASKED> held(team.place, team.lanes, c);
    Pc gm[ITERS], bt[ITERS];
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        gm[it] = *(const Pc*)(gamma + held.at[it]);
        bt[it] = *(const Pc*)(beta + held.at[it]);
    }
    const float inv_c = 1.f / (float)c;
    const int per_block = WIDE ? 1 : (int)blockDim.x / lanes;
    const int64_t first = (int64_t)blockIdx.x * per_block * turns;
    const int64_t end = first + (int64_t)per_block * turns < rows ? first + (int64_t)per_block * turns : rows;
    for (int64_t row = first + (WIDE ? 0 : threadIdx.x / lanes); row < end; row += per_block) {
        const int64_t base = row * c;
        float v[ITERS][V];
        Pc kept[ITERS];
        float s = 0.f;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) kept[it] = fetch<STREAMED, T, V>(x + base + held.at[it]);
        if (residual) {
            Pc more[ITERS];
#pragma unroll
            for (int it = 0; it < ITERS; ++it) more[it] = fetch<STREAMED, T, V>(residual + base + held.at[it]);
#pragma unroll
            for (int it = 0; it < ITERS; ++it) {
                float r[V];
                widen<T, V>(more[it], r);
                widen<T, V>(kept[it], v[it]);
#pragma unroll
                for (int i = 0; i < V; ++i) r[i] += v[it][i];
                kept[it] = narrow<T, V>(r);
            }
        }
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            widen<T, V>(kept[it], v[it]);
#pragma unroll
            for (int i = 0; i < V; ++i) s += held.counted(it, i, v[it][i]);
        }
        const float mean = team.sum(s) * inv_c;
        float q = 0.f;
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                v[it][i] -= mean;
                q += held.counted(it, i, v[it][i] * v[it][i]);
            }
        const float rstd = 1.f / sqrtf(team.sum(q) * inv_c + eps);
        if (mean_out && team.place == 0) {
            mean_out[row] = mean;
            rstd_out[row] = rstd;
        }
        // (the sum may lie where x or the residual was: every value of the row has been read when its statistics are known)
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            float o[V], g[V], b[V];
            widen<T, V>(gm[it], g);
            widen<T, V>(bt[it], b);
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = v[it][i] * rstd * g[i] + b[i];
            if (held.stores(it)) {
                if (residual) *(Pc*)(sum + base + held.at[it]) = kept[it];
                *(Pc*)(y + base + held.at[it]) = narrow<T, V>(o);
            }
        }
    }
}

// Bytes bound it: 2048 x 2048 x 128 bfloat16 in 572 us (5.6 TB/s), 610 where the statistics are formed again (four sums over a team one after
// the other, not two); 5120 x 384 x 64 in 130 (5.8 TB/s), 128 x 256 x 256 with dsum in 14.7.  Sixteen wavefronts on a compute unit carry that: twice as many,
// in registers or blocks, took longer (662), and each block more makes the second launch longer.
// A block goes through its rows with the sums of dgamma and dbeta in registers (a lane's channels are the same in every row), joins them
// over its teams and, in float64, its wavefronts in a fixed order and leaves 2 c float32 partial sums; with one block in all these are the result.
// AHEAD: the next row is on its way while this one is worked on.
template <typename T, int V, int ITERS, bool MASKED, bool WIDE, bool STREAMED, bool AHEAD>
__global__ __launch_bounds__(WIDE ? kWideThreads : backward_threads(V * ITERS)) void k_ln_backward(
    const T* __restrict__ s, const T* __restrict__ gamma, const float* __restrict__ mean_in, const float* __restrict__ rstd_in, const T* dy,
    const T* dsum, T* dx, float* __restrict__ partial, float* __restrict__ dgamma, float* __restrict__ dbeta, bool accumulate, int64_t rows,
    int c, int lanes, float eps) {
    constexpr int THREADS = backward_threads(V * ITERS);
    extern __shared__ float joined[];                  // every wavefront's sums of dgamma and dbeta; WIDE: what Team needs
    typedef Pack<T, V> Pc;
    Team<WIDE> team(lanes, joined);
    const Held<V, ITERS, MASKED> held(team.place, team.lanes, c);
    float dg[ITERS][V] = {}, db[ITERS][V] = {};
    Pc gm[ITERS];
#pragma unroll
    for (int it = 0; it < ITERS; ++it) gm[it] = *(const Pc*)(gamma + held.at[it]);
    const float inv_c = 1.f / (float)c;
    const int per_block = WIDE ? 1 : (int)blockDim.x / lanes;
    const int64_t stride = (int64_t)gridDim.x * per_block;
    int64_t row = (int64_t)blockIdx.x * per_block + (WIDE ? 0 : threadIdx.x / lanes);
    Pc pu[ITERS], pd[ITERS], ps[ITERS];
    [[maybe_unused]] Pc nu[ITERS], nd[ITERS], ns[ITERS];
    auto load = [&](Pc(&x)[ITERS], Pc(&y)[ITERS], Pc(&z)[ITERS], int64_t base) {
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            x[it] = fetch<STREAMED, T, V>(s + base + held.at[it]);
            y[it] = fetch<STREAMED, T, V>(dy + base + held.at[it]);
        }
        if (dsum) {
#pragma unroll
            for (int it = 0; it < ITERS; ++it) z[it] = fetch<STREAMED, T, V>(dsum + base + held.at[it]);
        }
    };
    if (AHEAD && row < rows) load(nu, nd, ns, row * c);
    for (; row < rows; row += stride) {
        const int64_t base = row * c;
        float u[ITERS][V], d[ITERS][V];
        if constexpr (AHEAD) {
#pragma unroll
            for (int it = 0; it < ITERS; ++it) {
                pu[it] = nu[it];
                pd[it] = nd[it];
                ps[it] = ns[it];
            }
            if (row + stride < rows) load(nu, nd, ns, base + stride * c);
        } else {
            load(pu, pd, ps, base);
        }
#pragma unroll
        for (int it = 0; it < ITERS; ++it) widen<T, V>(pu[it], u[it]);
        float mean, rstd;
        if (mean_in) {
            mean = mean_in[row];
            rstd = rstd_in[row];
        } else {
            float t = 0.f, q = 0.f;
#pragma unroll
            for (int it = 0; it < ITERS; ++it)
#pragma unroll
                for (int i = 0; i < V; ++i) t += held.counted(it, i, u[it][i]);
            mean = team.sum(t) * inv_c;
#pragma unroll
            for (int it = 0; it < ITERS; ++it)
#pragma unroll
                for (int i = 0; i < V; ++i) q += held.counted(it, i, (u[it][i] - mean) * (u[it][i] - mean));
            rstd = 1.f / sqrtf(team.sum(q) * inv_c + eps);
        }
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            float g[V];
            widen<T, V>(gm[it], g);
            widen<T, V>(pd[it], d[it]);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                u[it][i] = (u[it][i] - mean) * rstd;
                dg[it][i] += d[it][i] * u[it][i];              // (another place's values too, which leave() never takes)
                db[it][i] += d[it][i];
                d[it][i] *= g[i];
                const float h = held.counted(it, i, d[it][i]);
                a += h;
                b += h * u[it][i];
            }
        }
        team.sum(a, b);
        a *= inv_c;
        b *= inv_c;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = rstd * (d[it][i] - a - u[it][i] * b);
            if (dsum) {
                float r[V];
                widen<T, V>(ps[it], r);
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] += r[i];
            }
            if (held.stores(it)) *(Pc*)(dx + base + held.at[it]) = narrow<T, V>(o);
        }
    }
    const bool alone = gridDim.x == 1;
    float* out = partial + (size_t)blockIdx.x * 2 * c;
    auto leave = [&](int i, double v) {                // partial sum number i of 2 c
        if (alone) {
            float* to = i < c ? dgamma + i : dbeta + i - c;
            *to = (float)(accumulate ? *to + v : v);
        } else {
            out[i] = (float)v;
        }
    };
    if constexpr (WIDE) {
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (!MASKED || i >= held.skip[it]) {
                    leave(held.at[it] + i, dg[it][i]);
                    leave(c + held.at[it] + i, db[it][i]);
                }
    } else {
        across_teams(lanes, dg, db);
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
        for (int ch = threadIdx.x; ch < c; ch += THREADS) {
            const int p = ch / V, i = MASKED && p == last ? ch - (c - V) : ch % V;
            const float* from = joined + (p / lanes * V + i) * lanes + (p & (lanes - 1));
            double g = 0., b = 0.;
#pragma unroll
            for (int w = 0; w < THREADS / 64; ++w) {
                g += from[w * 2 * slots];
                b += from[w * 2 * slots + slots];
            }
            leave(ch, g);
            leave(c + ch, b);
        }
    }
}

// dgamma and dbeta from the blocks' partial sums, in float64 (the loads take the time): a block takes 64 of the 2 c columns, its sixteen wavefronts every sixteenth of the partial sums each
__global__ __launch_bounds__(1024) void k_ln_join(const float* __restrict__ partial, int blocks, int c, bool accumulate,
                                                  float* __restrict__ dgamma, float* __restrict__ dbeta) {
    __shared__ double part[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = blockIdx.x * 64 + lane;
    double sum = 0.;
    if (i < 2 * c) {
#pragma unroll 8
        for (int b = wave; b < blocks; b += 16) sum += partial[(size_t)b * 2 * c + i];
    }
    part[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || i >= 2 * c) return;
    sum = 0.;
#pragma unroll
    for (int w = 0; w < 16; ++w) sum += part[w][lane];
    float* to = i < c ? dgamma + i : dbeta + i - c;
    *to = (float)(accumulate ? *to + sum : sum);
}

// ---- which kernel takes a shape ------------------------------------------------------------
// Pieces are 16 bytes (one value where the row is shorter).  A lane holds at most sixteen values: with the sums of dgamma and dbeta beside them
// more would leave two wavefronts per SIMD, or spill.  Of the ways to cover a row by lanes times pieces the one with the
// fewest idle places is taken, of equals the one with the fewest pieces a lane; short rows have teams of fewer than eight lanes with a
// piece each (2 M rows of 32 bfloat16 backward, eight lanes: 105 us, four: 77).  Rows of more than 64 such lanes are a block's,
// of as many wavefronts as they need (50000 x 1100 bfloat16 backward, 256 threads: 123 us, 192: 76).
struct Shape {
    int v, iters, lanes;
    bool masked, wide;
};
static Shape shape_of(int dtype, int c) {
    Shape s{dtype == FF_F32 ? 4 : 8, 1, 1, false, false};
    if (c < s.v) s.v = 1;
    const int pieces = (c + s.v - 1) / s.v, most = s.v == 8 ? 2 : 4;
    s.wide = pieces > 64 * most;
    int best = 1 << 30;
    auto take = [&](int iters, int lanes) {
        if (iters * lanes >= best) return;
        best = iters * lanes;
        s.iters = iters;
        s.lanes = lanes;
    };
    for (int iters = 1; iters <= most; ++iters) {
        const int need = (pieces + iters - 1) / iters;
        if (s.wide) {
            const int lanes = (need + 63) & ~63;
            if (lanes <= kWideThreads) take(iters, lanes);
        } else {
            int lanes = iters == 1 ? 1 : 8;
            while (lanes < need) lanes <<= 1;
            if (lanes <= 64) take(iters, lanes);
        }
    }
    s.masked = c != s.lanes * s.iters * s.v;
    return s;
}

// Inputs of 160 MB to 1 GB are loaded past the caches, which hold 256 MB and then keep more of what is written for its reader: 5120 x 384 x 64
// backward 144 -> 140 us, 196608 x 256 61 -> 55, with the gradient that passes by 77 -> 71.  Smaller ones may lie in the caches (65536 x 128 float32, 34 MB,
// 13.6 -> 15.9), larger ones pass through them whole either way (2048 x 2048 x 128 forward 379 -> 386, the one
// shape measured above 1 GB; 0.5 GB is the largest measured that gains, and where between them the rule should turn is not known).
static bool streams(int64_t input_bytes) { return input_bytes > 160000000 && input_bytes < 1000000000; }

template <typename F> static void with_shape(const Shape& s, int64_t input_bytes, F go) {
    auto pieces = [&](auto v, auto masked, auto streamed) {
        constexpr int V = decltype(v)::value;
        auto at = [&](auto wide) {
            if (s.iters == 1) go(v, std::integral_constant<int, 1>{}, masked, wide, streamed);
            else if (s.iters == 2) go(v, std::integral_constant<int, 2>{}, masked, wide, streamed);
            else if constexpr (V == 4) {
                if (s.iters == 3) go(v, std::integral_constant<int, 3>{}, masked, wide, streamed);
                else go(v, std::integral_constant<int, 4>{}, masked, wide, streamed);
            }
        };
        if (s.wide) at(std::true_type{});
        else at(std::false_type{});
    };
    auto full = [&](auto v) {
        const bool streamed = streams(input_bytes);
        if (s.masked && streamed) pieces(v, std::true_type{}, std::true_type{});
        else if (s.masked) pieces(v, std::true_type{}, std::false_type{});
        else if (streamed) pieces(v, std::false_type{}, std::true_type{});
        else pieces(v, std::false_type{}, std::false_type{});
    };
    if (s.v == 8) full(std::integral_constant<int, 8>{});
    else if (s.v == 4) full(std::integral_constant<int, 4>{});
    else go(std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{}, std::true_type{}, std::false_type{}, std::false_type{});
}

static int64_t turns_of(int64_t rows, int per_block) { return (rows + per_block - 1) / per_block; }

// How often a block of the forward pass loads rows, `bytes` at a time.  The rows of a block follow each other and blocks start in
// order, so that what the card works on at one time lies together: 2048 x 2048 x 128 took 505 us with as many blocks as fit on
// the card, each striding over the whole tensor, 428 with a turn each, 377 with two.  Blocks of less than 8 KiB come faster than
// the card starts them (196608 x 384: 77 us with one turn of 3 KiB, 59 with four), more turns gain nothing (16: 411).
static int forward_turns(int64_t all, int64_t bytes) {
    const int64_t most_blocks = 1 << 22;               // the grid's threads stay below 2^32
    int64_t turns = 10240 / bytes, spread = all / (16 * compute_units());
    if (turns > spread) turns = spread;
    if (turns < 1) turns = 1;
    if (all / turns >= most_blocks) turns = (all + most_blocks - 1) / most_blocks;
    return (int)turns;
}

template <typename T>
static void forward_t(const ff_norm_desc& d, const void* x, const void* residual, const void* gamma, const void* beta, void* sum, void* y,
                      float* mean, float* rstd, hipStream_t stream) {
    const Shape s = shape_of(d.dtype, d.c);
    with_shape(s, d.rows * d.c * (int64_t)sizeof(T) * (residual ? 2 : 1), [&](auto v, auto iters, auto masked, auto wide, auto streamed) {
        constexpr int V = decltype(v)::value, I = decltype(iters)::value;
        constexpr bool R = decltype(masked)::value, W = decltype(wide)::value, S = decltype(streamed)::value;
        if constexpr (V != (sizeof(T) == 4 ? 8 : 4)) {
            const int threads = W ? s.lanes : kForwardThreads;
            const int per_block = W ? 1 : threads / s.lanes;
            const int64_t all = turns_of(d.rows, per_block);
            const int turns = forward_turns(all, (int64_t)per_block * d.c * sizeof(T) * (residual ? 2 : 1));
            const int64_t blocks = (all + turns - 1) / turns;
            hipLaunchKernelGGL((k_ln_forward<T, V, I, R, W, S>), dim3((unsigned)blocks), dim3(threads), 0, stream, (const T*)x, (const T*)residual,
                               (const T*)gamma, (const T*)beta, (T*)sum, (T*)y, mean, rstd, d.rows, d.c, s.lanes, turns, d.ln_eps);
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

// Blocks of the backward pass.  Numbers of its own, not the device's, so that the order of the sums does not depend on the machine:
// about sixteen wavefronts on each of 256 compute units, eight where a lane holds more than eight values, and equally many blocks on
// each (20000 x 3000 float32 in 512 blocks of 384 threads 139 us, in 682 171).
constexpr int kBackwardBlocks = 256;
static int backward_blocks(const ff_norm_desc& d, const Shape& s) {
    const bool many = s.v * s.iters > 8;
    const int64_t turns = turns_of(d.rows, s.wide ? 1 : backward_threads(s.v * s.iters) / s.lanes);
    if (turns <= 4) return turns > 0;                  // one block: no partial sums, no second launch
    const int per_unit = s.wide ? (many ? 512 + s.lanes / 2 : 1024) / s.lanes : 1, most = per_unit * kBackwardBlocks;
    return (int)(turns < most ? turns : most);
}

size_t layernorm_backward_workspace(const ff_norm_desc& d) {
    const size_t n = (size_t)backward_blocks(d, shape_of(d.dtype, d.c)) * 2 * d.c * sizeof(float);
    return n < 256 ? 256 : (n + 255) & ~(size_t)255;
}

// Whether a lane of the backward pass asks for its next row ahead.  Streamed inputs always (up to eight values a lane: 5120 x 384 x 64 with saved
// statistics 145 -> 140 us, 196608 x 256 with dsum 71 -> 68).  Of those that may lie in the caches the bfloat16 ones with saved statistics, whose turns
// are the shortest (128 x 256 x 256 14.6 -> 13.7, with dsum 17.2 -> 15.8, 65536 x 384 32.6 -> 29.4; formed again 14.4 -> 15.0 and 33.8 -> 36.1, float32 65536 x 384
// 51.6 -> 52.5).  Of the largest the float32 ones (2^20 x 128 300 -> 289, 2048 x 2048 x 128 1230 -> 1186; bfloat16 571 -> 611).
static bool asks_ahead(const Shape& s, int size, bool saved, int64_t input_bytes) {
    return size == 2 ? saved && input_bytes < 1000000000 : s.iters * s.v <= 8 && input_bytes >= 1000000000;
}

template <typename T>
static void backward_t(const ff_norm_desc& d, const Shape& s, int blocks, const void* src, const void* gamma, const float* mean, const float* rstd, const void* dy,
                       const void* dsum, void* dx, float* dgamma, float* dbeta, bool accumulate, float* partial, hipStream_t stream) {
    const int64_t input_bytes = d.rows * d.c * (int64_t)sizeof(T) * (dsum ? 3 : 2);
    with_shape(s, input_bytes, [&](auto v, auto iters, auto masked, auto wide, auto streamed) {
        constexpr int V = decltype(v)::value, I = decltype(iters)::value;
        constexpr bool R = decltype(masked)::value, W = decltype(wide)::value, S = decltype(streamed)::value;
        if constexpr (V != (sizeof(T) == 4 ? 8 : 4)) {
            const size_t lds = W ? 4 * kWideThreads / 64 * sizeof(float) : (size_t)backward_threads(I * V) / 64 * 2 * I * V * s.lanes * sizeof(float);     // at most 64 KiB
            auto launch = [&](auto ahead) {
                constexpr bool A = decltype(ahead)::value;
                hipLaunchKernelGGL((k_ln_backward<T, V, I, R, W, S, A>), dim3(blocks), dim3(W ? s.lanes : backward_threads(I * V)), lds, stream, (const T*)src,
                                   (const T*)gamma, mean, rstd, (const T*)dy, (const T*)dsum, (T*)dx, partial, dgamma, dbeta, accumulate, d.rows, d.c,
                                   s.lanes, d.ln_eps);
            };
            if constexpr (W || S) launch(std::integral_constant<bool, !W && I * V <= 8>{});
            else if (asks_ahead(s, sizeof(T), mean, input_bytes)) launch(std::true_type{});
            else launch(std::false_type{});
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
