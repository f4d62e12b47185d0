// The optimiser of a whole model in one launch: the norm of all gradients, the AdamW step with states of 32 or 8 bits.
//
// A model of this kind has thousands of tensors of 64 to 65536 values.  The plan cuts them into pieces of at most kPiece values,
// one record each with everything a block needs (addresses, length, decay): a block reads one record and works on one piece, so
// that small tensors cost a block and large ones as many as they have pieces.
#include <math.h>

#include "ff_common.h"

namespace ff {

constexpr int kGroup = 256;              // values that share an exponent in 8-bit states; half a wavefront holds them, eight a lane
constexpr int kPer = 8;
constexpr int kTurn = 8 * kGroup;        // values that a block of 256 threads holds at one time
constexpr int kPiece = 2 * kTurn;
constexpr int kNormBlocks = 1024;        // partial sums of the norm
constexpr int kTopM = 14, kTopV = 30;    // exponent field of a group's largest magnitude among the codes: the highest that rounding up cannot leave

struct Piece {
    void* p;
    const void* g;
    float* master;
    void* m;
    void* v;
    uint8_t* m_exp;
    uint8_t* v_exp;
    int64_t first_value;                 // index of the piece's first value among all tensors'
    uint32_t first_group;                // index of its first group of 256, counted over the tensors
    int32_t n;
    float decay;
    uint32_t tag;                        // the plan's types: a piece of another plan is left alone
};
static_assert(sizeof(Piece) == 80, "the plan's records");

struct PlanHead {
    int64_t pieces, values;
    char rest[80 - 16];
};
static_assert(sizeof(PlanHead) == sizeof(Piece), "a head as long as a record");

struct StepArgs {
    float lr, step_size, beta1, rest1, beta2, rest2, inv_root, eps, max_norm;
    uint32_t seed;
};

static uint32_t tag_of(const ff_adamw_desc& d) { return 0x46000000u | (d.param_dtype << 16) | (d.grad_dtype << 8) | d.state_bits; }

size_t adamw_plan_size(const ff_adamw_desc& d, const ff_adamw_tensor* ts) {
    size_t pieces = 0;
    for (int i = 0; i < d.n_tensors; ++i) pieces += (size_t)((ts[i].numel + kPiece - 1) / kPiece);
    return sizeof(PlanHead) + pieces * sizeof(Piece);
}
bool adamw_plan_whole(size_t bytes) {
    return bytes >= sizeof(PlanHead) && bytes % sizeof(Piece) == 0 && bytes / sizeof(Piece) - 1 <= 0x7fffffffu;
}
static int pieces_of(size_t bytes) { return (int)(bytes / sizeof(Piece) - 1); }

void adamw_plan_fill(const ff_adamw_desc& d, const ff_adamw_tensor* ts, void* plan) {
    PlanHead* head = (PlanHead*)plan;
    *head = PlanHead{};
    Piece* out = (Piece*)plan + 1;
    const size_t ps = d.param_dtype == FF_F32 ? 4 : 2, gs = d.grad_dtype == FF_F32 ? 4 : 2, ss = d.state_bits == 32 ? 4 : 1;
    int64_t value = 0, group = 0;
    for (int i = 0; i < d.n_tensors; ++i) {
        const ff_adamw_tensor& t = ts[i];
        for (int64_t at = 0; at < t.numel; at += kPiece) {
            Piece r{};
            r.g = (const char*)t.g + at * gs;
            if (d.state_bits) {
                r.p = (char*)t.p + at * ps;
                r.master = t.master ? t.master + at : nullptr;
                r.m = (char*)t.m + at * ss;
                r.v = (char*)t.v + at * ss;
                r.m_exp = t.m_exp ? t.m_exp + at / kGroup : nullptr;
                r.v_exp = t.v_exp ? t.v_exp + at / kGroup : nullptr;
                r.decay = t.weight_decay;
            }
            r.first_value = value + at;
            r.first_group = (uint32_t)(group + at / kGroup);
            r.n = (int32_t)(t.numel - at < kPiece ? t.numel - at : kPiece);
            r.tag = tag_of(d);
            *out++ = r;
        }
        value += t.numel;
        group += (t.numel + kGroup - 1) / kGroup;
    }
    head->pieces = out - ((Piece*)plan + 1);
    head->values = value;
}

// ---- 8-bit states ------------------------------------------------------------------------
// over the 32 lanes of half a wavefront
__device__ __forceinline__ uint32_t max32(uint32_t x) {
    auto with = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
    x = with(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kDppXor1, 0xf, 0xf, true));
    x = with(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kDppXor2, 0xf, 0xf, true));
    x = with(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kDppHalfMirror, 0xf, 0xf, true));
    x = with(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kDppRor8, 0xf, 0xf, true));
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return with(r[0], r[1]);
}

// 32 bits from the index of a value and the step's seed, each round xor with the upper half and a product with an odd factor
// (2^32 / golden ratio, and the leading digits of pi and of e - 2): enough for the bits of neighbours and of successive
// steps to be unrelated.
__device__ __forceinline__ uint32_t dither_bits(uint32_t index, uint32_t seed) {
    uint32_t h = index + seed * 0x9E3779B1u;
    h = (h ^ (h >> 16)) * 0x243F6A89u;
    h = (h ^ (h >> 15)) * 0xB7E15163u;
    return h ^ (h >> 16);
}

// code of |x| in a group whose largest magnitude has exponent field e; r: 16 random bits below the code's last place
template <int TOP> __device__ __forceinline__ uint32_t encode(float mag, uint32_t e, uint32_t r) {
    return (__float_as_uint(__builtin_ldexpf(mag, TOP - (int)e)) + (r << 4)) >> 20;
}
template <int TOP> __device__ __forceinline__ float decode(uint32_t code, uint32_t e) {
    const float x = __builtin_ldexpf(__uint_as_float(code << 20), (int)e - TOP);
    return e == 255u ? __uint_as_float(0x7fc00000u) : x;
}
__device__ __forceinline__ float decode_m(uint8_t code, uint32_t e) {
    const float x = decode<kTopM>(code & 0x7fu, e);
    return code & 0x80u ? -x : x;
}

// ---- norm of all gradients ---------------------------------------------------------------
// squares and sums in float64: no square leaves its range, and the order of the sums does not show in the float32 result
__device__ __forceinline__ double block_sum(double x) {
    __shared__ double part[4];
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    return part[0] + part[1] + part[2] + part[3];
}

template <typename G>
__global__ __launch_bounds__(256) void k_grad_norm(const Piece* __restrict__ pieces, int n_pieces, uint32_t tag, double* __restrict__ partial) {
    double sum = 0.;
    for (int i = blockIdx.x; i < n_pieces; i += gridDim.x) {
        const Piece& pc = pieces[i];
        if (pc.tag != tag) continue;
        const G* g = (const G*)pc.g;
        for (int j = threadIdx.x; j < pc.n; j += 256) {
            const double x = to_f32<G>(g[j]);
            sum += x * x;
        }
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

__global__ __launch_bounds__(256) void k_norm_join(const double* __restrict__ partial, int n, float* __restrict__ norm) {
    double sum = 0.;
    for (int i = threadIdx.x; i < n; i += 256) sum += partial[i];
    sum = block_sum(sum);
    if (threadIdx.x == 0) *norm = (float)sqrt(sum);
}

size_t grad_norm_workspace() { return kNormBlocks * sizeof(double); }

ff_status grad_norm_run(const ff_adamw_desc& d, const void* plan, size_t plan_bytes, float* norm, void* ws, hipStream_t stream) {
    const Piece* pieces = (const Piece*)plan + 1;
    const int n = pieces_of(plan_bytes);
    const int blocks = n < kNormBlocks ? n : kNormBlocks;
    double* partial = (double*)ws;
    Timed t(KK_GRAD_NORM, stream);
    if (blocks > 0) {
        if (d.grad_dtype == FF_F32) hipLaunchKernelGGL((k_grad_norm<float>), dim3(blocks), dim3(256), 0, stream, pieces, n, tag_of(d), partial);
        else hipLaunchKernelGGL((k_grad_norm<bf16_t>), dim3(blocks), dim3(256), 0, stream, pieces, n, tag_of(d), partial);
    }
    hipLaunchKernelGGL(k_norm_join, dim3(1), dim3(256), 0, stream, partial, blocks, norm);
    return check_launch("ff_grad_norm");
}

// ---- the step ----------------------------------------------------------------------------
template <typename P, typename G, int BITS>
__global__ __launch_bounds__(256) void k_adamw(const Piece* __restrict__ pieces, uint32_t tag, StepArgs a, const float* __restrict__ norm) {
    const Piece& pc = pieces[blockIdx.x];
    float k = 1.f;
    if (norm) {
        const float n = *norm;
        if (!(n <= 3.402823466e38f)) return;                   // not finite: the step is left out
        const float c = a.max_norm / (n + 1e-6f);
        k = c < 1.f ? c : 1.f;
    }
    if (pc.tag != tag) return;
    const int lane = threadIdx.x & 31;
    const float keep = 1.f - a.lr * pc.decay;
    const G* g_ = (const G*)pc.g;
    P* p_ = (P*)pc.p;
    for (int base = (threadIdx.x >> 5) * kGroup; base < pc.n; base += kTurn) {
        float m[kPer], v[kPer], w[kPer];
        uint32_t em = 0, ev = 0;
        if constexpr (BITS == 8) {
            em = pc.m_exp[base / kGroup];
            ev = pc.v_exp[base / kGroup];
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int at = base + lane + 32 * i;
            m[i] = v[i] = w[i] = 0.f;
            if (at < pc.n) {
                const float g = to_f32<G>(g_[at]) * k;
                if constexpr (BITS == 8) {
                    m[i] = decode_m(((const uint8_t*)pc.m)[at], em);
                    v[i] = decode<kTopV>(((const uint8_t*)pc.v)[at], ev);
                } else {
                    m[i] = ((const float*)pc.m)[at];
                    v[i] = ((const float*)pc.v)[at];
                }
                w[i] = pc.master ? pc.master[at] : to_f32<P>(p_[at]);
                m[i] = a.beta1 * m[i] + a.rest1 * g;
                v[i] = a.beta2 * v[i] + a.rest2 * (g * g);
                w[i] = w[i] * keep - a.step_size * (m[i] / (sqrtf(v[i]) * a.inv_root + a.eps));
            }
        }
        if constexpr (BITS == 8) {
            uint32_t mm = 0, mv = 0;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const uint32_t bm = __float_as_uint(m[i]) & 0x7fffffffu, bv = __float_as_uint(v[i]) & 0x7fffffffu;
                mm = mm > bm ? mm : bm;
                mv = mv > bv ? mv : bv;
            }
            em = max32(mm) >> 23;
            ev = max32(mv) >> 23;
            if (lane == 0) {
                pc.m_exp[base / kGroup] = (uint8_t)em;
                pc.v_exp[base / kGroup] = (uint8_t)ev;
            }
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int at = base + lane + 32 * i;
            if (at >= pc.n) continue;
            if (pc.master) pc.master[at] = w[i];
            p_[at] = from_f32<P>(w[i]);
            if constexpr (BITS == 8) {
                const uint32_t r = dither_bits(pc.first_group * kGroup + (uint32_t)at, a.seed);
                uint32_t cm = encode<kTopM>(fabsf(m[i]), em, r & 0xffffu) | (__float_as_uint(m[i]) >> 31 << 7);
                uint32_t cv = encode<kTopV>(v[i], ev, r >> 16);
                cv = cv == 0 && v[i] > 0.f ? 1u : cv;
                ((uint8_t*)pc.m)[at] = (uint8_t)(em == 255u ? 0u : cm);
                ((uint8_t*)pc.v)[at] = (uint8_t)(ev == 255u ? 0u : cv);
            } else {
                ((float*)pc.m)[at] = m[i];
                ((float*)pc.v)[at] = v[i];
            }
        }
    }
}

template <typename P, typename G>
static void step_launch(int bits, int n, const Piece* pieces, uint32_t tag, const StepArgs& a, const float* norm, hipStream_t stream) {
    if (bits == 8) hipLaunchKernelGGL((k_adamw<P, G, 8>), dim3(n), dim3(256), 0, stream, pieces, tag, a, norm);
    else hipLaunchKernelGGL((k_adamw<P, G, 32>), dim3(n), dim3(256), 0, stream, pieces, tag, a, norm);
}

ff_status adamw_step_run(const ff_adamw_desc& d, const void* plan, size_t plan_bytes, const ff_adamw_hyper& h, const float* norm,
                         hipStream_t stream) {
    const Piece* pieces = (const Piece*)plan + 1;
    const int n = pieces_of(plan_bytes);
    if (n == 0) return FF_OK;
    const double c1 = 1. - pow(h.beta1, (double)h.step), c2 = 1. - pow(h.beta2, (double)h.step);
    StepArgs a{(float)h.lr, (float)(h.lr / c1), (float)h.beta1, (float)(1. - h.beta1), (float)h.beta2, (float)(1. - h.beta2),
               (float)(1. / sqrt(c2)), (float)h.eps, norm ? (float)h.max_norm : 0.f, h.seed};
    const uint32_t tag = tag_of(d);
    Timed t(KK_ADAMW, stream);
    if (d.param_dtype == FF_F32) {
        if (d.grad_dtype == FF_F32) step_launch<float, float>(d.state_bits, n, pieces, tag, a, norm, stream);
        else step_launch<float, bf16_t>(d.state_bits, n, pieces, tag, a, norm, stream);
    } else {
        if (d.grad_dtype == FF_F32) step_launch<bf16_t, float>(d.state_bits, n, pieces, tag, a, norm, stream);
        else step_launch<bf16_t, bf16_t>(d.state_bits, n, pieces, tag, a, norm, stream);
    }
    return check_launch("ff_adamw_step");
}

// ---- moments as float32 ------------------------------------------------------------------
template <int BITS>
__global__ __launch_bounds__(256) void k_moments(const Piece* __restrict__ pieces, uint32_t tag, float* __restrict__ m_out, float* __restrict__ v_out) {
    const Piece& pc = pieces[blockIdx.x];
    if (pc.tag != tag) return;
    for (int at = threadIdx.x; at < pc.n; at += 256) {
        if (m_out) m_out[pc.first_value + at] = BITS == 8 ? decode_m(((const uint8_t*)pc.m)[at], pc.m_exp[at / kGroup]) : ((const float*)pc.m)[at];
        if (v_out) v_out[pc.first_value + at] = BITS == 8 ? decode<kTopV>(((const uint8_t*)pc.v)[at], pc.v_exp[at / kGroup]) : ((const float*)pc.v)[at];
    }
}

ff_status adamw_moments_run(const ff_adamw_desc& d, const void* plan, size_t plan_bytes, float* m_out, float* v_out, hipStream_t stream) {
    const Piece* pieces = (const Piece*)plan + 1;
    const int n = pieces_of(plan_bytes);
    if (n == 0) return FF_OK;
    Timed t(KK_MOMENTS, stream);
    if (d.state_bits == 8) hipLaunchKernelGGL((k_moments<8>), dim3(n), dim3(256), 0, stream, pieces, tag_of(d), m_out, v_out);
    else hipLaunchKernelGGL((k_moments<32>), dim3(n), dim3(256), 0, stream, pieces, tag_of(d), m_out, v_out);
    return check_launch("ff_adamw_moments");
}

}  // namespace ff
