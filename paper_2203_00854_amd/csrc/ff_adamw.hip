// The optimiser of a whole model in one launch: the norm of all gradients, the AdamW step with states of 32 or 8 bits.
//
// A model of this kind has thousands of tensors of 64 to 65536 values.  The plan cuts them into pieces of at most kPiece values,
// one record each with everything a block needs (addresses, length, decay): a block reads one record and works on one piece, so
// that small tensors cost a block and large ones as many as they have pieces.
#include <math.h>
#include <stdlib.h>

#include <algorithm>
#include <type_traits>

#include "ff_common.h"

namespace ff {

constexpr int kGroup = 256;              // values that share an exponent in 8-bit states
constexpr int kTurn = 8 * kGroup;        // values that a block of 256 threads holds at one time
constexpr int kPiece = kTurn;            // (two turns to a piece: 264 us where one takes 245, by the blocks that end together)
constexpr int kNormBlocks = 2048;        // partial sums of the norm
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
// (A plan is an empty record, so that one without values has an address too, and one record a piece.)

struct StepArgs {
    float lr, step_size, beta1, rest1, beta2, rest2, inv_root, eps, max_norm;
    uint32_t seed;
};

static uint32_t tag_of(const ff_adamw_desc& d) { return 0x46000000u | (d.param_dtype << 16) | (d.grad_dtype << 8) | d.state_bits; }

size_t adamw_plan_size(const ff_adamw_desc& d, const ff_adamw_tensor* ts) {
    size_t pieces = 0;
    for (int i = 0; i < d.n_tensors; ++i) pieces += (size_t)((ts[i].numel + kPiece - 1) / kPiece);
    return (1 + pieces) * sizeof(Piece);
}
bool adamw_plan_whole(size_t bytes) {
    return bytes >= sizeof(Piece) && bytes % sizeof(Piece) == 0 && bytes / sizeof(Piece) - 1 < (1u << 24);     // 2^32 threads in blocks of 256
}
static int pieces_of(size_t bytes) { return (int)(bytes / sizeof(Piece) - 1); }
size_t adamw_least_values(const ff_adamw_desc& d, size_t plan_bytes) {         // all pieces but each tensor's last are full
    const size_t pieces = pieces_of(plan_bytes), last = pieces < (size_t)d.n_tensors ? pieces : (size_t)d.n_tensors;
    return (pieces - last) * kPiece + last;
}

void adamw_plan_fill(const ff_adamw_desc& d, const ff_adamw_tensor* ts, void* plan) {
    Piece* out = (Piece*)plan;
    *out++ = Piece{};
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
}

// Whether a tensor that the step writes shares memory with another one (tied weights listed twice, say): their blocks would race.
// -1 if there is no host memory to find out.
int adamw_overlaps(const ff_adamw_desc& d, const ff_adamw_tensor* ts) {
    struct Span {
        uintptr_t from, to;
        bool written;
    };
    if (d.state_bits == 0 || d.n_tensors == 0) return 0;
    Span* spans = (Span*)malloc(sizeof(Span) * 7 * (size_t)d.n_tensors);
    if (!spans) return -1;
    const int64_t ps = d.param_dtype == FF_F32 ? 4 : 2, gs = d.grad_dtype == FF_F32 ? 4 : 2, ss = d.state_bits == 32 ? 4 : 1;
    size_t n = 0;
    const auto before = [](const Span& a, const Span& b) { return a.from < b.from; };
    // one kind of tensor after the other: each is mostly in order already (3504 tensors 0.2 ms)
    auto take = [&](bool written, auto from, auto bytes) {
        Span* first = spans + n;
        for (int i = 0; i < d.n_tensors; ++i)
            if (from(ts[i]) && ts[i].numel) spans[n++] = Span{(uintptr_t)from(ts[i]), (uintptr_t)from(ts[i]) + (uintptr_t)bytes(ts[i]), written};
        if (!std::is_sorted(first, spans + n, before)) std::sort(first, spans + n, before);
        std::inplace_merge(spans, first, spans + n, before);
    };
    typedef const ff_adamw_tensor& Tensor;
    const auto groups = [](Tensor t) { return (t.numel + kGroup - 1) / kGroup; };
    const auto states = [=](Tensor t) { return t.numel * ss; };
    take(true, [](Tensor t) { return t.p; }, [=](Tensor t) { return t.numel * ps; });
    take(true, [](Tensor t) { return t.master; }, [](Tensor t) { return t.numel * 4; });
    take(true, [](Tensor t) { return t.m; }, states);
    take(true, [](Tensor t) { return t.v; }, states);
    take(true, [](Tensor t) { return t.m_exp; }, groups);
    take(true, [](Tensor t) { return t.v_exp; }, groups);
    take(false, [](Tensor t) { return t.g; }, [=](Tensor t) { return t.numel * gs; });
    uintptr_t end = 0, end_written = 0;
    int found = 0;
    for (size_t i = 0; i < n; ++i) {
        if (spans[i].from < (spans[i].written ? end : end_written)) found = 1;
        if (spans[i].to > end) end = spans[i].to;
        if (spans[i].written && spans[i].to > end_written) end_written = spans[i].to;
    }
    free(spans);
    return found;
}

// ---- four neighbours ---------------------------------------------------------------------
// A record's pointers are read from memory, where the compiler cannot see that they lead to global memory: it is told, or it would use loads
// that look for LDS behind every address.
template <typename T> struct At {
    typedef __attribute__((address_space(1))) T One;
    typedef T Vec __attribute__((ext_vector_type(4), aligned(sizeof(T))));        // at the alignment of one value
    typedef __attribute__((address_space(1))) Vec Four;
};
template <typename T> __device__ __forceinline__ typename At<T>::One* global(void* p) { return (typename At<T>::One*)p; }
template <typename T> __device__ __forceinline__ const typename At<T>::One* global(const void* p) { return (const typename At<T>::One*)p; }

// How values at, .. at + 3 of a piece of n are reached: all known to be there, that and past the caches, some of them past the end of at least
// four, or of fewer than four.
enum How { kWhole, kStreamed, kTail, kTiny };
template <How HOW> constexpr bool kAllThere = HOW == kWhole || HOW == kStreamed;
template <How HOW, typename T> __device__ __forceinline__ typename At<T>::Vec fetch(const typename At<T>::One* p) {
    const typename At<T>::Four* four = (const typename At<T>::Four*)p;
    if constexpr (HOW == kStreamed) return __builtin_nontemporal_load(four);
    else return *four;
}
template <How HOW, typename T> __device__ __forceinline__ void put(typename At<T>::One* p, typename At<T>::Vec v) {
    typename At<T>::Four* four = (typename At<T>::Four*)p;
    if constexpr (HOW == kStreamed) __builtin_nontemporal_store(v, four);
    else *four = v;
}
// kTail: where the four would pass the end, they are the last four of the piece, moved down, with zeros behind: one load for all lanes, without branches.
template <How HOW, typename T> __device__ __forceinline__ typename At<T>::Vec tail4(const typename At<T>::One* base, int at, int n) {
    typename At<T>::Vec f = {};
    if constexpr (HOW == kTail) {
        const int from = at + 4 > n ? n - 4 : at, past = at - from;
        f = *(const typename At<T>::Four*)(base + from);
        if constexpr (sizeof(T) == 4) {
            if (past & 1) f = typename At<T>::Vec{f[1], f[2], f[3], 0};
            if (past & 2) f = typename At<T>::Vec{f[2], f[3], 0, 0};
            if (past >= 4) f = typename At<T>::Vec{};
        } else {
            typedef std::conditional_t<sizeof(T) == 2, uint64_t, uint32_t> Word;
            f = __builtin_bit_cast(typename At<T>::Vec, past < 4 ? (Word)(__builtin_bit_cast(Word, f) >> 8 * sizeof(T) * past) : (Word)0);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (at + i < n) f[i] = base[at + i];
    }
    return f;
}
template <How HOW, typename T> __device__ __forceinline__ void load4(const void* base, int at, int n, float (&v)[4]) {
    typename At<T>::Vec f;
    if constexpr (kAllThere<HOW>) f = fetch<HOW, T>(global<T>(base) + at);
    else f = tail4<HOW, T>(global<T>(base), at, n);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = to_f32<T>(f[i]);
}
template <How HOW, typename T> __device__ __forceinline__ void store4(void* base, int at, int n, const float (&v)[4]) {
    const auto p = global<T>(base) + at;
    typename At<T>::Vec f;
    if constexpr (sizeof(T) == 2) {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        typedef float f32x4 __attribute__((ext_vector_type(4)));
        f = __builtin_bit_cast(typename At<T>::Vec, __builtin_convertvector((f32x4{v[0], v[1], v[2], v[3]}), bf16x4));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = v[i];
    }
    if constexpr (kAllThere<HOW>) {
        put<HOW, T>(p, f);
    } else if (at + 4 <= n) {
        put<kWhole, T>(p, f);
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (at + i < n) p[i] = f[i];
    }
}
template <How HOW> __device__ __forceinline__ uint32_t load4(const void* base, int at, int n) {                     // four codes
    typename At<uint8_t>::Vec f;
    if constexpr (kAllThere<HOW>) f = fetch<HOW, uint8_t>(global<uint8_t>(base) + at);
    else f = tail4<HOW, uint8_t>(global<uint8_t>(base), at, n);
    return __builtin_bit_cast(uint32_t, f);
}
template <How HOW> __device__ __forceinline__ void store4(void* base, int at, int n, uint32_t w) {
    const auto p = global<uint8_t>(base) + at;
    if constexpr (kAllThere<HOW>) {
        put<HOW, uint8_t>(p, __builtin_bit_cast(At<uint8_t>::Vec, w));
    } else if (at + 4 <= n) {
        put<kWhole, uint8_t>(p, __builtin_bit_cast(At<uint8_t>::Vec, w));
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (at + i < n) p[i] = (uint8_t)(w >> 8 * i);
    }
}

// The turn of a piece, 512 values to a wavefront: without a check of any lane where all of them are there.
template <How HOW, typename F> __device__ __forceinline__ void turns_as(int n, F go) {
    for (int first = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 2 * kGroup; first < n; first += kTurn) {
        const int base = first + (threadIdx.x & 32) * (kGroup / 32);
        if (first + 2 * kGroup <= n) go(std::integral_constant<How, HOW>{}, base);
        else if (n >= 4) go(std::integral_constant<How, kTail>{}, base);
        else go(std::integral_constant<How, kTiny>{}, base);
    }
}
// What passes once per step goes past the caches, which keeps them for the gradients between their norm and the step: 48 blocks with a
// master copy 300 -> 245 us for both, float32 alone 316 -> 244, 8 bits 139 -> 120.  Not where a tensor lies across the
// lines, whose parts would reach memory one by one (400 ragged tensors 64 -> 71).  (A loop of its own for each: of two branches inside
// one loop the compiler would join the loads, and lose their hint.)
template <typename F> __device__ __forceinline__ void turns(int n, bool streamed, F go) {
    if (streamed) turns_as<kStreamed>(n, go);
    else turns_as<kWhole>(n, go);
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
constexpr uint32_t kDitherSeed = 0x9E3779B1u;
__device__ __forceinline__ uint32_t dither_bits(uint32_t h) {                  // h: index + seed kDitherSeed
    h = (h ^ (h >> 16)) * 0x243F6A89u;
    h = (h ^ (h >> 15)) * 0xB7E15163u;
    return h ^ (h >> 16);
}

// A group's exponent field e turns codes into values by a shift of the exponent, e - TOP, and into NaN where a member was not finite.
template <int TOP> struct Scale {
    int shift;
    uint32_t nan;
    __device__ __forceinline__ explicit Scale(uint32_t e) : shift((int)e - TOP), nan(e == 255u ? 0x7fc00000u : 0u) {}
    // code i of four; TOP 14 has a sign in the upper bit
    __device__ __forceinline__ float value(uint32_t four, int i) const {
        const uint32_t w = four >> 8 * i;
        uint32_t bits = (w & (TOP == kTopM ? 0x7fu : 0xffu)) << 20 | nan;
        if constexpr (TOP == kTopM) bits |= w << 24 & 0x80000000u;
        return __builtin_ldexpf(__uint_as_float(bits), shift);
    }
    // code of a magnitude; r: 16 random bits, which stand below the code's last place
    __device__ __forceinline__ uint32_t code(float mag, uint32_t r) const { return (__float_as_uint(__builtin_ldexpf(mag, -shift)) + (r << 4)) >> 20; }
};

// ---- norm of all gradients ---------------------------------------------------------------
// Squares and sums in float64: no square leaves its range, and the order of the sums does not show in the float32 result.  Bound by HBM and two
// dependent launches: 49.1 M bfloat16 values 19 us (5.2 TB/s) and 5 for the join, whose loads are all under way at once.  As many blocks as the card holds, each
// with the next record on its way: blocks of neighbouring pieces, two or four pieces at a time, took 27 to 32 for both.
// (A piece of another plan has no values here, and makes the norm one that no step is taken with.)
constexpr double kNoNorm = __builtin_nan("");
template <int WAVES> __device__ __forceinline__ double block_sum(double x) {
    __shared__ double part[WAVES];
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    x = part[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) x += part[w];
    return x;
}

template <typename G>
__global__ __launch_bounds__(256) void k_grad_norm(const Piece* __restrict__ pieces, int n_pieces, uint32_t tag, double* __restrict__ partial) {
    double sum = 0.;
    const void* g = pieces[blockIdx.x].g;
    int n = pieces[blockIdx.x].tag == tag ? pieces[blockIdx.x].n : 0;
    for (int i = blockIdx.x; i < n_pieces; i += gridDim.x) {
        // the next piece's record is on its way while this one's values are
        const Piece& next = pieces[i + (int)gridDim.x < n_pieces ? i + (int)gridDim.x : i];
        const void* g_next = next.g;
        const int n_next = next.tag == tag ? next.n : 0;
        float v[kPiece / 1024][4] = {};
        if (n == kPiece) {
#pragma unroll
            for (int t = 0; t < kPiece / 1024; ++t) load4<kWhole, G>(g, (threadIdx.x + 256 * t) * 4, n, v[t]);
        } else if (n >= 4) {
#pragma unroll
            for (int t = 0; t < kPiece / 1024; ++t) load4<kTail, G>(g, (threadIdx.x + 256 * t) * 4, n, v[t]);
        } else if (n > 0) {
#pragma unroll
            for (int t = 0; t < kPiece / 1024; ++t) load4<kTiny, G>(g, (threadIdx.x + 256 * t) * 4, n, v[t]);
        } else {
            sum = kNoNorm;
        }
#pragma unroll
        for (int t = 0; t < kPiece / 1024; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) sum += (double)v[t][j] * (double)v[t][j];
        g = g_next;
        n = n_next;
    }
    sum = block_sum<4>(sum);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

__global__ __launch_bounds__(1024) void k_norm_join(const double* __restrict__ partial, int n, float* __restrict__ norm) {
    double sum = 0.;
#pragma unroll
    for (int i = 0; i < kNormBlocks; i += 1024)
        if (i + (int)threadIdx.x < n) sum += partial[i + threadIdx.x];
    sum = block_sum<16>(sum);
    if (threadIdx.x == 0) *norm = (float)sqrt(sum);
}

// A few pieces by one block, a wavefront each: no second launch.  Passes one after another, two launches and one: 16 float32 pieces of 2048 values 6.6 and
// 4.1 us, 32 6.5 and 4.2, 48 6.6 and 5.3, 64 6.6 and 6.1; 32 tensors of up to 2047 6.6 and 5.9, 64 of up to 300 6.6 and 8.9.
constexpr int kFewPieces = 32;
template <typename G>
__global__ __launch_bounds__(1024) void k_norm_few(const Piece* __restrict__ pieces, int n_pieces, uint32_t tag, float* __restrict__ norm) {
    const int lane = threadIdx.x & 63;
    double sum = 0.;
    for (int i = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); i < n_pieces; i += 16) {
        const Piece& pc = pieces[i];
        const int n = pc.tag == tag ? pc.n : 0;
        float v[kPiece / 256][4] = {};
        if (n == kPiece) {
#pragma unroll
            for (int t = 0; t < kPiece / 256; ++t) load4<kWhole, G>(pc.g, (lane + 64 * t) * 4, n, v[t]);
        } else if (n >= 4) {
#pragma unroll
            for (int t = 0; t < kPiece / 256; ++t) load4<kTail, G>(pc.g, (lane + 64 * t) * 4, n, v[t]);
        } else if (n > 0) {
#pragma unroll
            for (int t = 0; t < kPiece / 256; ++t) load4<kTiny, G>(pc.g, (lane + 64 * t) * 4, n, v[t]);
        } else {
            sum = kNoNorm;
        }
#pragma unroll
        for (int t = 0; t < kPiece / 256; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) sum += (double)v[t][j] * (double)v[t][j];
    }
    sum = block_sum<16>(sum);
    if (threadIdx.x == 0) *norm = (float)sqrt(sum);
}

size_t grad_norm_workspace() { return kNormBlocks * sizeof(double); }

ff_status grad_norm_run(const ff_adamw_desc& d, const void* plan, size_t plan_bytes, float* norm, void* ws, hipStream_t stream) {
    const Piece* pieces = (const Piece*)plan + 1;
    const int n = pieces_of(plan_bytes);
    const int blocks = n < kNormBlocks ? n : kNormBlocks;
    double* partial = (double*)ws;
    Timed t(KK_GRAD_NORM, stream);
    if (n <= kFewPieces) {
        if (d.grad_dtype == FF_F32) hipLaunchKernelGGL((k_norm_few<float>), dim3(1), dim3(1024), 0, stream, pieces, n, tag_of(d), norm);
        else hipLaunchKernelGGL((k_norm_few<bf16_t>), dim3(1), dim3(1024), 0, stream, pieces, n, tag_of(d), norm);
        return check_launch("ff_grad_norm");
    }
    if (d.grad_dtype == FF_F32) hipLaunchKernelGGL((k_grad_norm<float>), dim3(blocks), dim3(256), 0, stream, pieces, n, tag_of(d), partial);
    else hipLaunchKernelGGL((k_grad_norm<bf16_t>), dim3(blocks), dim3(256), 0, stream, pieces, n, tag_of(d), partial);
    hipLaunchKernelGGL(k_norm_join, dim3(1), dim3(1024), 0, stream, partial, blocks, norm);
    return check_launch("ff_grad_norm");
}

// ---- the step ----------------------------------------------------------------------------
// The square root and the reciprocal are the machine's, good to a unit in their last place: they reach the weight alone, where
// they are 2^-23 of the step.  The root takes no subnormal numbers: a v below 2^-126 counts as that (as whole numbers, so that NaN stays the larger).
__device__ __forceinline__ float root_of(float v) {
    const uint32_t b = __float_as_uint(v);
    return __builtin_amdgcn_sqrtf(__uint_as_float(b > 0x00800000u ? b : 0x00800000u));
}

// Bound by HBM: with 32-bit states 22 to 30 bytes a value, with 8 bits 10 to 18 and 66 vector instructions a value, which take about as long where
// the tensors are bfloat16.  48 Evoformer blocks (49.1 M values): 215 us with master copies (6.4 TB/s), 107 with float32 weights
// and 8-bit states (6.4 TB/s).
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
    const float decay = a.lr * pc.decay;
    const bool master = pc.master != nullptr;
    const uintptr_t states = BITS == 32 ? (uintptr_t)pc.m | (uintptr_t)pc.v : 0;
    const bool streamed = (((uintptr_t)pc.p | (uintptr_t)pc.g | (uintptr_t)pc.master | states) & 15u) == 0;
    turns(pc.n, streamed, [&](auto how, int base) {
        constexpr How H = decltype(how)::value;
        constexpr bool W = kAllThere<H>;
        float m[2][4], v[2][4], w[2][4], g[2][4];
        [[maybe_unused]] uint32_t fm[2], fv[2], em = 0, ev = 0;
        const bool group = W || base < pc.n;                   // (at the end of a piece half a wavefront may have none)
        if constexpr (BITS == 8) {
            if (group) {
                em = global<uint8_t>((const void*)pc.m_exp)[base / kGroup];
                ev = global<uint8_t>((const void*)pc.v_exp)[base / kGroup];
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = base + h * 128 + lane * 4;
            load4<H, G>(pc.g, at, pc.n, g[h]);
            if (master) load4<H, float>(pc.master, at, pc.n, w[h]);
            else load4<H, P>(pc.p, at, pc.n, w[h]);
            if constexpr (BITS == 8) {
                fm[h] = load4<H>(pc.m, at, pc.n);
                fv[h] = load4<H>(pc.v, at, pc.n);
            } else {
                load4<H, float>(pc.m, at, pc.n, m[h]);
                load4<H, float>(pc.v, at, pc.n, v[h]);
            }
        }
        if constexpr (BITS == 8) {
            const Scale<kTopM> sm(em);
            const Scale<kTopV> sv(ev);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    m[h][i] = sm.value(fm[h], i);
                    v[h][i] = sv.value(fv[h], i);
                }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = g[h][i] * k;
                m[h][i] = a.beta1 * m[h][i] + a.rest1 * x;
                v[h][i] = a.beta2 * v[h][i] + a.rest2 * (x * x);
                const float root = root_of(v[h][i]) * a.inv_root + a.eps;
                // (the decay's share and the step's meet before the one rounding against the weight: 1 - decay next to 1 loses a fifth of a decay of 1e-7)
                w[h][i] -= decay * w[h][i] + a.step_size * (m[h][i] * __builtin_amdgcn_rcpf(root));
            }
            const int at = base + h * 128 + lane * 4;
            if (master) store4<H, float>(pc.master, at, pc.n, w[h]);
            store4<H, P>(pc.p, at, pc.n, w[h]);
            if constexpr (BITS == 32) {
                store4<H, float>(pc.m, at, pc.n, m[h]);
                store4<H, float>(pc.v, at, pc.n, v[h]);
            }
        }
        if constexpr (BITS == 8) {
            // places past the tensor's end have loaded zeros, but for NaN in a group that holds it: they stay out of the maximum
            uint32_t mm = 0, mv = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (W || base + h * 128 + lane * 4 + i < pc.n) {
                        const uint32_t bm = __float_as_uint(m[h][i]) & 0x7fffffffu, bv = __float_as_uint(v[h][i]) & 0x7fffffffu;
                        mm = mm > bm ? mm : bm;
                        mv = mv > bv ? mv : bv;
                    }
            em = max32(mm) >> 23;
            ev = max32(mv) >> 23;
            if (lane == 0 && group) {
                global<uint8_t>(pc.m_exp)[base / kGroup] = (uint8_t)em;
                global<uint8_t>(pc.v_exp)[base / kGroup] = (uint8_t)ev;
            }
            const Scale<kTopM> sm(em);
            const Scale<kTopV> sv(ev);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = base + h * 128 + lane * 4;
                const uint32_t index = pc.first_group * kGroup + a.seed + (uint32_t)at;
                uint32_t cm = 0, cv = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t r = dither_bits(index + i), bm = __float_as_uint(m[h][i]), bv = __float_as_uint(v[h][i]);
                    cm |= (sm.code(fabsf(m[h][i]), r & 0xffffu) | (bm >> 24 & 0x80u)) << 8 * i;
                    const uint32_t c = sv.code(v[h][i], r >> 16), least = bv < 1u ? bv : 1u;      // a positive v is not held as 0
                    cv |= (c > least ? c : least) << 8 * i;
                }
                store4<H>(pc.m, at, pc.n, em == 255u ? 0u : cm);
                store4<H>(pc.v, at, pc.n, ev == 255u ? 0u : cv);
            }
        }
    });
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
               (float)(1. / sqrt(c2)), (float)h.eps, norm ? (float)h.max_norm : 0.f, h.seed * kDitherSeed};
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
// 2 bytes read, 8 written a value: 49.1 M values 86 us, 5.7 TB/s.
template <int BITS>
__global__ __launch_bounds__(256) void k_moments(const Piece* __restrict__ pieces, uint32_t tag, float* __restrict__ m_out, float* __restrict__ v_out) {
    const Piece& pc = pieces[blockIdx.x];
    if (pc.tag != tag) return;
    const int lane = threadIdx.x & 31;
    const uintptr_t states = BITS == 32 ? (uintptr_t)pc.m | (uintptr_t)pc.v : 0;
    const bool streamed = (((uintptr_t)m_out | (uintptr_t)v_out | (uintptr_t)pc.first_value * 4 | states) & 15u) == 0;
    turns(pc.n, streamed, [&](auto how, int base) {
        constexpr How H = decltype(how)::value;
        constexpr bool W = kAllThere<H>;
        float m[2][4], v[2][4];
        if constexpr (BITS == 8) {
            const bool group = W || base < pc.n;
            const Scale<kTopM> sm(group ? global<uint8_t>((const void*)pc.m_exp)[base / kGroup] : 0u);
            const Scale<kTopV> sv(group ? global<uint8_t>((const void*)pc.v_exp)[base / kGroup] : 0u);
            uint32_t fm[2], fv[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                fm[h] = load4<H>(pc.m, base + h * 128 + lane * 4, pc.n);
                fv[h] = load4<H>(pc.v, base + h * 128 + lane * 4, pc.n);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    m[h][i] = sm.value(fm[h], i);
                    v[h][i] = sv.value(fv[h], i);
                }
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                load4<H, float>(pc.m, base + h * 128 + lane * 4, pc.n, m[h]);
                load4<H, float>(pc.v, base + h * 128 + lane * 4, pc.n, v[h]);
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (m_out) store4<H, float>(m_out + pc.first_value, base + h * 128 + lane * 4, pc.n, m[h]);
            if (v_out) store4<H, float>(v_out + pc.first_value, base + h * 128 + lane * 4, pc.n, v[h]);
        }
    });
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
