// Layer norm in training: forward pass with residual sum and statistics, backward pass with the gradients of gamma and beta.
#include <type_traits>

#include "ff_common.h"

namespace ff {

constexpr int kBackwardBlocks = 1024;    // partial sums of dgamma and dbeta

// sum of x over the block's 256 threads, the same in each
__device__ __forceinline__ float block_total(float x, float* part) {
    x = wave_sum(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

// one row per block, thread t holds channels t, t + 256, ...
template <typename T, int PER>
__global__ __launch_bounds__(256) void k_ln_forward_any(const T* x, const T* residual, const T* __restrict__ gamma, const T* __restrict__ beta,
                                                        T* sum, T* __restrict__ y, float* __restrict__ mean_out, float* __restrict__ rstd_out,
                                                        int64_t rows, int c, float eps) {
    __shared__ float part[4];
    const float inv_c = 1.f / (float)c;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const int64_t at = row * c;
        float v[PER], s = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int ch = threadIdx.x + 256 * i;
            v[i] = 0.f;
            if (ch < c) {
                v[i] = to_f32<T>(x[at + ch]);
                if (residual) {
                    const T kept = from_f32<T>(v[i] + to_f32<T>(residual[at + ch]));
                    sum[at + ch] = kept;
                    v[i] = to_f32<T>(kept);
                }
                s += v[i];
            }
        }
        const float mean = block_total(s, part) * inv_c;
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (threadIdx.x + 256 * i < c) q += (v[i] - mean) * (v[i] - mean);
        const float rstd = 1.f / sqrtf(block_total(q, part) * inv_c + eps);
        if (mean_out && threadIdx.x == 0) {
            mean_out[row] = mean;
            rstd_out[row] = rstd;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int ch = threadIdx.x + 256 * i;
            if (ch < c) y[at + ch] = from_f32<T>((v[i] - mean) * rstd * to_f32<T>(gamma[ch]) + to_f32<T>(beta[ch]));
        }
    }
}

template <typename T, int PER>
__global__ __launch_bounds__(256) void k_ln_backward_any(const T* __restrict__ s, const T* __restrict__ gamma, const float* __restrict__ mean_in,
                                                         const float* __restrict__ rstd_in, const T* dy, const T* dsum, T* dx,
                                                         float* __restrict__ partial, int64_t rows, int c, float eps) {
    __shared__ float part[4];
    const float inv_c = 1.f / (float)c;
    float dg[PER] = {}, db[PER] = {};
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const int64_t at = row * c;
        float u[PER], d[PER], t = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int ch = threadIdx.x + 256 * i;
            u[i] = d[i] = 0.f;
            if (ch < c) {
                u[i] = to_f32<T>(s[at + ch]);
                d[i] = to_f32<T>(dy[at + ch]);
                t += u[i];
            }
        }
        float mean, rstd;
        if (mean_in) {
            mean = mean_in[row];
            rstd = rstd_in[row];
        } else {
            mean = block_total(t, part) * inv_c;
            float q = 0.f;
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (threadIdx.x + 256 * i < c) q += (u[i] - mean) * (u[i] - mean);
            rstd = 1.f / sqrtf(block_total(q, part) * inv_c + eps);
        }
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int ch = threadIdx.x + 256 * i;
            if (ch < c) {
                u[i] = (u[i] - mean) * rstd;
                dg[i] += d[i] * u[i];
                db[i] += d[i];
                d[i] *= to_f32<T>(gamma[ch]);
                a += d[i];
                b += d[i] * u[i];
            }
        }
        a = block_total(a, part) * inv_c;
        b = block_total(b, part) * inv_c;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int ch = threadIdx.x + 256 * i;
            if (ch < c) {
                float r = rstd * (d[i] - a - u[i] * b);
                if (dsum) r += to_f32<T>(dsum[at + ch]);
                dx[at + ch] = from_f32<T>(r);
            }
        }
    }
    float* out = partial + (size_t)blockIdx.x * 2 * c;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int ch = threadIdx.x + 256 * i;
        if (ch < c) {
            out[ch] = dg[i];
            out[c + ch] = db[i];
        }
    }
}

// dgamma and dbeta from the blocks' partial sums, in their order
__global__ __launch_bounds__(256) void k_ln_join(const float* __restrict__ partial, int blocks, int c, bool accumulate,
                                                 float* __restrict__ dgamma, float* __restrict__ dbeta) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= 2 * c) return;
    float sum = 0.f;
    for (int b = 0; b < blocks; ++b) sum += partial[(size_t)b * 2 * c + i];
    float* to = i < c ? dgamma + i : dbeta + i - c;
    *to = accumulate ? *to + sum : sum;
}

static int backward_blocks(const ff_norm_desc& d) { return (int)(d.rows < kBackwardBlocks ? d.rows : kBackwardBlocks); }

size_t layernorm_backward_workspace(const ff_norm_desc& d) {
    const size_t n = (size_t)backward_blocks(d) * 2 * d.c * sizeof(float);
    return n < 256 ? 256 : (n + 255) & ~(size_t)255;
}

template <typename T>
static void forward_t(const ff_norm_desc& d, const void* x, const void* residual, const void* gamma, const void* beta, void* sum, void* y,
                      float* mean, float* rstd, hipStream_t stream) {
    const dim3 grid((unsigned)(d.rows < 4096 ? d.rows : 4096)), block(256);
    auto go = [&](auto per) {
        hipLaunchKernelGGL((k_ln_forward_any<T, decltype(per)::value>), grid, block, 0, stream, (const T*)x, (const T*)residual, (const T*)gamma,
                           (const T*)beta, (T*)sum, (T*)y, mean, rstd, d.rows, d.c, d.ln_eps);
    };
    if (d.c <= 256) go(std::integral_constant<int, 1>{});
    else if (d.c <= 1024) go(std::integral_constant<int, 4>{});
    else go(std::integral_constant<int, 32>{});
}

ff_status layernorm_forward_run(const ff_norm_desc& d, const void* x, const void* residual, const void* gamma, const void* beta, void* sum,
                                void* y, float* mean, float* rstd, hipStream_t stream) {
    Timed t(KK_LN_FORWARD, stream);
    if (d.dtype == FF_F32) forward_t<float>(d, x, residual, gamma, beta, sum, y, mean, rstd, stream);
    else forward_t<bf16_t>(d, x, residual, gamma, beta, sum, y, mean, rstd, stream);
    return check_launch("ff_layernorm_forward");
}

template <typename T>
static void backward_t(const ff_norm_desc& d, const void* s, const void* gamma, const float* mean, const float* rstd, const void* dy,
                       const void* dsum, void* dx, float* partial, hipStream_t stream) {
    const dim3 grid((unsigned)backward_blocks(d)), block(256);
    auto go = [&](auto per) {
        hipLaunchKernelGGL((k_ln_backward_any<T, decltype(per)::value>), grid, block, 0, stream, (const T*)s, (const T*)gamma, mean, rstd,
                           (const T*)dy, (const T*)dsum, (T*)dx, partial, d.rows, d.c, d.ln_eps);
    };
    if (d.c <= 256) go(std::integral_constant<int, 1>{});
    else if (d.c <= 1024) go(std::integral_constant<int, 4>{});
    else go(std::integral_constant<int, 32>{});
}

ff_status layernorm_backward_run(const ff_norm_desc& d, const void* s, const void* gamma, const float* mean, const float* rstd,
                                 const void* dy, const void* dsum, void* dx, float* dgamma, float* dbeta, bool accumulate, void* ws,
                                 hipStream_t stream) {
    if (d.rows > 0) {
        Timed t(KK_LN_BACKWARD, stream);
        if (d.dtype == FF_F32) backward_t<float>(d, s, gamma, mean, rstd, dy, dsum, dx, (float*)ws, stream);
        else backward_t<bf16_t>(d, s, gamma, mean, rstd, dy, dsum, dx, (float*)ws, stream);
    }
    Timed t(KK_LN_JOIN, stream);
    hipLaunchKernelGGL(k_ln_join, dim3((2 * d.c + 255) / 256), dim3(256), 0, stream, (const float*)ws, backward_blocks(d), d.c, accumulate,
                       dgamma, dbeta);
    return check_launch("ff_layernorm_backward");
}

}  // namespace ff
