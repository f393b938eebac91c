// Layer norm over the rows of a matrix, and its backward pass.
//   m = mean of x over a row, r = 1 / sqrt(mean of (x - m)^2 + eps), xh = (x - m) r, y = xh w + b
//   u = g_y w:  g_x = r (u - mean(u) - xh mean(u xh)),  g_w = sum over rows of g_y xh,  g_b = sum over rows of g_y
#include "hag_elem.hpp"

namespace hag {

__device__ __forceinline__ float block_sum(float v, float *lds) {
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) v += __shfl_xor(v, off);
    __syncthreads();
    if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < kBlock / kWave; ++w) v += lds[w];
    return v;
}

template <typename T, typename P>
__global__ __launch_bounds__(kBlock) void norm_kernel(const T *__restrict__ x, int64_t stride, int32_t d, const P *__restrict__ w, const P *__restrict__ b, float eps,
                                                      T *__restrict__ y, float *__restrict__ mean, float *__restrict__ rstd) {
    __shared__ float lds[kBlock / kWave];
    const int64_t row = blockIdx.x;
    const T *p = x + row * stride;
    // the mean is taken of the differences from the row's first element: rows of one value, however large, then have that mean and no deviation
    const float first = (float)p[0];
    float s = 0.f;
    for (int c = threadIdx.x; c < d; c += kBlock) s += (float)p[c] - first;
    const float m = first + block_sum(s, lds) / d;
    s = 0.f;
    for (int c = threadIdx.x; c < d; c += kBlock) { const float v = (float)p[c] - m; s += v * v; }
    const float r = 1.f / sqrtf(block_sum(s, lds) / d + eps);
    for (int c = threadIdx.x; c < d; c += kBlock) {
        const float xh = ((float)p[c] - m) * r;
        y[row * d + c] = (T)(xh * (w ? (float)w[c] : 1.f) + (b ? (float)b[c] : 0.f));
    }
    if (threadIdx.x == 0) {
        if (mean) mean[row] = m;
        if (rstd) rstd[row] = r;
    }
}

template <typename T, typename P>
__global__ __launch_bounds__(kBlock) void norm_grad_kernel(const T *__restrict__ gy, int64_t gy_stride, const T *__restrict__ x, int64_t stride, int32_t d,
                                                           const P *__restrict__ w, const float *__restrict__ mean, const float *__restrict__ rstd, T *__restrict__ gx) {
    __shared__ float lds[kBlock / kWave];
    const int64_t row = blockIdx.x;
    const T *p = x + row * stride, *g = gy + row * gy_stride;
    const float m = mean[row], r = rstd[row];
    float s1 = 0.f, s2 = 0.f;
    for (int c = threadIdx.x; c < d; c += kBlock) {
        const float u = (float)g[c] * (w ? (float)w[c] : 1.f);
        s1 += u;
        s2 += u * (((float)p[c] - m) * r);
    }
    s1 = block_sum(s1, lds) / d;
    s2 = block_sum(s2, lds) / d;
    for (int c = threadIdx.x; c < d; c += kBlock) {
        const float u = (float)g[c] * (w ? (float)w[c] : 1.f);
        gx[row * d + c] = (T)(r * (u - s1 - ((float)p[c] - m) * r * s2));
    }
}

// partial[slice] = the sums of a slice of the rows, [2, d]: g_w, g_b
template <typename T>
__global__ __launch_bounds__(kBlock) void norm_sums_kernel(const T *__restrict__ gy, int64_t gy_stride, const T *__restrict__ x, int64_t stride, int64_t n, int32_t d,
                                                           const float *__restrict__ mean, const float *__restrict__ rstd, float *__restrict__ partial) {
    __shared__ float lds[kBlock / kWave][2][kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, c = blockIdx.x * kWave + lane;
    float gw = 0.f, gb = 0.f;
    if (c < d) {
        for (int64_t row = (int64_t)blockIdx.y * (kBlock / kWave) + wave; row < n; row += (int64_t)gridDim.y * (kBlock / kWave)) {
            const float g = (float)gy[row * gy_stride + c];
            gw += g * (((float)x[row * stride + c] - mean[row]) * rstd[row]);
            gb += g;
        }
    }
    lds[wave][0][lane] = gw;
    lds[wave][1][lane] = gb;
    __syncthreads();
    if (wave > 0 || c >= d) return;
    for (int v = 1; v < kBlock / kWave; ++v) { gw += lds[v][0][lane]; gb += lds[v][1][lane]; }
    partial[((int64_t)blockIdx.y * 2) * d + c] = gw;
    partial[((int64_t)blockIdx.y * 2 + 1) * d + c] = gb;
}

template <typename P>
__global__ __launch_bounds__(kBlock) void norm_reduce_kernel(const float *__restrict__ partial, int32_t slices, int32_t d, P *__restrict__ g_w, P *__restrict__ g_b) {
    const int i = blockIdx.x * kBlock + threadIdx.x;
    if (i >= 2 * d) return;
    float sum = 0.f;
    for (int s = 0; s < slices; ++s) sum += partial[(int64_t)s * 2 * d + i];
    if (i < d) {
        if (g_w) g_w[i] = (P)sum;
    } else if (g_b) {
        g_b[i - d] = (P)sum;
    }
}

constexpr int kNormSlices = 128;

}  // namespace hag

using namespace hag;

extern "C" {

static const char *norm_refusal(int64_t n, int64_t d, hag_dtype_t dtype, hag_dtype_t param_dtype) {
    if (n < 0 || d <= 0 || n > 0x7fffffffLL || d > (1 << 20)) return "n must be in 0 .. 2^31 - 1, d in 1 .. 2^20";
    if (!elem_type(dtype)) return "elements are HAG_F32, HAG_BF16 or HAG_F16";
    if (param_dtype != dtype && param_dtype != HAG_F32) return "weight and bias have the elements' type or HAG_F32";
    return nullptr;
}

int hag_layer_norm(int64_t n, int64_t d, hag_dtype_t dtype, const void *x, int64_t x_stride, hag_dtype_t param_dtype, const void *weight, const void *bias, float eps, void *y,
                   float *mean, float *rstd, void *stream) {
    if (const char *why = norm_refusal(n, d, dtype, param_dtype)) { set_error(why); return HAG_EINVAL; }
    if (x_stride < 0) { set_error("negative row stride"); return HAG_EINVAL; }
    if (!(eps >= 0.f)) { set_error("eps must not be negative"); return HAG_EINVAL; }
    if (n == 0) return HAG_OK;
    if (!x || !y) { set_error("NULL pointer"); return HAG_EINVAL; }
    return elem_switch(dtype, [&](auto e) {
        using T = decltype(e);
        auto launch = [&](auto p) {
            using P = decltype(p);
            hipLaunchKernelGGL((norm_kernel<T, P>), dim3((unsigned)n), dim3(kBlock), 0, (hipStream_t)stream, (const T *)x, x_stride, (int32_t)d, (const P *)weight, (const P *)bias, eps,
                               (T *)y, mean, rstd);
            HIP_TRY(hipGetLastError());
            return (int)HAG_OK;
        };
        return param_dtype == dtype ? launch(T()) : launch(float());
    });
}

size_t hag_layer_norm_grad_workspace_bytes(int64_t n, int64_t d) {
    return norm_refusal(n, d, HAG_F32, HAG_F32) ? 0 : (size_t)kNormSlices * 2 * (size_t)d * sizeof(float);
}

int hag_layer_norm_grad(int64_t n, int64_t d, hag_dtype_t dtype, const void *g_y, int64_t g_y_stride, const void *x, int64_t x_stride, hag_dtype_t param_dtype, const void *weight,
                        const float *mean, const float *rstd, void *g_x, void *g_weight, void *g_bias, void *workspace, void *stream) {
    if (const char *why = norm_refusal(n, d, dtype, param_dtype)) { set_error(why); return HAG_EINVAL; }
    if (x_stride < 0 || g_y_stride < 0) { set_error("negative row stride"); return HAG_EINVAL; }
    const bool params = g_weight || g_bias;
    if ((n > 0 && (!g_y || !x || !mean || !rstd || !g_x)) || (params && !workspace)) { set_error("NULL pointer"); return HAG_EINVAL; }
    if ((uintptr_t)workspace & 15) { set_error("workspace must be 16-byte aligned"); return HAG_EINVAL; }
    hipStream_t s = (hipStream_t)stream;
    return elem_switch(dtype, [&](auto e) {
        using T = decltype(e);
        auto launch = [&](auto p) {
            using P = decltype(p);
            if (n > 0) {
                hipLaunchKernelGGL((norm_grad_kernel<T, P>), dim3((unsigned)n), dim3(kBlock), 0, s, (const T *)g_y, g_y_stride, (const T *)x, x_stride, (int32_t)d, (const P *)weight, mean,
                                   rstd, (T *)g_x);
                HIP_TRY(hipGetLastError());
            }
            if (params) {
                hipLaunchKernelGGL(norm_sums_kernel<T>, dim3((unsigned)((d + kWave - 1) / kWave), kNormSlices), dim3(kBlock), 0, s, (const T *)g_y, g_y_stride, (const T *)x, x_stride, n,
                                   (int32_t)d, mean, rstd, (float *)workspace);
                HIP_TRY(hipGetLastError());
                hipLaunchKernelGGL(norm_reduce_kernel<P>, dim3((unsigned)((2 * d + kBlock - 1) / kBlock)), dim3(kBlock), 0, s, (const float *)workspace, kNormSlices, (int32_t)d,
                                   (P *)g_weight, (P *)g_bias);
                HIP_TRY(hipGetLastError());
            }
            return (int)HAG_OK;
        };
        return param_dtype == dtype ? launch(T()) : launch(float());
    });
}

}  // extern "C"
