// Group norm with an activation, channels last, and its backward pass.
#include "dense8.hpp"
#include "group_norm.hpp"
#include "hpacmlt.h"

namespace hpacml {

namespace {

__device__ __forceinline__ float sigmoid(float z) { return 1.f / (1.f + expf(-z)); }

__device__ __forceinline__ float activation(float z, int32_t act) {
    if (act == HPACML_ACT_RELU)
        return relu_keep_nan(z);
    return act == HPACMLT_ACT_SILU ? z * sigmoid(z) : z;
}
// g = dy act'(z)
__device__ __forceinline__ float activation_gradient(float dy, float z, int32_t act) {
    if (act == HPACML_ACT_RELU)
        return z <= 0.f ? 0.f : dy;
    if (act == HPACMLT_ACT_SILU) {
        const float s = sigmoid(z);
        return dy * (s * (1.f + z * (1.f - s)));
    }
    return dy;
}

__device__ __forceinline__ double join_block(double t, double (&of_wave)[4]) {
#pragma unroll
    for (int s = 1; s < 64; s *= 2)
        t += __shfl_xor(t, s);
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        of_wave[threadIdx.x >> 6] = t;
    __syncthreads();
    return (of_wave[0] + of_wave[1]) + (of_wave[2] + of_wave[3]);
}

// A block per image and group.
template <typename T>
__global__ __launch_bounds__(256) void norm_kernel(GroupNorm a) {
    __shared__ double of_wave[4];
    const int per = a.channels / a.groups;
    const int64_t image = blockIdx.x / a.groups, n = a.points * per;
    const int c0 = (int)(blockIdx.x % a.groups) * per;
    const T *x = (const T *)a.x + image * a.points * a.ldx + c0;
    double t = 0;
    for (int64_t i = threadIdx.x; i < n; i += 256)
        t += load_value(x + i / per * a.ldx + i % per);
    const float mean = (float)(join_block(t, of_wave) / (double)n);
    t = 0;
    for (int64_t i = threadIdx.x; i < n; i += 256) {
        const double d = load_value(x + i / per * a.ldx + i % per) - mean;
        t += d * d;
    }
    const float rstd = (float)(1.0 / sqrt(join_block(t, of_wave) / (double)n + (double)a.eps));
    for (int64_t i = threadIdx.x; i < n; i += 256) {
        const int c = (int)(i % per);
        const float z = __builtin_fmaf(load_value(x + i / per * a.ldx + c) - mean, rstd * (a.gamma ? a.gamma[c0 + c] : 1.f), a.beta ? a.beta[c0 + c] : 0.f);
        store_value((T *)a.y + (image * a.points + i / per) * a.ldy + c0 + c, activation(z, a.act));
    }
    if (threadIdx.x == 0 && a.mean) {
        a.mean[blockIdx.x] = mean;
        a.rstd[blockIdx.x] = rstd;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void dx_kernel(GroupNorm a) {
    __shared__ double of_wave[4];
    const int per = a.channels / a.groups;
    const int64_t image = blockIdx.x / a.groups, n = a.points * per;
    const int c0 = (int)(blockIdx.x % a.groups) * per;
    const float mean = a.mean[blockIdx.x], rstd = a.rstd[blockIdx.x];
    auto value = [&](int64_t i, float &g, float &h) {
        const int c = c0 + (int)(i % per);
        const int64_t row = image * a.points + i / per;
        const float gamma = a.gamma ? a.gamma[c] : 1.f, d = load_value((const T *)a.x + row * a.ldx + c) - mean;
        const float z = __builtin_fmaf(d, rstd * gamma, a.beta ? a.beta[c] : 0.f);
        g = activation_gradient(load_value((const T *)a.dy + row * a.lddy + c), z, a.act) * gamma;
        h = d * rstd;
    };
    double t = 0, u = 0;
    for (int64_t i = threadIdx.x; i < n; i += 256) {
        float g, h;
        value(i, g, h);
        t += g;
        u += (double)g * h;
    }
    const float m1 = (float)(join_block(t, of_wave) / (double)n), m2 = (float)(join_block(u, of_wave) / (double)n);
    for (int64_t i = threadIdx.x; i < n; i += 256) {
        float g, h;
        value(i, g, h);
        store_value((T *)a.y + (image * a.points + i / per) * a.ldy + c0 + i % per, rstd * (g - m1 - h * m2));
    }
}

// A block per channel.
template <typename T>
__global__ __launch_bounds__(256) void parameters_kernel(GroupNorm a) {
    __shared__ double of_wave[4];
    const int c = blockIdx.x, group = c / (a.channels / a.groups);
    const float gamma = a.gamma ? a.gamma[c] : 1.f, beta = a.beta ? a.beta[c] : 0.f;
    double t = 0, u = 0;
    for (int64_t row = threadIdx.x; row < a.images * a.points; row += 256) {
        const int64_t at = row / a.points * a.groups + group;
        const float d = load_value((const T *)a.x + row * a.ldx + c) - a.mean[at];
        const float g = activation_gradient(load_value((const T *)a.dy + row * a.lddy + c), __builtin_fmaf(d, a.rstd[at] * gamma, beta), a.act);
        t += g;
        u += (double)g * (d * a.rstd[at]);
    }
    const double db = join_block(t, of_wave), dg = join_block(u, of_wave);
    if (threadIdx.x == 0) {
        if (a.dgamma)
            a.dgamma[c] = (float)dg + (a.accumulate ? a.dgamma[c] : 0.f);
        if (a.dbeta)
            a.dbeta[c] = (float)db + (a.accumulate ? a.dbeta[c] : 0.f);
    }
}

template <typename T>
hipError_t launch_backward(const GroupNorm &a, hipStream_t stream) {
    if (a.y && a.images)
        dx_kernel<T><<<(uint32_t)(a.images * a.groups), 256, 0, stream>>>(a);
    if (a.dgamma || a.dbeta)
        parameters_kernel<T><<<a.channels, 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

int64_t group_norm_scratch(int32_t dtype, int64_t images, int64_t points, int32_t channels, int32_t groups, bool backward) { return 0; }

hipError_t launch_group_norm(const GroupNorm &a, int32_t dtype, hipStream_t stream) {
    if (a.images == 0)
        return hipSuccess;
    if (dtype == HPACML_F32)
        norm_kernel<float><<<(uint32_t)(a.images * a.groups), 256, 0, stream>>>(a);
    else
        norm_kernel<uint16_t><<<(uint32_t)(a.images * a.groups), 256, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_group_norm_backward(const GroupNorm &a, int32_t dtype, hipStream_t stream) {
    return dtype == HPACML_F32 ? launch_backward<float>(a, stream) : launch_backward<uint16_t>(a, stream);
}

}  // namespace hpacml
