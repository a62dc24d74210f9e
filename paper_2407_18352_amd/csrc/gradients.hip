// The norm of many gradients, and clipping.
//
// One launch reads every value once: a block goes from chunk to chunk of the
// whole set (runs of a few thousand values of one gradient) and leaves one
// partial result.  Squares and their sums are in 64 bits: a square of any fp32
// value is exact and in range there.  The second launch joins the partial
// results, every block all of them in the same order, and scales.
#include "dense8.hpp"
#include "gradients.hpp"
#include "hpacmlt.h"

namespace hpacml {

namespace {

// a partial result: the bits of a 64-bit sum, or of the largest magnitude in fp32
template <bool MAX>
struct Partial {
    static __device__ __forceinline__ uint64_t join(uint64_t a, uint64_t b) {
        if (MAX)
            return a > b ? a : b;         // a NaN's are above every number's
        return __builtin_bit_cast(uint64_t, __builtin_bit_cast(double, a) + __builtin_bit_cast(double, b));
    }
    static __device__ __forceinline__ uint64_t with(uint64_t a, float v) {
        if (MAX)
            return join(a, __builtin_bit_cast(uint32_t, v) & 0x7FFFFFFFu);
        const double d = v;
        return __builtin_bit_cast(uint64_t, __builtin_fma(d, d, __builtin_bit_cast(double, a)));
    }
};

template <bool MAX>
__device__ __forceinline__ uint64_t join_block(uint64_t t, uint64_t (&of_wave)[4]) {
#pragma unroll
    for (int s = 1; s < 64; s *= 2)
        t = Partial<MAX>::join(t, (uint64_t)__shfl_xor((unsigned long long)t, s));
    if ((threadIdx.x & 63) == 0)
        of_wave[threadIdx.x >> 6] = t;
    __syncthreads();
    return Partial<MAX>::join(Partial<MAX>::join(of_wave[0], of_wave[1]), Partial<MAX>::join(of_wave[2], of_wave[3]));
}

template <typename T>
constexpr int per_load = 16 / sizeof(T);

template <typename T>
__device__ __forceinline__ void values_of(u32x4 u, float (&v)[per_load<T>]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t w = u[e];
        if constexpr (sizeof(T) == 4)
            v[e] = __builtin_bit_cast(float, w);
        else {
            v[2 * e] = __builtin_bit_cast(float, w << 16);
            v[2 * e + 1] = __builtin_bit_cast(float, w & 0xFFFF0000u);
        }
    }
}

template <bool MAX, typename T>
__device__ __forceinline__ uint64_t chunk_norm(const T *p, int32_t count, uint64_t t) {
    constexpr int kPer = per_load<T>;
    const int32_t whole = count / kPer;
#pragma unroll 4
    for (int32_t i = threadIdx.x; i < whole; i += 256) {
        float v[kPer];
        values_of<T>(*(const u32x4_any *)(p + i * kPer), v);
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            t = Partial<MAX>::with(t, v[e]);
    }
    const int32_t i = whole * kPer + threadIdx.x;
    return i < count ? Partial<MAX>::with(t, load_value(p + i)) : t;
}

template <bool MAX>
__global__ __launch_bounds__(256) void norm_kernel(const GradChunk *chunks, int64_t n, uint64_t *partial) {
    __shared__ uint64_t of_wave[4];
    uint64_t t = 0;
    for (int64_t c = blockIdx.x; c < n; c += gridDim.x) {
        const GradChunk g = chunks[c];
        t = g.types & 1 ? chunk_norm<MAX>((const uint16_t *)g.from, g.count, t) : chunk_norm<MAX>((const float *)g.from, g.count, t);
    }
    t = join_block<MAX>(t, of_wave);
    if (threadIdx.x == 0)
        partial[blockIdx.x] = t;
}

// the norm of `blocks` partial results, in 64 bits
template <bool MAX>
__device__ __forceinline__ double joined(const uint64_t *partial, int blocks, uint64_t (&of_wave)[4]) {
    uint64_t t = 0;
    for (int i = threadIdx.x; i < blocks; i += 256)
        t = Partial<MAX>::join(t, partial[i]);
    t = join_block<MAX>(t, of_wave);
    return MAX ? (double)__builtin_bit_cast(float, (uint32_t)t) : sqrt(__builtin_bit_cast(double, t));
}

template <bool MAX>
__global__ __launch_bounds__(256) void join_norm_kernel(const uint64_t *partial, int blocks, float *norm) {
    __shared__ uint64_t of_wave[4];
    const double d = joined<MAX>(partial, blocks, of_wave);
    if (threadIdx.x == 0)
        *norm = (float)d;
}

template <typename T, typename U>
__device__ __forceinline__ void chunk_scale(const T *p, U *to, int32_t count, float f) {
    constexpr int kPer = per_load<T>;
    const int32_t whole = count / kPer;
#pragma unroll 4
    for (int32_t i = threadIdx.x; i < whole; i += 256) {
        float v[kPer];
        values_of<T>(*(const u32x4_any *)(p + i * kPer), v);
        u32x4 out[kPer * sizeof(U) / 16 ? kPer * sizeof(U) / 16 : 1];
        if constexpr (sizeof(U) == 4) {
#pragma unroll
            for (int e = 0; e < kPer; ++e)
                out[e / 4][e % 4] = __builtin_bit_cast(uint32_t, v[e] * f);
#pragma unroll
            for (int e = 0; e < kPer / 4; ++e)
                *(u32x4_any *)(to + i * kPer + e * 4) = out[e];
        } else if constexpr (kPer == 8) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                out[0][e] = pack_bf16(v[2 * e] * f, v[2 * e + 1] * f);
            *(u32x4_any *)(to + i * kPer) = out[0];
        } else {
#pragma unroll
            for (int e = 0; e < kPer; ++e)
                store_value(to + i * kPer + e, v[e] * f);
        }
    }
    const int32_t i = whole * kPer + threadIdx.x;
    if (i < count)
        store_value(to + i, load_value(p + i) * f);
}

template <bool MAX>
__global__ __launch_bounds__(256) void clip_kernel(const GradChunk *chunks, int64_t n, const uint64_t *partial, int blocks, double most, float *norm) {
    __shared__ uint64_t of_wave[4];
    const double d = joined<MAX>(partial, blocks, of_wave), q = most / (d + 1e-6);
    const float f = (float)(q > 1.0 ? 1.0 : q);         // a NaN stays one
    if (blockIdx.x == 0 && threadIdx.x == 0)
        *norm = (float)d;
    for (int64_t c = blockIdx.x; c < n; c += gridDim.x) {
        const GradChunk g = chunks[c];
        if (f == 1.f && g.from == g.to)
            continue;
        if (g.types == 0)
            chunk_scale((const float *)g.from, (float *)g.to, g.count, f);
        else if (g.types == 1)
            chunk_scale((const uint16_t *)g.from, (float *)g.to, g.count, f);
        else if (g.types == 2)
            chunk_scale((const float *)g.from, (uint16_t *)g.to, g.count, f);
        else
            chunk_scale((const uint16_t *)g.from, (uint16_t *)g.to, g.count, f);
    }
}

int blocks_for(int64_t n) { return n < kGradBlocks ? (int)n : kGradBlocks; }

hipError_t launch_partial(const GradChunk *chunks, int64_t n, int32_t kind, void *partial, hipStream_t stream) {
    if (n == 0)
        return hipSuccess;
    if (kind == HPACMLT_NORM_MAX)
        norm_kernel<true><<<blocks_for(n), 256, 0, stream>>>(chunks, n, (uint64_t *)partial);
    else
        norm_kernel<false><<<blocks_for(n), 256, 0, stream>>>(chunks, n, (uint64_t *)partial);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_grad_norm(const GradChunk *chunks, int64_t n, int32_t kind, float *norm, void *partial, hipStream_t stream) {
    const hipError_t e = launch_partial(chunks, n, kind, partial, stream);
    if (e != hipSuccess)
        return e;
    if (kind == HPACMLT_NORM_MAX)
        join_norm_kernel<true><<<1, 256, 0, stream>>>((const uint64_t *)partial, blocks_for(n), norm);
    else
        join_norm_kernel<false><<<1, 256, 0, stream>>>((const uint64_t *)partial, blocks_for(n), norm);
    return hipGetLastError();
}

hipError_t launch_grad_clip(const GradChunk *chunks, int64_t n, int32_t kind, double most, float *norm, void *partial, hipStream_t stream) {
    const hipError_t e = launch_partial(chunks, n, kind, partial, stream);
    if (e != hipSuccess)
        return e;
    const int grid = n ? blocks_for(n) : 1;
    if (kind == HPACMLT_NORM_MAX)
        clip_kernel<true><<<grid, 256, 0, stream>>>(chunks, n, (const uint64_t *)partial, blocks_for(n), most, norm);
    else
        clip_kernel<false><<<grid, 256, 0, stream>>>(chunks, n, (const uint64_t *)partial, blocks_for(n), most, norm);
    return hipGetLastError();
}

}  // namespace hpacml
