// The norm of many gradients, and clipping.
//
// One launch reads every value once: a block goes from chunk to chunk of the
// whole set (runs of a few thousand values of one gradient) and leaves one
// partial result.  134 million values from bf16 to fp32 take 231 us, of which 80 are
// the norm (268 MB, beside the write-back of the results before) and 148 the
// scaling (5.4 TB/s); the gradients of a small model 9 us, two launches.  Squares and their sums are in 64 bits: a square of any fp32
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

// f(index of the load's first value, its words) for the thread's whole loads of a
// run, eight under way together, and g(index) for a value of its end.
template <typename T, typename F, typename G>
__device__ __forceinline__ void over_chunk(const T *p, int32_t count, F f, G g) {
    constexpr int kPer = per_load<T>, kAtOnce = 8;
    const int32_t whole = count / kPer;
    int32_t i = threadIdx.x;
    for (; i + (kAtOnce - 1) * 256 < whole; i += kAtOnce * 256) {
        u32x4 w[kAtOnce];
#pragma unroll
        for (int b = 0; b < kAtOnce; ++b)
            w[b] = *(const u32x4_any *)(p + (i + b * 256) * kPer);
#pragma unroll
        for (int b = 0; b < kAtOnce; ++b)
            f((i + b * 256) * kPer, w[b]);
    }
    for (; i < whole; i += 256)
        f(i * kPer, *(const u32x4_any *)(p + i * kPer));
    const int32_t end = whole * kPer + (int32_t)threadIdx.x;
    if (end < count)
        g(end);
}

// into four sums: one would wait for itself at every value
template <bool MAX, typename T>
__device__ __forceinline__ void chunk_norm(const T *p, int32_t count, uint64_t (&t)[4]) {
    over_chunk(p, count,
               [&](int32_t, u32x4 w) {
                   float v[per_load<T>];
                   values_of<T>(w, v);
#pragma unroll
                   for (int e = 0; e < per_load<T>; ++e)
                       t[e % 4] = Partial<MAX>::with(t[e % 4], v[e]);
               },
               [&](int32_t i) { t[0] = Partial<MAX>::with(t[0], load_value(p + i)); });
}

template <bool MAX>
__global__ __launch_bounds__(256) void norm_kernel(const GradChunk *chunks, int64_t n, uint64_t *partial) {
    __shared__ uint64_t of_wave[4];
    uint64_t sums[4] = {0, 0, 0, 0};
    GradChunk next = chunks[blockIdx.x];
    for (int64_t c = blockIdx.x; c < n; c += gridDim.x) {
        const GradChunk g = next;
        next = chunks[min(c + gridDim.x, n - 1)];
        if (g.types & 1)
            chunk_norm<MAX>((const uint16_t *)g.from, g.count, sums);
        else
            chunk_norm<MAX>((const float *)g.from, g.count, sums);
    }
    uint64_t t = Partial<MAX>::join(Partial<MAX>::join(sums[0], sums[1]), Partial<MAX>::join(sums[2], sums[3]));
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
    over_chunk(p, count,
               [&](int32_t i, u32x4 w) {
                   float v[kPer];
                   values_of<T>(w, v);
                   if constexpr (sizeof(U) == 4) {
#pragma unroll
                       for (int q = 0; q < kPer / 4; ++q) {
                           f32x4 out;
#pragma unroll
                           for (int e = 0; e < 4; ++e)
                               out[e] = v[q * 4 + e] * f;
                           *(f32x4_any *)(to + i + q * 4) = out;
                       }
                   } else if constexpr (kPer == 8) {
                       u32x4 out;
#pragma unroll
                       for (int e = 0; e < 4; ++e)
                           out[e] = pack_bf16(v[2 * e] * f, v[2 * e + 1] * f);
                       *(u32x4_any *)(to + i) = out;
                   } else {
                       typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
                       typedef u32x2 __attribute__((aligned(2))) u32x2_any;
                       *(u32x2_any *)(to + i) = u32x2{pack_bf16(v[0] * f, v[1] * f), pack_bf16(v[2] * f, v[3] * f)};
                   }
               },
               [&](int32_t i) { store_value(to + i, load_value(p + i) * f); });
}

template <bool MAX>
__global__ __launch_bounds__(256) void clip_kernel(const GradChunk *chunks, int64_t n, const uint64_t *partial, int blocks, double most, float *norm) {
    __shared__ uint64_t of_wave[4];
    GradChunk next{};
    if (n > 0)
        next = chunks[blockIdx.x];
    const double d = joined<MAX>(partial, blocks, of_wave), q = most / (d + 1e-6);
    const float f = (float)(q > 1.0 ? 1.0 : q);         // a NaN stays one
    if (blockIdx.x == 0 && threadIdx.x == 0)
        *norm = (float)d;
    for (int64_t c = blockIdx.x; c < n; c += gridDim.x) {
        const GradChunk g = next;
        next = chunks[min(c + gridDim.x, n - 1)];
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
