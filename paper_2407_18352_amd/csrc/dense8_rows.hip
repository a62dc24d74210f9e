// Row-wise kernels of the 8-bit dense layers: codes and scales of a row, and
// activations put away in 8 bits and brought back.  All are bound by memory.
#include "dense8.hpp"

namespace hpacml {

namespace {

constexpr int kThreads = 256;
constexpr int64_t kMaxBlocks = 1 << 16;   // the kernels loop beyond them

dim3 blocks_for(int64_t items, int64_t per_block) {
    const int64_t n = (items + per_block - 1) / per_block;
    return dim3((uint32_t)(n < kMaxBlocks ? n : kMaxBlocks));
}

__device__ __forceinline__ uint32_t wave_max(uint32_t v, int lanes) {
    for (int d = lanes / 2; d > 0; d /= 2)
        v = max(v, (uint32_t)__shfl_xor((int)v, d));
    return v;
}

// One wave per row: the largest magnitude (as bits, so that an infinity or a
// NaN is the largest), then the codes.
template <typename T>
__global__ void __launch_bounds__(kThreads) codes_kernel(const T *__restrict__ x, int64_t ldx, int64_t rows,
                                                         int32_t width, int8_t *__restrict__ codes, int64_t pitch,
                                                         float *__restrict__ scales) {
    const int lane = threadIdx.x & 63;
    for (int64_t r = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6); r < rows;
         r += (int64_t)gridDim.x * (kThreads / 64)) {
        const T *row = x + r * ldx;
        uint32_t top = 0;
        for (int k = lane; k < width; k += 64)
            top = max(top, __builtin_bit_cast(uint32_t, load_value(row + k)) & 0x7FFFFFFFu);
        top = wave_max(top, 64);
        const float amax = __builtin_bit_cast(float, top);
        const bool finite = top < 0x7F800000u, live = finite && amax >= 0x1p-119f;
        const float inv = live ? 127.f / amax : 0.f;
        if (lane == 0)
            scales[r] = !finite ? __builtin_nanf("") : live ? amax / 127.f : 0.f;
        for (int k = lane; k < pitch; k += 64)
            codes[r * pitch + k] = k < width && live ? (int8_t)rintf(load_value(row + k) * inv) : (int8_t)0;
    }
}

// 32 lanes per block of channels.
template <typename Z, typename A, bool RELU>
__global__ void __launch_bounds__(kThreads) save_kernel(hpacml8_checkpoint c, const Z *__restrict__ z, int64_t ldz,
                                                        A *a, int64_t lda) {
    const int64_t blocks = (c.width + 31) / 32;
    for (int64_t id = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); id < c.rows * blocks;
         id += (int64_t)gridDim.x * (kThreads / 32)) {
        const int64_t r = id / blocks, blk = id - r * blocks;
        const int k = (int)blk * 32 + (threadIdx.x & 31);
        float v = 0.f;
        if (k < c.width) {
            v = load_value(z + r * ldz + k);
            if (RELU)
                v = relu_keep_nan(v);
        }
        const uint32_t e = block_exp(wave_max(__builtin_bit_cast(uint32_t, v) & 0x7FFFFFFFu, 32), RELU);
        ((uint8_t *)c.codes)[r * c.ld_codes + k] = (uint8_t)block_code<RELU>(v, block_factor(e));
        if ((threadIdx.x & 31) == 0)
            ((uint8_t *)c.exps)[r * c.ld_exps + blk] = (uint8_t)e;
        if (a && k < c.width)
            store_value(a + r * lda + k, v);
    }
}

template <typename A, bool RELU>
__global__ void __launch_bounds__(kThreads) load_kernel(hpacml8_checkpoint c, A *__restrict__ a, int64_t lda) {
    for (int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x; id < c.rows * c.width;
         id += (int64_t)gridDim.x * kThreads) {
        const int64_t r = id / c.width, k = id - r * c.width;
        const float s = block_scale(((const uint8_t *)c.exps)[r * c.ld_exps + k / 32]);
        store_value(a + r * lda + k, block_value<RELU>(((const uint8_t *)c.codes)[r * c.ld_codes + k], s));
    }
}

}  // namespace

hipError_t launch_codes_by_row(const void *x, int32_t dtype, int64_t ldx, int64_t rows, int32_t width, int8_t *codes,
                               int64_t pitch, float *scales, hipStream_t stream) {
    const dim3 grid = blocks_for(rows, kThreads / 64);
    if (dtype == HPACML_F32)
        codes_kernel<float><<<grid, kThreads, 0, stream>>>((const float *)x, ldx, rows, width, codes, pitch, scales);
    else
        codes_kernel<uint16_t><<<grid, kThreads, 0, stream>>>((const uint16_t *)x, ldx, rows, width, codes, pitch,
                                                              scales);
    return hipGetLastError();
}

namespace {
template <typename Z, typename A>
void save_as(const hpacml8_checkpoint &c, const void *z, int64_t ldz, void *a, int64_t lda, hipStream_t stream) {
    const dim3 grid = blocks_for(c.rows * ((c.width + 31) / 32), kThreads / 32);
    if (c.act == HPACML_ACT_RELU)
        save_kernel<Z, A, true><<<grid, kThreads, 0, stream>>>(c, (const Z *)z, ldz, (A *)a, lda);
    else
        save_kernel<Z, A, false><<<grid, kThreads, 0, stream>>>(c, (const Z *)z, ldz, (A *)a, lda);
}
template <typename A>
void load_as(const hpacml8_checkpoint &c, void *a, int64_t lda, hipStream_t stream) {
    const dim3 grid = blocks_for(c.rows * c.width, kThreads);
    if (c.act == HPACML_ACT_RELU)
        load_kernel<A, true><<<grid, kThreads, 0, stream>>>(c, (A *)a, lda);
    else
        load_kernel<A, false><<<grid, kThreads, 0, stream>>>(c, (A *)a, lda);
}
}  // namespace

hipError_t launch_checkpoint_save(const hpacml8_checkpoint &c, const void *z, int32_t z_dtype, int64_t ldz, void *a,
                                  int32_t a_dtype, int64_t lda, hipStream_t stream) {
    if (z_dtype == HPACML_F32 && a_dtype == HPACML_F32)
        save_as<float, float>(c, z, ldz, a, lda, stream);
    else if (z_dtype == HPACML_F32)
        save_as<float, uint16_t>(c, z, ldz, a, lda, stream);
    else if (a_dtype == HPACML_F32)
        save_as<uint16_t, float>(c, z, ldz, a, lda, stream);
    else
        save_as<uint16_t, uint16_t>(c, z, ldz, a, lda, stream);
    return hipGetLastError();
}

hipError_t launch_checkpoint_load(const hpacml8_checkpoint &c, void *a, int32_t a_dtype, int64_t lda,
                                  hipStream_t stream) {
    if (a_dtype == HPACML_F32)
        load_as<float>(c, a, lda, stream);
    else
        load_as<uint16_t>(c, a, lda, stream);
    return hipGetLastError();
}

}  // namespace hpacml
