// Row-wise kernels of the 8-bit dense layers: codes and scales of a row, and
// activations put away in 8 bits and brought back.  All are bound by memory, a
// large copy reaching 4.96 TB/s: 131,072 rows of 4096 in bf16 take 0.31 ms for
// their codes (1.6 GB, 5.1 TB/s), 0.49 ms to put away and rewrite (2.7 GB, 5.5
// TB/s) and 0.28 ms to bring back (1.6 GB, 5.8 TB/s).
#include "dense8_rows.hpp"

namespace hpacml {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxBlocks = 1 << 14;   // the kernels loop beyond them

dim3 blocks_for(int64_t rows, int64_t per_block) {
    const int64_t n = (rows + per_block - 1) / per_block;
    return dim3((uint32_t)(n < kMaxBlocks ? n : kMaxBlocks));
}

// LANES lanes per row, HELD chunks of each lane in registers: rows up to
// LANES * HELD chunks are read once, longer ones a second time (from the
// caches) for their codes.
template <typename T, int LANES, int HELD>
__global__ void __launch_bounds__(kThreads) codes_kernel(const T *__restrict__ x, int64_t ldx, int64_t rows,
                                                         int32_t width, int8_t *__restrict__ codes, int32_t slabs,
                                                         float *__restrict__ scales) {
    constexpr int kRows = kThreads / LANES;
    const int lane = threadIdx.x % LANES, chunks = slabs * (kSlabBytes / kChunk);
    for (int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES; r < rows; r += (int64_t)gridDim.x * kRows) {
        const T *row = x + r * ldx;
        float v[HELD][kChunk];
        uint32_t top = 0;
        for (int c = lane; c < chunks; c += LANES * HELD) {
#pragma unroll
            for (int h = 0; h < HELD; ++h) {
                const int k = (c + h * LANES) * kChunk;
                load_chunk(row + k, width - k, v[h]);
            }
#pragma unroll
            for (int h = 0; h < HELD; ++h)
                top = max(top, top_bits(v[h]));
        }
        top = lanes_max<LANES>(top);
        const RowScale sc(top);
        if (lane == 0)
            scales[r] = sc.scale;
        for (int c = lane; c < chunks; c += LANES * HELD) {
#pragma unroll
            for (int h = 0; h < HELD; ++h) {
                const int at = c + h * LANES;
                if (at >= chunks)
                    break;
                if (chunks > LANES * HELD)
                    load_chunk(row + at * kChunk, width - at * kChunk, v[h]);
                *(uint2 *)(codes + blocked_offset(r, at * kChunk, slabs)) = sc.codes(v[h]);
            }
        }
    }
}

// A block of threads covers `cols` chunks (a power of two, at least the four
// of a block of channels) of kThreads / cols rows.
template <typename Z, typename A, bool RELU>
__global__ void __launch_bounds__(kThreads) save_kernel(hpacml8_checkpoint c, const Z *z, int64_t ldz,
                                                        A *a, int64_t lda, int cols_log) {
    const int col = threadIdx.x & ((1 << cols_log) - 1), per = kThreads >> cols_log;
    const int chunks = (c.width + 31) / 32 * 4;
    for (int64_t r = (int64_t)blockIdx.x * per + (threadIdx.x >> cols_log); r < c.rows; r += (int64_t)gridDim.x * per)
        for (int at = col; at < chunks; at += 1 << cols_log) {
            const int k = at * kChunk, n = c.width - k;
            float v[kChunk];
            load_chunk(z + r * ldz + k, n, v);
            if (RELU) {
#pragma unroll
                for (int e = 0; e < kChunk; ++e)
                    v[e] = relu_keep_nan(v[e]);
            }
            const uint32_t byte = block_exp(lanes_max<4>(top_bits(v)), RELU);
            const float f = block_factor(byte);
            uint32_t q[2] = {0, 0};
#pragma unroll
            for (int e = 0; e < kChunk; ++e)
                q[e / 4] |= block_code<RELU>(v[e], f) << (8 * (e % 4));
            *(uint2 *)((uint8_t *)c.codes + r * c.ld_codes + k) = uint2{q[0], q[1]};
            if ((at & 3) == 0)
                ((uint8_t *)c.exps)[r * c.ld_exps + at / 4] = (uint8_t)byte;
            if (a)
                store_chunk(a + r * lda + k, n, v);
        }
}

template <typename A, bool RELU>
__global__ void __launch_bounds__(kThreads) load_kernel(hpacml8_checkpoint c, A *__restrict__ a, int64_t lda,
                                                        int cols_log) {
    const int col = threadIdx.x & ((1 << cols_log) - 1), per = kThreads >> cols_log;
    const int chunks = (c.width + kChunk - 1) / kChunk;
    for (int64_t r = (int64_t)blockIdx.x * per + (threadIdx.x >> cols_log); r < c.rows; r += (int64_t)gridDim.x * per)
        for (int at = col; at < chunks; at += 1 << cols_log) {
            const int k = at * kChunk;
            const uint2 q = *(const uint2 *)((const uint8_t *)c.codes + r * c.ld_codes + k);
            const float s = block_scale(((const uint8_t *)c.exps)[r * c.ld_exps + at / 4]);
            float v[kChunk];
#pragma unroll
            for (int e = 0; e < kChunk; ++e)
                v[e] = block_value<RELU>(((e < 4 ? q.x : q.y) >> (8 * (e % 4))) & 0xFFu, s);
            store_chunk(a + r * lda + k, c.width - k, v);
        }
}

template <typename T, int LANES, int HELD>
void codes_as(const void *x, int64_t ldx, int64_t rows, int32_t width, int8_t *codes, int32_t slabs, float *scales,
              hipStream_t stream) {
    codes_kernel<T, LANES, HELD><<<blocks_for(rows, kThreads / LANES), kThreads, 0, stream>>>((const T *)x, ldx, rows,
                                                                                             width, codes, slabs, scales);
}

template <typename T>
void codes_of(const void *x, int64_t ldx, int64_t rows, int32_t width, int8_t *codes, float *scales, hipStream_t st) {
    const int32_t slabs = (int32_t)slabs_of(width), chunks = slabs * (kSlabBytes / kChunk);
    if (chunks <= 8)
        codes_as<T, 8, 1>(x, ldx, rows, width, codes, slabs, scales, st);
    else if (chunks <= 16)
        codes_as<T, 16, 1>(x, ldx, rows, width, codes, slabs, scales, st);
    else if (chunks <= 32)
        codes_as<T, 32, 1>(x, ldx, rows, width, codes, slabs, scales, st);
    else if (chunks <= 64)
        codes_as<T, 64, 1>(x, ldx, rows, width, codes, slabs, scales, st);
    else if (chunks <= 128)
        codes_as<T, 64, 2>(x, ldx, rows, width, codes, slabs, scales, st);
    else if (chunks <= 256)
        codes_as<T, 64, 4>(x, ldx, rows, width, codes, slabs, scales, st);
    else
        codes_as<T, 64, 8>(x, ldx, rows, width, codes, slabs, scales, st);
}

// log2 of the chunks a row of a block of threads covers: 4 .. 256
int cols_log(int chunks) {
    int l = 2;
    while ((1 << l) < chunks && (1 << l) < kThreads)
        ++l;
    return l;
}

template <typename Z, typename A>
void save_as(const hpacml8_checkpoint &c, const void *z, int64_t ldz, void *a, int64_t lda, hipStream_t stream) {
    const int l = cols_log((c.width + 31) / 32 * 4);
    const dim3 grid = blocks_for(c.rows, kThreads >> l);
    if (c.act == HPACML_ACT_RELU)
        save_kernel<Z, A, true><<<grid, kThreads, 0, stream>>>(c, (const Z *)z, ldz, (A *)a, lda, l);
    else
        save_kernel<Z, A, false><<<grid, kThreads, 0, stream>>>(c, (const Z *)z, ldz, (A *)a, lda, l);
}
template <typename A>
void load_as(const hpacml8_checkpoint &c, void *a, int64_t lda, hipStream_t stream) {
    const int l = cols_log((c.width + kChunk - 1) / kChunk);
    const dim3 grid = blocks_for(c.rows, kThreads >> l);
    if (c.act == HPACML_ACT_RELU)
        load_kernel<A, true><<<grid, kThreads, 0, stream>>>(c, (A *)a, lda, l);
    else
        load_kernel<A, false><<<grid, kThreads, 0, stream>>>(c, (A *)a, lda, l);
}

}  // namespace

hipError_t launch_codes_by_row(const void *x, int32_t dtype, int64_t ldx, int64_t rows, int32_t width, int8_t *codes,
                               float *scales, hipStream_t stream) {
    if (dtype == HPACML_F32)
        codes_of<float>(x, ldx, rows, width, codes, scales, stream);
    else
        codes_of<uint16_t>(x, ldx, rows, width, codes, scales, stream);
    return hipGetLastError();
}

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
