// Matrices in 8-bit floating point with a scale for each block of 128 values:
// their order in memory, launchers, and the device arithmetic they share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dense8.hpp"
#include "f8_rules.hpp"

namespace hpacml {
namespace f8 {

// Codes lie as the matrix instruction reads them: units of 32 rows x 64 values
// (2 KB), those of 32 rows after one another, an even number of them (whole
// blocks of 128 values).  In a unit lane l of a wave has row l % 32 and the 32
// values from 32 (l / 32) on, its first 16 at 16 l, the others 1 KB behind: a
// wave's 16-byte reads, from memory or LDS, are 1 KB in one piece.  Scales are
// the exponents' bytes e + 127; those of 128 rows and a block are 32 words, row
// r's in byte r / 32 of word r % 32, so that one word serves the four matrix
// instructions of 128 rows (they select a byte of it).  What pads the last rows
// and blocks has codes 0 and some finite scale.
constexpr int kUnit = 2048;
// a launch has fewer than 2^32 threads, and quantizing has 256 for each 128 x 128
constexpr bool too_many_blocks(int64_t rows, int64_t width) { return blocks_of(rows) * blocks_of(width) >= 1 << 24; }
constexpr int64_t row_units(int64_t rows) { return (rows + 31) / 32; }
constexpr int64_t codes_bytes(int64_t rows, int64_t width) { return row_units(rows) * blocks_of(width) * 2 * kUnit; }
constexpr int64_t scales_bytes(int64_t rows, int64_t width) { return (rows + 127) / 128 * blocks_of(width) * 128; }
// of value k of a row
__host__ __device__ constexpr int64_t code_offset(int64_t row, int64_t k, int64_t blocks) {
    return ((row >> 5) * blocks * 2 + (k >> 6)) * kUnit + ((k >> 4) & 1) * 1024 + (((k >> 5) & 1) * 32 + (row & 31)) * 16 + (k & 15);
}
// of block kb of a row
__host__ __device__ constexpr int64_t scale_offset(int64_t row, int64_t kb, int64_t blocks) {
    return ((row >> 7) * blocks + kb) * 128 + (row & 31) * 4 + ((row >> 5) & 3);
}

struct Matrix {
    char *codes, *scales;
    int64_t rows, width;
};

// ---- launchers ------------------------------------------------------------------

struct QuantizeArgs {
    const void *x, *y;      // y: x counts as 0 where y <= 0 (NULL: nowhere)
    int64_t ldx, ldy, rows, width;
    Matrix by_row, by_column;   // codes NULL: not wanted
    float *sums;            // column sums of 128 rows each, [blocks of rows][width] (NULL: not wanted)
    int32_t square;
};
hipError_t launch_quantize(const QuantizeArgs &a, int32_t dtype, hipStream_t stream);
hipError_t launch_load(const Matrix &m, void *x, int32_t dtype, int64_t ldx, hipStream_t stream);

// y (+)= act(p q^T + b).  partial: room for product_partial_bytes.
struct ProductArgs {
    Matrix p, q;
    const float *b;
    void *y;
    int64_t ldy;
    int32_t relu, accumulate;
    float *partial;
};
int64_t product_partial_bytes(int64_t p_rows, int64_t q_rows, int64_t width);
hipError_t launch_product(const ProductArgs &a, int32_t y_dtype, hipStream_t stream);

// of few_rows
hipError_t launch_product_few(const ProductArgs &a, int32_t y_dtype, hipStream_t stream);
// the same for rows x, whose codes it forms (of a.p: the rows)
hipError_t launch_linear_few(const ProductArgs &a, const void *x, int32_t x_dtype, int64_t ldx, int32_t y_dtype, hipStream_t stream);

// ---- device arithmetic --------------------------------------------------------------

typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// The scale's byte of a block whose largest magnitude has these bits: 448 is
// 1.75 * 2^8, so 2^e is 2^-8 of the magnitude's power of two, or twice that
// above 1.75 of it.  From 0x1.Fp127 on, which would round to 2^128: 255.
__device__ __forceinline__ uint32_t scale_byte(uint32_t most) {
    const int32_t b = (int32_t)((most + 0x1FFFFFu) >> 23) - 8;
    return most >= 0x7F780000u ? 255u : (uint32_t)max(b, 1);
}
// 2^-e
__device__ __forceinline__ float scale_factor(uint32_t byte) { return __builtin_bit_cast(float, (254u - byte) << 23); }

// four codes
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float factor) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * factor, b * factor, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * factor, d * factor, w, true);
}
constexpr uint32_t kNanCodes = 0x7F7F7F7Fu;      // of a block whose scale's byte is 255

__device__ __forceinline__ uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7FFFFFFFu; }

// 16 neighbouring values, as they lie in memory
template <typename X>
struct Sixteen {
    static constexpr int kWords = (int)sizeof(X);
    u32x4 w[kWords];
    __device__ __forceinline__ void load(const X *p) {
#pragma unroll
        for (int i = 0; i < kWords; ++i)
            w[i] = *(const u32x4_any *)(p + i * (16 / kWords));
    }
    __device__ __forceinline__ void values(float (&v)[16]) const {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if constexpr (kWords == 4) {
                const uint32_t u = w[i / 4][i % 4];
                v[i] = __builtin_bit_cast(float, u);
            } else {
                const uint32_t u = w[i / 8][i / 2 % 4];
                v[i] = __builtin_bit_cast(float, i & 1 ? u & 0xFFFF0000u : u << 16);
            }
        }
    }
};
// the first `have` of them, 0 behind (the end of a row)
template <typename X>
__device__ __forceinline__ void load_some(const X *p, int have, float (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
        v[i] = i < have ? load_value(p + i) : 0.f;
}

// The products of 32 rows of each operand over 64 values, e4m3 with a scale
// byte per row: byte SA of `sa` and SB of `sb`.
template <int SA, int SB>
__device__ __forceinline__ f32x16 multiply(const i32x8 &a, const i32x8 &b, const f32x16 &c, uint32_t sa, uint32_t sb) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, SA, (int)sa, SB, (int)sb);
}

}  // namespace f8
}  // namespace hpacml
