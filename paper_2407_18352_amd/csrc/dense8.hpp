// Dense layers in 8 bits: launchers, and the device arithmetic they share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dense8_rules.hpp"
#include "hpacml8.h"

namespace hpacml {

// Operands laid out for the products: slabs of 64 bytes of k (64 codes, 32
// bf16), 16 rows of a slab after one another (1 KB), the slabs of 16 rows after
// one another.  Of a row's four 16-byte chunks, chunk c is at c ^ chunk_turn(row).
constexpr int kSlabBytes = 64;
constexpr int64_t slabs_of(int64_t bytes) { return (bytes + kSlabBytes - 1) / kSlabBytes; }
constexpr int64_t blocked_bytes(int64_t rows, int64_t slabs) { return (rows + 15) / 16 * slabs * 1024; }
__host__ __device__ constexpr int chunk_turn(int row) { return (row >> 1) & 3; }
// of byte k of a row
__host__ __device__ constexpr int64_t blocked_offset(int64_t row, int64_t k, int64_t slabs) {
    return ((row >> 4) * slabs + (k >> 6)) * 1024 + (row & 15) * kSlabBytes + ((((int)(k >> 4) & 3) ^ chunk_turn((int)row)) * 16) + (k & 15);
}

// codes, blocked, and scales [rows] of x [rows][width]; columns from width to
// the end of the last slab are written as 0.
hipError_t launch_codes_by_row(const void *x, int32_t dtype, int64_t ldx, int64_t rows, int32_t width, int8_t *codes,
                               float *scales, hipStream_t stream);

// y = act(s_i t_j sum_k q_ik w_jk + b_j); x's codes and scales go to q and s,
// except where the product forms them itself.
struct Linear8Args {
    const void *x;
    int64_t ldx;
    int8_t *q;            // codes of the rows, blocked
    float *s;             // [rows]
    const int8_t *w;      // codes of the weights, blocked
    const float *t;       // [n_out], to a multiple of four
    const float *b;       // the same; zeros without a bias
    void *y;
    int64_t rows, ldy;
    int32_t slabs, n_in, n_out, relu;
};
// rows that q and s need room for: of these, or of fewer where these use neither
int64_t linear8_scratch_rows(int64_t rows, int32_t n_in, int32_t n_out);
hipError_t launch_linear8(const Linear8Args &a, int32_t x_dtype, int32_t y_dtype, hipStream_t stream);

hipError_t launch_checkpoint_save(const hpacml8_checkpoint &c, const void *z, int32_t z_dtype, int64_t ldz, void *a,
                                  int32_t a_dtype, int64_t lda, hipStream_t stream);
hipError_t launch_checkpoint_load(const hpacml8_checkpoint &c, void *a, int32_t a_dtype, int64_t lda,
                                  hipStream_t stream);

// The backward pass.  Everything it puts into scratch, as byte offsets.
struct Backward8Plan {
    int32_t planes;       // bf16 terms of an operand: 1 (bf16) or 3 (fp32)
    bool few;             // one launch that reads everything in place, without scratch
    bool direct;          // dy is read in place
    int32_t slabs;        // of dy and of W's transpose along the outputs
    int64_t pitch;        // of dy's planes (elements)
    DwForm dw;
    size_t off_dy, off_wt, off_dw, off_db, bytes;
};
Backward8Plan backward8_plan(const hpacml8_checkpoint &c, const void *dy, int32_t dtype, int64_t lddy, int32_t n_out,
                             bool want_dw, bool want_dx);
struct Backward8Args {
    hpacml8_checkpoint c;
    const void *dy;
    int32_t dtype;
    int64_t lddy;
    int32_t n_out;
    const void *W;
    int64_t ldw;
    float *dw;
    int64_t lddw;
    float *db;
    void *dx;
    int64_t lddx;
    int32_t accumulate;
    char *scratch;
};
hipError_t launch_backward8(const Backward8Args &a, const Backward8Plan &p, hipStream_t stream);
hipError_t launch_backward8_few(const Backward8Args &a, hipStream_t stream);

// ---- device arithmetic --------------------------------------------------------

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ float bf16_bits_value(uint32_t h) { return __builtin_bit_cast(float, h << 16); }
// nearest even; a NaN stays one
__device__ __forceinline__ uint16_t bf16_bits(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// two of them in one word, the first in the low half (one instruction)
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

__device__ __forceinline__ float load_value(const float *p) { return *p; }
__device__ __forceinline__ float load_value(const uint16_t *p) { return bf16_bits_value(*p); }
__device__ __forceinline__ void store_value(float *p, float v) { *p = v; }
__device__ __forceinline__ void store_value(uint16_t *p, float v) { *p = bf16_bits(v); }

// 16 bytes at any element's address
typedef u32x4 __attribute__((aligned(2))) u32x4_any;
typedef f32x4 __attribute__((aligned(4))) f32x4_any;

// four values at p, aligned to four
__device__ __forceinline__ void store_four(float *p, const float (&v)[4]) { *(f32x4 *)p = f32x4{v[0], v[1], v[2], v[3]}; }
__device__ __forceinline__ void store_four(uint16_t *p, const float (&v)[4]) {
    *(uint2 *)p = uint2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
}

// max(x, 0) that keeps a NaN
__device__ __forceinline__ float relu_keep_nan(float x) { return x < 0.f ? 0.f : x; }

// The exponent byte of a block whose largest magnitude has these bits, and
// the factor 2^-e that turns its values into codes.  amax in [2^(E-127),
// 2^(E-126)) for exponent field E, so e + 127 = E - 7 (codes to 255) or
// E - 6 (codes to 127); not below 1 (e = -126).
__device__ __forceinline__ uint32_t block_exp(uint32_t amax_bits, bool relu) {
    const uint32_t field = amax_bits >> 23, less = relu ? 7u : 6u;
    return field == 255u ? 255u : field > less ? field - less : 1u;
}
__device__ __forceinline__ float block_factor(uint32_t byte) {
    return byte == 255u ? 1.f : __builtin_bit_cast(float, (254u - byte) << 23);
}
// 2^e of an exponent byte (infinite for 255)
__device__ __forceinline__ float block_scale(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }
// the same for products with an operand's `terms` terms: with three, second and
// third ones that are 0 or of the other sign make NaN of an infinite value's
// products by chance, so there 255 is a NaN (in one instruction: the byte comes
// into the fraction as well, below 2^-15 of a value, which bf16 drops)
__device__ __forceinline__ float block_scale(uint32_t byte, int terms) {
    return __builtin_bit_cast(float, __umul24(byte, terms > 1 ? 0x800001u : 0x800000u));
}

template <bool RELU>
__device__ __forceinline__ uint32_t block_code(float a, float factor) {
    const float r = rintf(a * factor);
    if (RELU)
        return a > 0.f ? (uint32_t)fminf(fmaxf(r, 1.f), 255.f) : 0u;
    return (uint32_t)((int32_t)fminf(fmaxf(r, -127.f), 127.f) + 128);
}
// exact in bf16 (8 significant bits)
template <bool RELU>
__device__ __forceinline__ float block_value(uint32_t code, float scale) {
    return RELU ? (float)code * scale : ((float)code - 128.f) * scale;
}

// x and y, each as the exact sum of three bf16 terms, each the nearest to what
// is left (the first at most the largest finite one); a word holds a term of
// both, x's in the low half.  An infinity is 1 of its sign, 0 and itself: the
// products taken are those of terms whose ranks sum to at most 2, so it meets
// the other operand's first term alone, which has that operand's sign and is 0
// only for a 0, and a sum with it is what the operands' own would be (as a first
// term it would meet second and third ones that are 0 or of the other sign).  A
// NaN's second and third terms are NaN.
__device__ __forceinline__ void split3(float x, float y, uint32_t out[3]) {
    const bool inf_x = __builtin_isinf(x), inf_y = __builtin_isinf(y);
    const float most_x = inf_x ? 1.f : 0x1.FEp127f, most_y = inf_y ? 1.f : 0x1.FEp127f;
    out[0] = pack_bf16(__builtin_amdgcn_fmed3f(x, -most_x, most_x), __builtin_amdgcn_fmed3f(y, -most_y, most_y));
    const float rx = x - __builtin_bit_cast(float, out[0] << 16), ry = y - __builtin_bit_cast(float, out[0] & 0xFFFF0000u);
    out[1] = pack_bf16(inf_x ? 0.f : rx, inf_y ? 0.f : ry);
    out[2] = pack_bf16(rx - __builtin_bit_cast(float, out[1] << 16), ry - __builtin_bit_cast(float, out[1] & 0xFFFF0000u));
}

}  // namespace hpacml
