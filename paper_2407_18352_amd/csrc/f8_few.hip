// y = act(x W^T + b) of few rows, in one launch.
//
// A few rows are asked for one answer at a time: what counts is reading the
// weights once, from as many CUs as there are, and the latency of what comes
// before and after.  A block takes 16 outputs and all the rows; its waves
// take blocks of the width in turn, straight from memory to registers, and join
// their sums through LDS (4096 -> 4096, one row: 11.6, 9.1 and 8.4 us with 4, 8
// and 16 waves, 7.7 with x's loads ahead of its codes; reading the weights alone
// takes 3.5).  Codes of x are formed by every block anew (or read,
// where the product is given them).  The products run on the bf16 matrix
// instruction, to which codes times their scale are exact: there is time for it.
#include <type_traits>

#include "f8.hpp"

namespace hpacml {
namespace f8 {

namespace {

// Sixteen waves where their registers hold what one of them loads at a time.
template <int NB>
constexpr int kWavesOf = NB == 1 ? 16 : 8;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

struct FewArgs {
    const void *x;           // rows, or NULL: p
    int64_t ldx;
    Matrix p, q;
    int64_t rows;
    const float *b;
    void *y;
    int64_t ldy;
    int32_t relu, accumulate;
};

// 32 codes of a lane, as four operands of the matrix instruction
struct Operand {
    bf16x8 v[4];
};
__device__ __forceinline__ Operand to_bf16(const uint32_t (&codes)[8], uint32_t byte) {
    const float s = __builtin_bit_cast(float, byte << 23);
    Operand o;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[i], s, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[i], s, true);
        o.v[i / 2][i % 2 * 4] = lo[0];
        o.v[i / 2][i % 2 * 4 + 1] = lo[1];
        o.v[i / 2][i % 2 * 4 + 2] = hi[0];
        o.v[i / 2][i % 2 * 4 + 3] = hi[1];
    }
    return o;
}

// Lane l holds row l % 16 and values 32 (l / 16).. of a block: codes
struct Codes {
    uint32_t c[8], byte;
};
__device__ __forceinline__ Codes read_codes(const Matrix &m, int64_t row, int group, int64_t kb, int64_t blocks) {
    const int64_t r = min(row, m.rows - 1);
    const char *at = m.codes + code_offset(r, kb * kBlock + group * 32, blocks);
    Codes o;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const u32x4 w = *(const u32x4 *)(at + h * 1024);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            o.c[h * 4 + e] = w[e];
    }
    o.byte = (uint8_t)m.scales[scale_offset(r, kb, blocks)];
    return o;
}

// Of 32 values of a row (the last row where there is none: what comes of it is
// not stored).
template <typename X>
struct Row {
    Sixteen<X> half[2];
};
__device__ __forceinline__ Codes form_codes(const float (&v)[2][16]) {
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i)
        most = max(most, magnitude(v[i / 16][i % 16]));
    most = max(most, (uint32_t)__shfl_xor((int)most, 16));
    most = max(most, (uint32_t)__shfl_xor((int)most, 32));
    Codes o;
    o.byte = scale_byte(most);
    const float f = scale_factor(o.byte);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float *u = &v[i / 4][i % 4 * 4];
        o.c[i] = o.byte == 255u ? kNanCodes : codes4(u[0], u[1], u[2], u[3], f);
    }
    return o;
}

// X: the type of x, or void: codes are given.  NB: sixteens of rows.
template <typename X, typename Y, int NB>
__global__ __launch_bounds__(64 * kWavesOf<NB>) void few_kernel(FewArgs a) {
    constexpr int kWaves = kWavesOf<NB>;
    __shared__ f32x4 of[kWaves][NB][64];
    constexpr int kAtOnce = NB < 4 ? 2 : 1;       // blocks of the width whose loads go out together
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, group = lane >> 4;
    const int64_t blocks = blocks_of(a.q.width), out0 = (int64_t)blockIdx.x * 16;
    f32x4 acc[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
        acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int64_t first = wave; first < blocks; first += kWaves * kAtOnce) {
        Codes w[kAtOnce], x[kAtOnce][NB];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int64_t kb = min(first + u * kWaves, blocks - 1);
            w[u] = read_codes(a.q, out0 + r, group, kb, blocks);
            if (first + u * kWaves >= blocks)       // the last block again, times 0
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    w[u].c[i] = 0;
        }
        if constexpr (std::is_void<X>::value) {
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
                for (int b = 0; b < NB; ++b)
                    x[u][b] = read_codes(a.p, b * 16 + r, group, min(first + u * kWaves, blocks - 1), blocks);
        } else {
            auto at = [&](int u, int b) {
                return (const X *)a.x + min((int64_t)(b * 16 + r), a.rows - 1) * a.ldx + min(first + u * kWaves, blocks - 1) * kBlock + group * 32;
            };
            if ((min(first + (kAtOnce - 1) * kWaves, blocks - 1) + 1) * kBlock <= a.q.width) {
                Row<X> row[kAtOnce][NB];         // all loads before the first value
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
                    for (int b = 0; b < NB; ++b)
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            row[u][b].half[h].load(at(u, b) + h * 16);
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        float v[2][16];
                        row[u][b].half[0].values(v[0]);
                        row[u][b].half[1].values(v[1]);
                        x[u][b] = form_codes(v);
                    }
            } else {
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        float v[2][16];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int64_t left = a.q.width - min(first + u * kWaves, blocks - 1) * kBlock - group * 32 - h * 16;
                            load_some(at(u, b) + h * 16, left > 16 ? 16 : left < 0 ? 0 : (int)left, v[h]);
                        }
                        x[u][b] = form_codes(v);
                    }
            }
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const Operand wo = to_bf16(w[u].c, w[u].byte);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const Operand xo = to_bf16(x[u][b].c, x[u][b].byte);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wo.v[i], xo.v[i], acc[b], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
        of[wave][b][lane] = acc[b];
    __syncthreads();
    for (int b = wave; b < NB; b += kWaves) {
        f32x4 t = of[0][b][lane];
#pragma unroll
        for (int w = 1; w < kWaves; ++w)
            t += of[w][b][lane];
        const int64_t row = b * 16 + r, out = out0 + group * 4;
        if (row >= a.rows)
            continue;
        Y *to = (Y *)a.y + row * a.ldy + out;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (out + e < a.q.rows) {
                float v = t[e] + (a.b ? a.b[out + e] : 0.f);
                if (a.relu)
                    v = relu_keep_nan(v);
                if constexpr (sizeof(Y) == 4)
                    v += a.accumulate ? to[e] : 0.f;
                store_value(to + e, v);
            }
    }
}

template <typename X, typename Y>
void launch(const FewArgs &a, hipStream_t stream) {
    const uint32_t grid = (uint32_t)((a.q.rows + 15) / 16);
    if (a.rows <= 16)
        few_kernel<X, Y, 1><<<grid, 64 * kWavesOf<1>, 0, stream>>>(a);
    else if (a.rows <= 32)
        few_kernel<X, Y, 2><<<grid, 64 * kWavesOf<2>, 0, stream>>>(a);
    else
        few_kernel<X, Y, 4><<<grid, 64 * kWavesOf<4>, 0, stream>>>(a);
}
template <typename X>
hipError_t launch_type(const FewArgs &a, int32_t y_dtype, hipStream_t stream) {
    if (y_dtype == HPACML_F32)
        launch<X, float>(a, stream);
    else
        launch<X, uint16_t>(a, stream);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_product_few(const ProductArgs &a, int32_t y_dtype, hipStream_t stream) {
    return launch_type<void>({nullptr, 0, a.p, a.q, a.p.rows, a.b, a.y, a.ldy, a.relu, a.accumulate}, y_dtype, stream);
}

hipError_t launch_linear_few(const ProductArgs &a, const void *x, int32_t x_dtype, int64_t ldx, int32_t y_dtype, hipStream_t stream) {
    const FewArgs f = {x, ldx, a.p, a.q, a.p.rows, a.b, a.y, a.ldy, a.relu, a.accumulate};
    return x_dtype == HPACML_F32 ? launch_type<float>(f, y_dtype, stream) : launch_type<uint16_t>(f, y_dtype, stream);
}

}  // namespace f8
}  // namespace hpacml
