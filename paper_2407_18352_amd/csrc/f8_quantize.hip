// Codes and scales of a matrix by row, by column, or both in one reading.
//
// A block of 256 threads takes 128 x 128 values: a thread four rows by 16
// columns, in registers.  The largest magnitude of a row's 128 columns joins
// eight lanes, that of a column's 128 rows the threads of a wave and, through
// LDS, the four waves.  The codes by row (16 of a thread are one store) and by
// column (four rows of a column are one word) are laid out in LDS as they lie in
// memory, 16 KB each, and copied out in whole pieces.  16-byte slots are turned
// by what the lanes of one LDS write differ in (turn_row, turn_column), so that
// they fall on different banks.  Reading and writing is what it has to do:
// 131,072 x 4096 in bf16 by row takes 0.30 ms (1.6 GB at 5.4 TB/s), 131,072 x 2048
// by row and column behind a ReLU 0.33 ms (4.9 TB/s), 65,536 x 512 by row and
// column 36 us (3.7 TB/s; limits on the registers, for more waves, change nothing
// there or cost spills); one block alone takes 6 us.
#include <type_traits>

#include "f8.hpp"

namespace hpacml {
namespace f8 {

namespace {

// slot of 16 bytes in a 16 KB image: unit * 128 + half * 64 + group * 32 + row
__device__ __forceinline__ int turn_row(int slot) { return slot ^ (((slot >> 4) & 1) | (((slot >> 6) & 1) << 1)); }
__device__ __forceinline__ int turn_column(int slot) {
    return slot ^ (((slot >> 4) & 1) | (((slot >> 8) & 3) << 1) | (((slot >> 6) & 1) << 3));
}

// another lane's value, by an operand permutation of the vector unit
template <int CONTROL>
__device__ __forceinline__ uint32_t permuted(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CONTROL, 15, 15, true);
}
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E, kMirror8 = 0x141, kTurn8 = 0x128;    // neighbours; pairs; eight mirrored; sixteen turned by eight

template <typename X, bool ROW, bool COLUMN, bool MASK, bool SUMS>
__global__ __launch_bounds__(256) void quantize_kernel(QuantizeArgs a) {
    __shared__ u32x4 image[ROW && COLUMN ? 2048 : 1024];
    __shared__ uint32_t most_of[4][128];
    __shared__ float sum_of[SUMS ? 4 : 1][128];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int rg = lane & 7, tc = lane >> 3;                 // rows 32 wave + 4 rg + j, columns 16 tc + i
    const int64_t row_tile = blockIdx.x / blocks_of(a.width), col_tile = blockIdx.x % blocks_of(a.width);
    const int64_t row0 = row_tile * 128 + wave * 32 + rg * 4, col0 = col_tile * 128 + tc * 16;
    const int64_t left = a.width - col0;
    const int have = left > 16 ? 16 : left < 0 ? 0 : (int)left;

    // all loads go out before the first value is looked at (with a row's values
    // taken apart behind its loads, 65,536 x 512 in bf16 took 42 us by row and column)
    float v[4][16];
    if (have == 16) {
        Sixteen<X> x[4], y[MASK ? 4 : 1];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t row = min(row0 + j, a.rows - 1);
            x[j].load((const X *)a.x + row * a.ldx + col0);
            if (MASK)
                y[j].load((const X *)a.y + row * a.ldy + col0);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[j].values(v[j]);
            if (MASK) {
                float m[16];
                y[j].values(m);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    v[j][i] = m[i] <= 0.f ? 0.f : v[j][i];
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t row = min(row0 + j, a.rows - 1);
            load_some((const X *)a.x + row * a.ldx + col0, have, v[j]);
            if (MASK) {
                float m[16];
                load_some((const X *)a.y + row * a.ldy + col0, have, m);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    v[j][i] = m[i] <= 0.f ? 0.f : v[j][i];
            }
        }
    }
    if (row0 + 3 >= a.rows)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                v[j][i] = row0 + j < a.rows ? v[j][i] : 0.f;
    uint32_t row_most[4], col_most[16];
    if (ROW) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                m = max(m, magnitude(v[j][i]));
            m = max(m, permuted<kTurn8>(m));
            m = max(m, (uint32_t)__shfl_xor((int)m, 16));
            m = max(m, (uint32_t)__shfl_xor((int)m, 32));
            row_most[j] = m;
        }
    }
    if (COLUMN || SUMS) {
        float col_sum[SUMS ? 16 : 1];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (COLUMN) {
                uint32_t m = max(max(magnitude(v[0][i]), magnitude(v[1][i])), max(magnitude(v[2][i]), magnitude(v[3][i])));
                m = max(m, permuted<kSwap1>(m));
                m = max(m, permuted<kSwap2>(m));
                col_most[i] = max(m, permuted<kMirror8>(m));
            }
            if (SUMS) {
                auto other = [](float t, auto control) {
                    return __builtin_bit_cast(float, permuted<decltype(control)::value>(__builtin_bit_cast(uint32_t, t)));
                };
                float t = (v[0][i] + v[1][i]) + (v[2][i] + v[3][i]);
                t += other(t, std::integral_constant<int, kSwap1>());
                t += other(t, std::integral_constant<int, kSwap2>());
                col_sum[i] = t + other(t, std::integral_constant<int, kMirror8>());
            }
        }
        if (rg == 0)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if (COLUMN)
                    most_of[wave][tc * 16 + i] = col_most[i];
                if (SUMS)
                    sum_of[wave][tc * 16 + i] = col_sum[i];
            }
        __syncthreads();
        if (COLUMN) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int c = tc * 16 + i;
                col_most[i] = max(max(most_of[0][c], most_of[1][c]), max(most_of[2][c], most_of[3][c]));
            }
        }
        if (SUMS && threadIdx.x < 128 && col_tile * 128 + threadIdx.x < a.width)
            a.sums[row_tile * a.width + col_tile * 128 + threadIdx.x] =
                (sum_of[0][threadIdx.x] + sum_of[1][threadIdx.x]) + (sum_of[2][threadIdx.x] + sum_of[3][threadIdx.x]);
    }
    if (a.square) {
        // the largest of all: of the columns where those are known, of the rows otherwise
        uint32_t m = 0;
        if (COLUMN) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                m = max(m, col_most[i]);
#pragma unroll
            for (int s = 8; s < 64; s *= 2)
                m = max(m, (uint32_t)__shfl_xor((int)m, s));
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                m = max(m, row_most[j]);
#pragma unroll
            for (int s = 1; s < 8; s *= 2)
                m = max(m, (uint32_t)__shfl_xor((int)m, s));
            if (lane == 0)
                most_of[wave][0] = m;
            __syncthreads();
            m = max(max(most_of[0][0], most_of[1][0]), max(most_of[2][0], most_of[3][0]));
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            row_most[j] = m;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            col_most[i] = m;
    }
    if (ROW) {
        const int64_t blocks = blocks_of(a.width);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t byte = scale_byte(row_most[j]);
            const float f = scale_factor(byte);
            u32x4 c;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                c[e] = byte == 255u ? kNanCodes : codes4(v[j][4 * e], v[j][4 * e + 1], v[j][4 * e + 2], v[j][4 * e + 3], f);
            // unit (32 rows: wave) * 2 + tc / 4, half tc % 2, group (tc / 2) % 2, row 4 rg + j
            image[turn_row((wave * 2 + (tc >> 2)) * 128 + (tc & 1) * 64 + ((tc >> 1) & 1) * 32 + rg * 4 + j)] = c;
            if (tc == 0)
                a.by_row.scales[scale_offset(row0 + j, col_tile, blocks)] = (char)byte;
        }
    }
    if (COLUMN) {
        const int64_t blocks = blocks_of(a.rows);
        char *to = (char *)(image + (ROW ? 1024 : 0));
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t byte = scale_byte(col_most[i]);
            const uint32_t w = byte == 255u ? kNanCodes : codes4(v[0][i], v[1][i], v[2][i], v[3][i], scale_factor(byte));
            const int c = tc * 16 + i, r = wave * 32 + rg * 4;       // row c of the transpose, values r..r + 3 of its 128
            const int slot = ((c >> 5) * 2 + (r >> 6)) * 128 + ((r >> 4) & 1) * 64 + ((r >> 5) & 1) * 32 + (c & 31);
            *(uint32_t *)(to + turn_column(slot) * 16 + (r & 15)) = w;
            if (rg == 0 && wave == 0)
                a.by_column.scales[scale_offset(col_tile * 128 + c, row_tile, blocks)] = (char)byte;
        }
    }
    __syncthreads();
    // 1024 slots of each, 128 a unit; units of rows that do not exist are not written
    if (ROW) {
        const int64_t blocks = blocks_of(a.width), units = row_units(a.rows);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int slot = i * 256 + threadIdx.x;
            const int64_t unit = row_tile * 4 + (slot >> 8);
            if (unit < units)
                *(u32x4 *)(a.by_row.codes + (unit * blocks + col_tile) * 2 * kUnit + (slot & 255) * 16) = image[turn_row(slot)];
        }
    }
    if (COLUMN) {
        const int64_t blocks = blocks_of(a.rows), units = row_units(a.width);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int slot = i * 256 + threadIdx.x;
            const int64_t unit = col_tile * 4 + (slot >> 8);
            if (unit < units)
                *(u32x4 *)(a.by_column.codes + (unit * blocks + row_tile) * 2 * kUnit + (slot & 255) * 16) =
                    image[(ROW ? 1024 : 0) + turn_column(slot)];
        }
    }
}

// A block takes 32 rows by 128 values, a thread 16 codes of a row.
template <typename X>
__device__ __forceinline__ void load_block(const Matrix &m, X *x, int64_t ldx, int64_t unit, int64_t part, int64_t blocks) {
    const int64_t row = unit * 32 + (threadIdx.x >> 3), k = (part * 8 + (threadIdx.x & 7)) * 16;
    if (row >= m.rows || k >= m.width)
        return;
    const u32x4 c = *(const u32x4 *)(m.codes + code_offset(row, k, blocks));
    const uint32_t byte = (uint8_t)m.scales[scale_offset(row, k / kBlock, blocks)];
    const float s = byte == 255u ? __builtin_nanf("") : byte == 0u ? 0x1p-127f : __builtin_bit_cast(float, byte << 23);
    float v[16];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[4 * e] = __builtin_amdgcn_cvt_f32_fp8(c[e], 0) * s;
        v[4 * e + 1] = __builtin_amdgcn_cvt_f32_fp8(c[e], 1) * s;
        v[4 * e + 2] = __builtin_amdgcn_cvt_f32_fp8(c[e], 2) * s;
        v[4 * e + 3] = __builtin_amdgcn_cvt_f32_fp8(c[e], 3) * s;
    }
    X *to = x + row * ldx + k;
    if (k + 16 <= m.width) {
#pragma unroll
        for (int e = 0; e < (int)sizeof(X); ++e) {
            u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(X) == 4)
                    w[i] = __builtin_bit_cast(uint32_t, v[4 * e + i]);
                else
                    w[i] = pack_bf16(v[8 * e + 2 * i], v[8 * e + 2 * i + 1]);
            }
            *(u32x4_any *)(to + e * (16 / sizeof(X))) = w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (k + i < m.width)
                store_value(to + i, v[i]);
    }
}
template <typename X>
__global__ __launch_bounds__(256) void load_kernel(Matrix m, X *x, int64_t ldx) {
    const int64_t blocks = blocks_of(m.width), all = row_units(m.rows) * blocks;
    for (int64_t at = blockIdx.x; at < all; at += gridDim.x)
        load_block(m, x, ldx, at / blocks, at % blocks, blocks);
}

template <typename X, bool ROW, bool COLUMN>
void launch_form(const QuantizeArgs &a, uint32_t blocks, hipStream_t stream) {
    if (a.sums) {
        if (a.y)
            quantize_kernel<X, ROW, COLUMN, true, true><<<blocks, 256, 0, stream>>>(a);
        else
            quantize_kernel<X, ROW, COLUMN, false, true><<<blocks, 256, 0, stream>>>(a);
    } else if constexpr (ROW || COLUMN) {
        if (a.y)
            quantize_kernel<X, ROW, COLUMN, true, false><<<blocks, 256, 0, stream>>>(a);
        else
            quantize_kernel<X, ROW, COLUMN, false, false><<<blocks, 256, 0, stream>>>(a);
    }
}

template <typename X>
void launch_type(const QuantizeArgs &a, uint32_t blocks, hipStream_t stream) {
    if (a.by_row.codes && a.by_column.codes)
        launch_form<X, true, true>(a, blocks, stream);
    else if (a.by_row.codes)
        launch_form<X, true, false>(a, blocks, stream);
    else if (a.by_column.codes)
        launch_form<X, false, true>(a, blocks, stream);
    else
        launch_form<X, false, false>(a, blocks, stream);
}

}  // namespace

hipError_t launch_quantize(const QuantizeArgs &a, int32_t dtype, hipStream_t stream) {
    const int64_t blocks = blocks_of(a.rows) * blocks_of(a.width);
    if (blocks == 0)
        return hipSuccess;
    if (too_many_blocks(a.rows, a.width))
        return hipErrorInvalidValue;
    if (dtype == HPACML_F32)
        launch_type<float>(a, (uint32_t)blocks, stream);
    else
        launch_type<uint16_t>(a, (uint32_t)blocks, stream);
    return hipGetLastError();
}

hipError_t launch_load(const Matrix &m, void *x, int32_t dtype, int64_t ldx, hipStream_t stream) {
    const int64_t blocks = row_units(m.rows) * blocks_of(m.width);
    if (blocks == 0)
        return hipSuccess;
    const uint32_t grid = (uint32_t)(blocks < 1 << 20 ? blocks : 1 << 20);
    if (dtype == HPACML_F32)
        load_kernel<<<grid, 256, 0, stream>>>(m, (float *)x, ldx);
    else
        load_kernel<<<grid, 256, 0, stream>>>(m, (uint16_t *)x, ldx);
    return hipGetLastError();
}

}  // namespace f8
}  // namespace hpacml
