// The backward pass of a few rows: one launch that reads everything where it
// lies.  The general form's four launches (operands laid out, dx, dw, parts
// joined) each wait for memory once or twice with little on the way; here a
// block waits once.  A block computes 32 x 32 results of dx or of dw: its eight
// waves split the sum (over the outputs, or over the rows), load what their
// share needs straight into registers, form the bf16 terms there, multiply, and
// add their results through LDS, always in the same order.  256 rows, 64 -> 64
// in fp32: 4.7 us of the device where the general form takes 16.7.  What bounds
// it is one wait for memory and the loads' issue, a column's values being a
// load each.  A wave takes one step of a sum at a time: with two on the way at
// once, and their code, it took 7.2 us where one took 5.2 (256 <- 256: 11.4 and
// 5.6).
//
// The products are those of the general form: a kept value is exact in bf16, an
// fp32 value is three bf16 terms; dw takes three products, dx the six whose
// terms' ranks sum to at most 2.  db is the product with ones.
#include "dense8_rows.hpp"

namespace hpacml {

namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves, kTile = 32;
constexpr int kStep = 32;        // of a sum, per matrix instruction

struct FewArgs {
    hpacml8_checkpoint c;
    const void *dy, *W;
    void *dx;
    float *dw, *db;               // NULL: not wanted
    int64_t lddy, ldw, lddx, lddw;
    int32_t n_out, accumulate;
    uint32_t dx_blocks, in_tiles, dw_in_tiles;
};

// eight values as bf16, or as their three terms, the largest first
template <int TERMS>
__device__ __forceinline__ void terms_of(const float (&v)[kChunk], bf16x8 (&t)[TERMS]) {
    u32x4 w[TERMS];
    if constexpr (TERMS == 1) {
        w[0] = u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    } else {
#pragma unroll
        for (int e = 0; e < kChunk; e += 2) {
            uint32_t two[3];
            split3(v[e], v[e + 1], two);
#pragma unroll
            for (int q = 0; q < TERMS; ++q)
                w[q][e / 2] = two[q];
        }
    }
#pragma unroll
    for (int q = 0; q < TERMS; ++q)
        t[q] = __builtin_bit_cast(bf16x8, w[q]);
}

template <typename T, bool RELU>
__global__ void __launch_bounds__(kThreads) few_backward_kernel(FewArgs p) {
    constexpr int kTerms = sizeof(T) == 4 ? 3 : 1;
    __shared__ __align__(16) float part[kWaves][kTile * kTile];
    __shared__ float part_sums[kWaves][kTile];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, grp = lane >> 4;
    const T *dy = (const T *)p.dy;
    const uint8_t *codes = (const uint8_t *)p.c.codes, *exps = (const uint8_t *)p.c.exps;
    const int64_t rows = p.c.rows;
    const int n_in = (int)p.c.width;

    // acc[a][b]: channels 16 a + 4 grp + e of row (or output) 16 b + l16
    f32x4 acc[2][2] = {}, sum[2] = {};
    auto mul = [](bf16x8 a, bf16x8 b, f32x4 &c) { c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); };
    // into LDS, and the sum of the waves' results i of the tile, [row][channel]
    auto share = [&]() {
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int b = 0; b < 2; ++b)
                *(f32x4 *)&part[wave][(b * 16 + l16) * kTile + ((a * 4 + grp) ^ (l16 & 7)) * 4] = acc[a][b];
        __syncthreads();
    };
    auto total = [&](int row, int col) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            v += part[w][row * kTile + ((col >> 2) ^ (row & 7)) * 4 + (col & 3)];
        return v;
    };

    if (blockIdx.x < p.dx_blocks) {
        const int64_t p0 = (int64_t)(blockIdx.x / p.in_tiles) * kTile;
        const int k0 = (int)(blockIdx.x % p.in_tiles) * kTile, steps = (p.n_out + kStep - 1) / kStep;
        const T *w_at[2], *g_at[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            w_at[t] = (const T *)p.W + min(k0 + t * 16 + l16, n_in - 1);
            g_at[t] = dy + min(p0 + t * 16 + l16, rows - 1) * p.lddy;
        }
        for (int step = wave; step < steps; step += kWaves) {
            float w[2][kChunk], g[2][kChunk];
            const int o = step * kStep + grp * kChunk;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                load_chunk(g_at[t] + o, p.n_out - o, g[t]);
#pragma unroll
                for (int e = 0; e < kChunk; ++e)
                    w[t][e] = load_value(w_at[t] + min(o + e, p.n_out - 1) * p.ldw);
            }
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < kChunk; ++e)
                    w[t][e] = o + e < p.n_out ? w[t][e] : 0.f;
            bf16x8 a[2][kTerms], b[2][kTerms];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                terms_of(w[t], a[t]);
                terms_of(g[t], b[t]);
            }
            // the products whose ranks sum to at most 2, the smallest first
#pragma unroll
            for (int rank = kTerms - 1; rank >= 0; --rank)
#pragma unroll
                for (int q = 0; q <= rank; ++q)
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        mul(a[t & 1][q], b[t >> 1][rank - q], acc[t & 1][t >> 1]);
        }
        share();
#pragma unroll
        for (int i = tid; i < kTile * kTile; i += kThreads) {
            const int64_t r = p0 + i / kTile;
            const int k = k0 + i % kTile;
            if (r < rows && k < n_in) {
                const bool through = !RELU || codes[r * p.c.ld_codes + k] != 0;
                const float v = total(i / kTile, i % kTile);
                store_value((T *)p.dx + r * p.lddx + k, through ? v : 0.f);
            }
        }
        return;
    }

    const uint32_t id = blockIdx.x - p.dx_blocks;
    const int j0 = (int)(id / p.dw_in_tiles) * kTile, k0 = (int)(id % p.dw_in_tiles) * kTile;
    const int64_t steps = (rows + kStep - 1) / kStep;
    const bool sums = p.db && k0 == 0;
    for (int64_t step = wave; step < steps; step += kWaves) {
        float g[2][kChunk], scale[kChunk];
        uint32_t code[2][kChunk];
        const int64_t r0 = step * kStep + grp * kChunk;
#pragma unroll
        for (int e = 0; e < kChunk; ++e) {
            const int64_t r = min(r0 + e, rows - 1);
            // rows of codes are whole blocks of channels: all of a tile's exist
            const uint32_t exp = exps[r * p.c.ld_exps + k0 / 32];
            scale[e] = r0 + e < rows ? block_scale(exp, kTerms) : 0.f;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                code[t][e] = codes[r * p.c.ld_codes + k0 + t * 16 + l16];
                const float v = load_value(dy + r * p.lddy + min(j0 + t * 16 + l16, p.n_out - 1));
                g[t][e] = r0 + e < rows ? v : 0.f;
            }
        }
        bf16x8 a[2][1], b[2][kTerms];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float v[kChunk];
#pragma unroll
            for (int e = 0; e < kChunk; ++e)
                v[e] = block_value<RELU>(code[t][e], scale[e]);
            terms_of(v, a[t]);       // exact
            terms_of(g[t], b[t]);
        }
#pragma unroll
        for (int q = kTerms - 1; q >= 0; --q)
#pragma unroll
            for (int t = 0; t < 4; ++t)
                mul(a[t & 1][0], b[t >> 1][q], acc[t & 1][t >> 1]);
        if (sums) {
            const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u});
#pragma unroll
            for (int q = kTerms - 1; q >= 0; --q)
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    mul(ones, b[t][q], sum[t]);
        }
    }
    if (lane < 16) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
            part_sums[wave][t * 16 + lane] = sum[t][0];
    }
    share();
    if (p.dw)
#pragma unroll
        for (int i = tid; i < kTile * kTile; i += kThreads) {
            const int j = j0 + i / kTile, k = k0 + i % kTile;
            if (j < p.n_out && k < n_in) {
                float *to = p.dw + j * p.lddw + k;
                const float v = total(i / kTile, i % kTile);
                *to = p.accumulate ? *to + v : v;
            }
        }
    if (sums && tid < kTile && j0 + tid < p.n_out) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            v += part_sums[w][tid];
        float *to = p.db + j0 + tid;
        *to = p.accumulate ? *to + v : v;
    }
}

template <typename T>
void launch_as(const FewArgs &f, uint32_t blocks, hipStream_t st) {
    if (f.c.act == HPACML_ACT_RELU)
        few_backward_kernel<T, true><<<blocks, kThreads, 0, st>>>(f);
    else
        few_backward_kernel<T, false><<<blocks, kThreads, 0, st>>>(f);
}

uint32_t tiles(int64_t n) { return (uint32_t)((n + kTile - 1) / kTile); }

}  // namespace

hipError_t launch_backward8_few(const Backward8Args &a, hipStream_t st) {
    FewArgs f{a.c, a.dy, a.W, a.dx, a.dw, a.db, a.lddy, a.ldw, a.lddx, a.lddw, a.n_out, a.accumulate, 0, tiles(a.c.width),
              a.dw ? tiles(a.c.width) : 1};
    f.dx_blocks = a.dx ? f.in_tiles * tiles(a.c.rows) : 0;
    const uint32_t blocks = f.dx_blocks + (a.dw || a.db ? f.dw_in_tiles * tiles(a.n_out) : 0);
    if (blocks > 0)
        a.dtype == HPACML_F32 ? launch_as<float>(f, blocks, st) : launch_as<uint16_t>(f, blocks, st);
    return hipGetLastError();
}

}  // namespace hpacml
