// The backward pass of a linear layer whose input was kept in 8 bits:
//   dw = dy^T a, db = the sum of dy's rows, dx = (dy W) where the codes are not 0.
// A kept value (8 significant bits times a power of two) is exact in bf16, so
// dw's products are exact on v_mfma_f32_16x16x32_bf16 and summed in fp32.  An
// fp32 operand is the exact sum of three bf16 terms: three products for dw,
// for dx those six of nine whose terms' ranks sum to at most 2.
#include "dense8.hpp"

namespace hpacml {

namespace {

constexpr int kThreads = 256;
constexpr int kTile = 64;
constexpr int64_t kMaxBlocks = 1 << 20;   // the kernels loop beyond them
constexpr int kPitch = kSlabBytes + 16;   // of an LDS row, bytes

// planes [planes][rows][pitch] of v [rows][width], zero beyond the width
template <typename T>
__global__ void __launch_bounds__(kThreads) planes_kernel(const T *__restrict__ v, int64_t ld, int64_t rows,
                                                          int32_t width, uint16_t *__restrict__ out, int64_t pitch) {
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < rows * pitch; i += (int64_t)gridDim.x * kThreads) {
        const int64_t r = i / pitch, k = i - r * pitch;
        const T *at = v + r * ld + k;
        if constexpr (sizeof(T) == 4) {
            uint16_t t[3] = {0, 0, 0};
            if (k < width)
                split3(*at, t);
            for (int q = 0; q < 3; ++q)
                out[q * rows * pitch + i] = t[q];
        } else {
            out[i] = k < width ? *at : (uint16_t)0;
        }
    }
}

// planes [planes][n_in][pitch] of W's transpose, zero beyond n_out
template <typename T>
__global__ void __launch_bounds__(kThreads) transpose_kernel(const T *__restrict__ W, int64_t ldw, int32_t n_out,
                                                             int32_t n_in, uint16_t *__restrict__ out, int64_t pitch) {
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n_in * pitch; i += (int64_t)gridDim.x * kThreads) {
        const int64_t k = i / pitch, j = i - k * pitch;
        if constexpr (sizeof(T) == 4) {
            uint16_t t[3] = {0, 0, 0};
            if (j < n_out)
                split3(W[j * ldw + k], t);
            for (int q = 0; q < 3; ++q)
                out[q * n_in * pitch + i] = t[q];
        } else {
            out[i] = j < n_out ? W[j * ldw + k] : (uint16_t)0;
        }
    }
}

struct DxArgs {
    const uint16_t *g, *wt;     // planes of dy [rows][pitch] and of W's transpose [n_in][pitch]
    const uint8_t *codes;       // NULL: everything is let through
    void *dx;
    int64_t rows, pitch, ld_codes, lddx;
    int32_t n_in, planes;
};

template <typename X>
__global__ void __launch_bounds__(kThreads) dx_kernel(DxArgs p, int64_t tiles, int32_t col_tiles) {
    __shared__ __align__(16) char gs[kTile][kPitch], ws[kTile][kPitch];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wr = (wave & 1) * 32, wc = (wave >> 1) * 32;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t r0 = tile / col_tiles * kTile;
        const int c0 = (int)(tile % col_tiles) * kTile;
        f32x4 acc[2][2] = {};
        for (int rank = p.planes - 1; rank >= 0; --rank)         // the smallest products first
            for (int q = 0; q <= rank; ++q) {
                const uint16_t *g = p.g + q * p.rows * p.pitch, *w = p.wt + (rank - q) * p.n_in * p.pitch;
                for (int64_t k = 0; k < p.pitch; k += 64) {
                    for (int i = tid; i < kTile * 8; i += kThreads) {
                        const int row = i >> 3, chunk = i & 7;
                        const int64_t r = min(r0 + row, p.rows - 1), n = min(c0 + row, p.n_in - 1);
                        *(u32x4 *)&gs[row][chunk * 16] = *(const u32x4 *)(g + r * p.pitch + k + chunk * 8);
                        *(u32x4 *)&ws[row][chunk * 16] = *(const u32x4 *)(w + n * p.pitch + k + chunk * 8);
                    }
                    __syncthreads();
                    for (int s = 0; s < 2; ++s) {
                        bf16x8 a[2], b[2];
                        for (int t = 0; t < 2; ++t) {
                            a[t] = *(const bf16x8 *)&gs[wr + t * 16 + (lane & 15)][s * 64 + (lane >> 4) * 16];
                            b[t] = *(const bf16x8 *)&ws[wc + t * 16 + (lane & 15)][s * 64 + (lane >> 4) * 16];
                        }
                        for (int t = 0; t < 2; ++t)
                            for (int u = 0; u < 2; ++u)
                                acc[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[t], b[u], acc[t][u], 0, 0, 0);
                    }
                    __syncthreads();
                }
            }
        for (int t = 0; t < 2; ++t)
            for (int u = 0; u < 2; ++u)
                for (int e = 0; e < 4; ++e) {
                    const int64_t r = r0 + wr + t * 16 + (lane >> 4) * 4 + e;
                    const int n = c0 + wc + u * 16 + (lane & 15);
                    if (r < p.rows && n < p.n_in) {
                        const bool through = !p.codes || p.codes[r * p.ld_codes + n] != 0;
                        store_value((X *)p.dx + r * p.lddx + n, through ? acc[t][u][e] : 0.f);
                    }
                }
    }
}

struct DwArgs {
    const uint16_t *g;          // planes of dy [rows][pitch]
    hpacml8_checkpoint c;
    float *dw, *db;             // dw [splits][n_out][n_in], db [splits][n_out]; NULL: not wanted
    int64_t pitch, rows_per_split;
    int32_t n_out, planes;
};

// One block: 64 outputs x 64 channels over one part of the rows.
template <bool RELU>
__global__ void __launch_bounds__(kThreads) dw_kernel(DwArgs p) {
    __shared__ __align__(16) uint16_t gs[kTile][kPitch / 2], xs[kTile][kPitch / 2];   // [output or channel][row]
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int k0 = blockIdx.x * kTile, j0 = blockIdx.y * kTile, wj = (wave & 1) * 32, wk = (wave >> 1) * 32;
    const int64_t from = blockIdx.z * p.rows_per_split, to = min(from + p.rows_per_split, p.c.rows);
    f32x4 acc[2][2] = {}, sum[2] = {};
    const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u});
    for (int q = p.planes - 1; q >= 0; --q)
        for (int64_t r0 = from; r0 < to; r0 += 64) {
            for (int i = tid; i < 64 * kTile; i += kThreads) {
                const int row = i >> 6, col = i & 63;
                const int64_t r = r0 + row;
                uint16_t g = 0, x = 0;
                if (r < to && j0 + col < p.pitch)
                    g = p.g[(q * p.c.rows + r) * p.pitch + j0 + col];
                if (r < to && k0 + col < p.c.width) {
                    const float s = block_scale(((const uint8_t *)p.c.exps)[r * p.c.ld_exps + (k0 + col) / 32]);
                    x = bf16_bits(block_value<RELU>(((const uint8_t *)p.c.codes)[r * p.c.ld_codes + k0 + col], s));
                }
                gs[col][row] = g;
                xs[col][row] = x;
            }
            __syncthreads();
            for (int s = 0; s < 2; ++s) {
                bf16x8 a[2], b[2];
                for (int t = 0; t < 2; ++t) {
                    a[t] = *(const bf16x8 *)&gs[wj + t * 16 + (lane & 15)][s * 32 + (lane >> 4) * 8];
                    b[t] = *(const bf16x8 *)&xs[wk + t * 16 + (lane & 15)][s * 32 + (lane >> 4) * 8];
                }
                for (int t = 0; t < 2; ++t) {
                    for (int u = 0; u < 2; ++u)
                        acc[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[t], b[u], acc[t][u], 0, 0, 0);
                    sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[t], ones, sum[t], 0, 0, 0);
                }
            }
            __syncthreads();
        }
    for (int t = 0; t < 2; ++t)
        for (int e = 0; e < 4; ++e) {
            const int j = j0 + wj + t * 16 + (lane >> 4) * 4 + e;
            if (j >= p.n_out)
                continue;
            if (p.db && blockIdx.x == 0 && wk == 0 && (lane & 15) == 0)
                p.db[(int64_t)blockIdx.z * p.n_out + j] = sum[t][e];
            for (int u = 0; u < 2; ++u) {
                const int k = k0 + wk + u * 16 + (lane & 15);
                if (p.dw && k < p.c.width)
                    p.dw[((int64_t)blockIdx.z * p.n_out + j) * p.c.width + k] = acc[t][u][e];
            }
        }
}

// out [rows][ld] (+)= the sum over the parts of parts [splits][rows][width]
__global__ void __launch_bounds__(kThreads) join_kernel(const float *__restrict__ parts, int32_t splits, int64_t rows,
                                                        int64_t width, float *__restrict__ out, int64_t ld,
                                                        int32_t accumulate) {
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < rows * width; i += (int64_t)gridDim.x * kThreads) {
        float v = 0.f;
        for (int s = 0; s < splits; ++s)
            v += parts[s * rows * width + i];
        float *o = out + i / width * ld + i % width;
        *o = accumulate ? *o + v : v;
    }
}

dim3 blocks_for(int64_t items) {
    const int64_t n = (items + kThreads - 1) / kThreads;
    return dim3((uint32_t)(n < 1 ? 1 : n < 65536 ? n : 65536));
}
size_t whole(size_t b) { return (b + 255) / 256 * 256; }

}  // namespace

Backward8Plan backward8_plan(const hpacml8_checkpoint &c, const void *, int32_t dtype, int64_t, int32_t n_out,
                             bool want_dw, bool want_dx) {
    Backward8Plan p{};
    p.planes = dtype == HPACML_F32 ? 3 : 1;
    p.direct = false;
    p.pitch = slab_pitch16(n_out);
    const int64_t tiles = (int64_t)((c.width + kTile - 1) / kTile) * ((n_out + kTile - 1) / kTile);
    int64_t splits = want_dw ? (1024 + tiles - 1) / tiles : 0;
    const int64_t most = c.rows / 512 < 1 ? 1 : c.rows / 512;
    splits = splits < most ? splits : most;
    p.rows_per_split = splits ? ((c.rows + splits - 1) / splits + 63) / 64 * 64 : 0;
    if (splits)
        splits = p.rows_per_split ? (c.rows + p.rows_per_split - 1) / p.rows_per_split : 1;
    p.splits = (int32_t)(splits < 1 ? 1 : splits);
    size_t at = 0;
    p.off_dy = at;
    at += whole((size_t)p.planes * c.rows * p.pitch * 2);
    p.off_wt = at;
    if (want_dx)
        at += whole((size_t)p.planes * c.width * p.pitch * 2);
    p.off_dw = at;
    if (want_dw)
        at += whole((size_t)p.splits * n_out * c.width * 4);
    p.off_db = at;
    if (want_dw)
        at += whole((size_t)p.splits * n_out * 4);
    p.bytes = at;
    return p;
}

hipError_t launch_backward8(const Backward8Args &a, const Backward8Plan &p, hipStream_t st) {
    const int64_t rows = a.c.rows;
    const bool f32 = a.dtype == HPACML_F32;
    uint16_t *g = (uint16_t *)(a.scratch + p.off_dy), *wt = (uint16_t *)(a.scratch + p.off_wt);
    if (rows > 0) {
        if (f32)
            planes_kernel<float><<<blocks_for(rows * p.pitch), kThreads, 0, st>>>((const float *)a.dy, a.lddy, rows, a.n_out, g, p.pitch);
        else
            planes_kernel<uint16_t><<<blocks_for(rows * p.pitch), kThreads, 0, st>>>((const uint16_t *)a.dy, a.lddy, rows, a.n_out, g, p.pitch);
    }
    if (a.dx && rows > 0) {
        if (f32)
            transpose_kernel<float><<<blocks_for(a.c.width * p.pitch), kThreads, 0, st>>>((const float *)a.W, a.ldw, a.n_out, a.c.width, wt, p.pitch);
        else
            transpose_kernel<uint16_t><<<blocks_for(a.c.width * p.pitch), kThreads, 0, st>>>((const uint16_t *)a.W, a.ldw, a.n_out, a.c.width, wt, p.pitch);
        const uint8_t *codes = a.c.act == HPACML_ACT_RELU ? (const uint8_t *)a.c.codes : nullptr;
        const int32_t col_tiles = (a.c.width + kTile - 1) / kTile;
        const int64_t tiles = (rows + kTile - 1) / kTile * col_tiles;
        const dim3 grid((uint32_t)(tiles < kMaxBlocks ? tiles : kMaxBlocks));
        DxArgs d{g, wt, codes, a.dx, rows, p.pitch, a.c.ld_codes, a.lddx, a.c.width, p.planes};
        if (f32)
            dx_kernel<float><<<grid, kThreads, 0, st>>>(d, tiles, col_tiles);
        else
            dx_kernel<uint16_t><<<grid, kThreads, 0, st>>>(d, tiles, col_tiles);
    }
    if (a.dw || a.db) {
        float *dw = a.dw ? (float *)(a.scratch + p.off_dw) : nullptr, *db = a.db ? (float *)(a.scratch + p.off_db) : nullptr;
        DwArgs d{g, a.c, dw, db, p.pitch, p.rows_per_split, a.n_out, p.planes};
        const dim3 grid(dw ? (a.c.width + kTile - 1) / kTile : 1, (a.n_out + kTile - 1) / kTile, p.splits);
        if (a.c.act == HPACML_ACT_RELU)
            dw_kernel<true><<<grid, kThreads, 0, st>>>(d);
        else
            dw_kernel<false><<<grid, kThreads, 0, st>>>(d);
        if (dw)
            join_kernel<<<blocks_for((int64_t)a.n_out * a.c.width), kThreads, 0, st>>>(dw, p.splits, a.n_out, a.c.width, a.dw, a.lddw, a.accumulate);
        if (db)
            join_kernel<<<blocks_for(a.n_out), kThreads, 0, st>>>(db, p.splits, 1, a.n_out, a.db, a.n_out, a.accumulate);
    }
    return hipGetLastError();
}

}  // namespace hpacml
