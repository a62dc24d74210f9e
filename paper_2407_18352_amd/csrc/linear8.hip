// y = act(s_i t_j sum_k q_ik w_jk + b_j): int8 codes on v_mfma_i32_16x16x64_i8,
// exact 32-bit sums, fp32 epilogue.
#include "dense8.hpp"

namespace hpacml {

namespace {

constexpr int kThreads = 256;
constexpr int kTile = 64;                    // rows and outputs of a block
constexpr int64_t kMaxBlocks = 1 << 20;       // the kernel loops beyond them
constexpr int kPitch = kSlabBytes + 16;      // of an LDS row

template <typename Y>
__global__ void __launch_bounds__(kThreads) linear8_kernel(Linear8Args p, int64_t tiles, int32_t col_tiles) {
    __shared__ __align__(16) int8_t qs[kTile][kPitch], ws[kTile][kPitch];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wr = (wave & 1) * 32, wc = (wave >> 1) * 32;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t r0 = tile / col_tiles * kTile;
        const int c0 = (int)(tile % col_tiles) * kTile;
        i32x4 acc[2][2] = {};
        for (int64_t k = 0; k < p.pitch; k += kSlabBytes) {
            for (int i = tid; i < kTile * 8; i += kThreads) {
                const int row = i >> 3, chunk = (i & 7) * 16;
                const int64_t r = min(r0 + row, p.rows - 1);
                const int64_t n = min(c0 + row, p.n_out - 1);
                *(i32x4 *)&qs[row][chunk] = *(const i32x4 *)(p.q + r * p.pitch + k + chunk);
                *(i32x4 *)&ws[row][chunk] = *(const i32x4 *)(p.w + n * p.pitch + k + chunk);
            }
            __syncthreads();
            for (int s = 0; s < 2; ++s) {
                i32x4 a[2], b[2];
                for (int t = 0; t < 2; ++t) {
                    a[t] = *(const i32x4 *)&qs[wr + t * 16 + (lane & 15)][s * 64 + (lane >> 4) * 16];
                    b[t] = *(const i32x4 *)&ws[wc + t * 16 + (lane & 15)][s * 64 + (lane >> 4) * 16];
                }
                for (int t = 0; t < 2; ++t)
                    for (int u = 0; u < 2; ++u)
                        acc[t][u] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[t], b[u], acc[t][u], 0, 0, 0);
            }
            __syncthreads();
        }
        for (int t = 0; t < 2; ++t)
            for (int u = 0; u < 2; ++u)
                for (int e = 0; e < 4; ++e) {
                    const int64_t r = r0 + wr + t * 16 + (lane >> 4) * 4 + e;
                    const int n = c0 + wc + u * 16 + (lane & 15);
                    if (r < p.rows && n < p.n_out) {
                        float v = (float)acc[t][u][e] * p.s[r] * p.t[n];
                        if (p.b)
                            v += p.b[n];
                        store_value((Y *)p.y + r * p.ldy + n, p.relu ? relu_keep_nan(v) : v);
                    }
                }
    }
}

}  // namespace

hipError_t launch_linear8(const Linear8Args &a, int32_t y_dtype, hipStream_t stream) {
    const int32_t col_tiles = (a.n_out + kTile - 1) / kTile;
    const int64_t tiles = (a.rows + kTile - 1) / kTile * col_tiles;
    const dim3 grid((uint32_t)(tiles < kMaxBlocks ? tiles : kMaxBlocks));
    if (y_dtype == HPACML_F32)
        linear8_kernel<float><<<grid, kThreads, 0, stream>>>(a, tiles, col_tiles);
    else
        linear8_kernel<uint16_t><<<grid, kThreads, 0, stream>>>(a, tiles, col_tiles);
    return hipGetLastError();
}

}  // namespace hpacml
