// y = act(s_i t_j sum_k q_ik w_jk + b_j): int8 codes on v_mfma_i32_16x16x64_i8,
// exact 32-bit sums, fp32 epilogue.
#include "dense8_nt.hpp"

namespace hpacml {

namespace {

template <typename Y, int WA, int WB, int NA, int NB>
__global__ void __launch_bounds__(64 * WA * WB, 2) linear8_kernel(Linear8Args p, uint32_t out_tiles, uint32_t point_tiles) {
    typedef nt::Product<nt::I8, Y, true, WA, WB, NA, NB> T;
    __shared__ __align__(1024) char lds[T::kLds];
    const int64_t pitch = (int64_t)p.slabs * 1024, width = (int64_t)p.slabs * kSlabBytes;
    T t;
    t.run({(const char *)p.w, p.n_out, pitch, width, 0}, {(const char *)p.q, p.rows, pitch, width, 0}, out_tiles, point_tiles, 1,
          lds, [&](const i32x4 (&acc)[NA][NB], int64_t a0, int64_t b0) {
              float s[NB];   // asked for before the stores begin
#pragma unroll
              for (int b = 0; b < NB; ++b)
                  s[b] = p.s[min(b0 + t.point_of(b), p.rows - 1)];
              t.store((Y *)p.y, p.ldy, a0, p.n_out, b0, p.rows,
                      [&](int a, int64_t n, int b, float (&v)[4]) {
                          const f32x4 sc = *(const f32x4 *)(p.t + n), bias = *(const f32x4 *)(p.b + n);
#pragma unroll
                          for (int e = 0; e < 4; ++e) {
                              v[e] = (float)acc[a][b][e] * s[b] * sc[e] + bias[e];
                              if (p.relu)
                                  v[e] = relu_keep_nan(v[e]);
                          }
                      },
                      [](int, int, u32x4 &) {});
          });
}

template <typename Y, int WA, int WB, int NA, int NB>
void launch_tile(const Linear8Args &a, hipStream_t stream) {
    typedef nt::Product<nt::I8, Y, true, WA, WB, NA, NB> T;
    const uint32_t out_tiles = (uint32_t)((a.n_out + T::kA - 1) / T::kA), point_tiles = (uint32_t)((a.rows + T::kB - 1) / T::kB);
    linear8_kernel<Y, WA, WB, NA, NB>
        <<<nt::blocks_for_tiles((int64_t)out_tiles * point_tiles, T::kPerCu), T::kThreads, 0, stream>>>(a, out_tiles, point_tiles);
}

template <typename Y>
void launch_as(const Linear8Args &a, hipStream_t stream) {
    const int64_t big = ((a.n_out + 255) / 256) * ((a.rows + 255) / 256);
    const int64_t mid = ((a.n_out + 127) / 128) * ((a.rows + 127) / 128);
    if (big >= 512 && a.slabs >= 32)
        launch_tile<Y, 4, 2, 4, 8>(a, stream);
    else if (mid >= 256 && a.n_out > 64)
        launch_tile<Y, 2, 2, 4, 4>(a, stream);
    else
        launch_tile<Y, 2, 2, 2, 2>(a, stream);
}

}  // namespace

hipError_t launch_linear8(const Linear8Args &a, int32_t y_dtype, hipStream_t stream) {
    if (y_dtype == HPACML_F32)
        launch_as<float>(a, stream);
    else
        launch_as<uint16_t>(a, stream);
    return hipGetLastError();
}

}  // namespace hpacml
