// y = act(s_i t_j sum_k q_ik w_jk + b_j): int8 codes on v_mfma_i32_16x16x64_i8,
// exact 32-bit sums, fp32 epilogue.
#include "dense8_nt.hpp"
#include "dense8_rows.hpp"

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

// ---- few points ---------------------------------------------------------------
//
// Up to 64 points: the weights are read once and what counts is how many of
// their bytes are on the way at a time.  A block takes 16 outputs (one per
// fragment row) and all points; its eight waves split k, read their fragments
// straight into registers (the blocked layout is the fragment), and add their
// exact integer sums through LDS.  FUSED (codes of up to 36 KB): every block
// forms the points' codes itself, its weights already on the way, which saves
// a launch.  One point through 4096 -> 4096: 4.9 us.
constexpr int kFewWaves = 8, kFewThreads = 64 * kFewWaves, kFewPoints = 64, kFusedBytes = 36 * 1024;
// of a row of codes in LDS: 16 rows at one k lie on different banks
constexpr int64_t fused_pitch(int64_t slabs) { return slabs * kSlabBytes + 16; }

template <typename X, typename Y, int P, bool FUSED>
__global__ void __launch_bounds__(kFewThreads) few_kernel(Linear8Args p) {
    constexpr int kAhead = P == 4 ? 4 : 8;           // slabs of a wave on the way at a time
    __shared__ __align__(16) int32_t part[kFewWaves][P][256];
    __shared__ __align__(16) int8_t codes[FUSED ? kFusedBytes : 16];
    __shared__ float scales[P * 16];
    __shared__ uint32_t tops[kFewWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = lane & 15;
    const int at = row * kSlabBytes + (((lane >> 4) ^ chunk_turn(row)) * 16);
    const int8_t *w = p.w + (int64_t)blockIdx.x * p.slabs * 1024 + at;
    const int pitch = (int)fused_pitch(p.slabs), chunks = p.slabs * (kSlabBytes / kChunk);

    u32x4 a[kAhead];
    auto weights = [&](int s0) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            a[i] = *(const u32x4 *)(w + (int64_t)min(s0 + i * kFewWaves, p.slabs - 1) * 1024);
    };
    weights(wave);

    if constexpr (FUSED) {
        // one point: by the whole block; more: a wave each
        const bool one = p.rows == 1;
        const int step = one ? kFewThreads : 64, first = one ? tid : lane;
        constexpr int kHeld = 4;
        float v[kHeld][kChunk];
        for (int r = one ? 0 : wave; r < p.rows; r += kFewWaves) {
            const X *x = (const X *)p.x + r * p.ldx;
            uint32_t top = 0;
            for (int c = first; c < chunks; c += kHeld * step) {
#pragma unroll
                for (int h = 0; h < kHeld; ++h) {
                    const int k = (c + h * step) * kChunk;
                    load_chunk(x + k, p.n_in - k, v[h]);
                }
#pragma unroll
                for (int h = 0; h < kHeld; ++h)
                    top = max(top, top_bits(v[h]));
            }
            top = lanes_max<64>(top);
            if (one) {
                if (lane == 0)
                    tops[wave] = top;
                __syncthreads();
#pragma unroll
                for (int i = 0; i < kFewWaves; ++i)
                    top = max(top, tops[i]);
            }
            const RowScale sc(top);
            if (first == 0)
                scales[r] = sc.scale;
            for (int c = first; c < chunks; c += kHeld * step) {
#pragma unroll
                for (int h = 0; h < kHeld; ++h) {
                    const int k = (c + h * step) * kChunk;
                    if (chunks > kHeld * step)
                        load_chunk(x + k, p.n_in - k, v[h]);
                    if (c + h * step < chunks)
                        *(uint2 *)(codes + r * pitch + k) = sc.codes(v[h]);
                }
            }
        }
        __syncthreads();
    }

    i32x4 acc[P] = {};
    for (int s0 = wave; s0 < p.slabs; s0 += kAhead * kFewWaves) {
        if (s0 != wave)
            weights(s0);
        // past the last slab: weights of that one, codes of 0
        u32x4 q[kAhead][P];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int s = min(s0 + i * kFewWaves, p.slabs - 1);
#pragma unroll
            for (int b = 0; b < P; ++b)
                q[i][b] = FUSED ? *(const u32x4 *)(codes + min(b * 16 + row, (int)p.rows - 1) * pitch + s * kSlabBytes + (lane >> 4) * 16)
                                : *(const u32x4 *)(p.q + ((int64_t)min(b, (int)((p.rows - 1) >> 4)) * p.slabs + s) * 1024 + at);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int b = 0; b < P; ++b)
                acc[b] = nt::I8::mul(a[i], s0 + i * kFewWaves < p.slabs ? q[i][b] : u32x4{0, 0, 0, 0}, acc[b]);
    }
#pragma unroll
    for (int b = 0; b < P; ++b)
        *(i32x4 *)&part[wave][b][lane * 4] = acc[b];
    __syncthreads();
    for (int i = tid; i < P * 256; i += kFewThreads) {
        // 16 threads after one another store 16 outputs of a point
        const int b = i >> 8, point = (i >> 4) & 15, o = i & 15, from = ((o >> 2) * 16 + point) * 4 + (o & 3);
        const int64_t r = b * 16 + point;
        const int n = blockIdx.x * 16 + o;
        if (r >= p.rows || n >= p.n_out)
            continue;
        int32_t sum = 0;
#pragma unroll
        for (int k = 0; k < kFewWaves; ++k)
            sum += part[k][b][from];
        float v = (float)sum * (FUSED ? scales[b * 16 + point] : p.s[r]) * p.t[n] + p.b[n];
        if (p.relu)
            v = relu_keep_nan(v);
        store_value((Y *)p.y + r * p.ldy + n, v);
    }
}

template <typename X, typename Y, bool FUSED>
void launch_few(const Linear8Args &a, hipStream_t stream) {
    const dim3 grid((a.n_out + 15) / 16);
    if (a.rows <= 16)
        few_kernel<X, Y, 1, FUSED><<<grid, kFewThreads, 0, stream>>>(a);
    else if (a.rows <= 32)
        few_kernel<X, Y, 2, FUSED><<<grid, kFewThreads, 0, stream>>>(a);
    else
        few_kernel<X, Y, 4, FUSED><<<grid, kFewThreads, 0, stream>>>(a);
}

template <typename Y>
void launch_product(const Linear8Args &a, hipStream_t stream) {
    if (a.rows <= kFewPoints)
        return launch_few<float, Y, false>(a, stream);   // x is not read
    switch (nt::tile_for(a.n_out, a.rows, a.slabs)) {
    case nt::Size::k64x64: return launch_tile<Y, 2, 2, 2, 2>(a, stream);
    case nt::Size::k128x128: return launch_tile<Y, 2, 2, 4, 4>(a, stream);
    case nt::Size::k128x256: return launch_tile<Y, 2, 4, 4, 4>(a, stream);
    case nt::Size::k256x256: return launch_tile<Y, 4, 2, 4, 8>(a, stream);
    }
}

template <typename X, typename Y>
void launch_as(const Linear8Args &a, hipStream_t stream) {
    if (linear8_fused(a.rows, a.n_in))
        launch_few<X, Y, true>(a, stream);
    else
        launch_product<Y>(a, stream);
}

}  // namespace

bool linear8_fused(int64_t rows, int32_t n_in) {
    return rows <= kFewPoints && rows * fused_pitch(slabs_of(n_in)) <= kFusedBytes;
}

hipError_t launch_linear8(const Linear8Args &a, int32_t x_dtype, int32_t y_dtype, hipStream_t stream) {
    if (!linear8_fused(a.rows, a.n_in)) {
        const hipError_t e = launch_codes_by_row(a.x, x_dtype, a.ldx, a.rows, a.n_in, a.q, a.s, stream);
        if (e != hipSuccess)
            return e;
    }
    if (x_dtype == HPACML_F32)
        y_dtype == HPACML_F32 ? launch_as<float, float>(a, stream) : launch_as<float, uint16_t>(a, stream);
    else
        y_dtype == HPACML_F32 ? launch_as<uint16_t, float>(a, stream) : launch_as<uint16_t, uint16_t>(a, stream);
    return hipGetLastError();
}

}  // namespace hpacml
