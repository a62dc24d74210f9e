// y = act(s_i t_j sum_k q_ik w_jk + b_j): int8 codes on v_mfma_i32_16x16x64_i8,
// exact 32-bit sums, fp32 epilogue.
//
// Three ways, by the number of points and the widths:
//   up to 64 points: few_kernel; one point through 4096 -> 4096 takes 4.4 us of
//     the device when its weights are in the caches, as they are when the same
//     layer is asked again and again (16.8 MB, 3.4 us at a copy's rate);
//   many points of a narrow layer: narrow_kernel, bound by memory; 65,536 x 512
//     -> 512 in bf16 takes 40 us (27 us at a copy's rate);
//   otherwise the codes are formed by a launch of their own and the product is
//     the general one, bound by the matrix cores: 131,072 x 4096 -> 4096 takes
//     0.31 ms for the codes (1.6 GB, 5.2 TB/s) and 1.66-1.8 ms for the product.
#include <type_traits>

#include "dense8_nt.hpp"
#include "dense8_rows.hpp"

namespace hpacml {

namespace {

// A result in fp32 before its activation.  A sum of codes (below 2^29) times a
// point's scale passes fp32's range where the scale is above 2^99, though the
// output's scale may bring it back: a far point's scale is taken in two factors
// (FAR; a rounding of the other points' results may change by it).  Waves with
// such a point run a form of their own: 65,536 x 256 <- 256 in bf16 takes 18.1 us
// so, 22.5 with two factors everywhere, 23.5 with a choice at each value.
constexpr float kFar = 0x1p90f;
template <bool FAR>
__device__ __forceinline__ float scaled(int32_t sum, float s, float t, float bias) {
    if (!FAR)
        return (float)sum * s * t + bias;
    const bool two = s > kFar;
    return (float)sum * (two ? s * 0x1p-64f : s) * t * (two ? 0x1p64f : 1.f) + bias;
}
// one of the wave's points is such a one (not by a NaN)
template <int N>
__device__ __forceinline__ bool any_far(const float (&s)[N]) {
    float most = s[0];
#pragma unroll
    for (int i = 1; i < N; ++i)
        most = fmaxf(most, s[i]);
    return __any(most > kFar);
}

template <typename Y, bool MERGE, int WA, int WB, int NA, int NB>
__global__ void __launch_bounds__(64 * WA * WB, 2) linear8_kernel(Linear8Args p, uint32_t out_tiles, uint32_t point_tiles) {
    typedef nt::Product<nt::I8, Y, true, MERGE, WA, WB, NA, NB> T;
    __shared__ __align__(1024) char lds[T::kLds];
    const int64_t pitch = (int64_t)p.slabs * 1024, width = (int64_t)p.slabs * kSlabBytes;
    T t;
    t.run({(const char *)p.w, p.n_out, pitch, width, 0}, {(const char *)p.q, p.rows, pitch, width, 0}, out_tiles, point_tiles, 1,
          lds, [&](const i32x4 (&acc)[NA][NB], int64_t a0, int64_t b0) {
              float s[NB];   // asked for before the stores begin
#pragma unroll
              for (int b = 0; b < NB; ++b)
                  s[b] = p.s[min(b0 + t.point_of(b), p.rows - 1)];
              auto store = [&](auto far) {
                  t.store((Y *)p.y, p.ldy, a0, p.n_out, b0, p.rows,
                          [&](int a, int64_t n, int b, float (&v)[4]) {
                              const f32x4 sc = *(const f32x4 *)(p.t + n), bias = *(const f32x4 *)(p.b + n);
#pragma unroll
                              for (int e = 0; e < 4; ++e) {
                                  v[e] = scaled<decltype(far)::value>(acc[a][b][e], s[b], sc[e], bias[e]);
                                  if (p.relu)
                                      v[e] = relu_keep_nan(v[e]);
                              }
                          },
                          [](int, int, u32x4 &) {});
              };
              if (any_far(s))
                  store(std::true_type());
              else
                  store(std::false_type());
          });
}

template <typename Y, bool MERGE, int WA, int WB, int NA, int NB>
void launch_tile(const Linear8Args &a, hipStream_t stream) {
    typedef nt::Product<nt::I8, Y, true, MERGE, WA, WB, NA, NB> T;
    const uint32_t out_tiles = (uint32_t)((a.n_out + T::kA - 1) / T::kA), point_tiles = (uint32_t)((a.rows + T::kB - 1) / T::kB);
    linear8_kernel<Y, MERGE, WA, WB, NA, NB>
        <<<nt::blocks_for_tiles((int64_t)out_tiles * point_tiles, T::kPerCu), T::kThreads, 0, stream>>>(a, out_tiles, point_tiles);
}

template <typename Y, bool MERGE>
void launch_tiled(const Linear8Args &a, hipStream_t stream) {
    switch (nt::tile_for(a.n_out, a.rows, a.slabs)) {
    case nt::Size::k64x64: return launch_tile<Y, MERGE, 2, 2, 2, 2>(a, stream);
    case nt::Size::k128x128: return launch_tile<Y, MERGE, 2, 2, 4, 4>(a, stream);
    case nt::Size::k128x256: return launch_tile<Y, MERGE, 2, 4, 4, 4>(a, stream);
    case nt::Size::k256x256: return launch_tile<Y, MERGE, 4, 2, 4, 8>(a, stream);
    }
}

// ---- few points ---------------------------------------------------------------
//
// Up to 64 points: the weights are read once and what counts is how many of
// their bytes are on the way at a time.  A block takes 16 outputs (one per
// fragment row) and all points; its eight waves split k, read their fragments
// straight into registers (the blocked layout is the fragment), and add their
// exact integer sums through LDS.  FUSED (up to 32 points, codes of up to 36
// KB): every block forms the points' codes itself, its weights already on the
// way, which saves a launch: 512 -> 512 in bf16, device us and us of a call from
// the host, so and with a launch for the codes: 8 points 3.5 and 6.6, 5.4 and
// 9.5; 24 points 5.6 and 6.6, 6.0 and 9.6; 48 points 7.9 and 7.8, 6.2 and 9.4.
// 64 points, so and as tiles, device us with the launch for the codes: 512 ->
// 512 6.4 and 7.3, 1024 -> 1024 6.7 and 8.7, 4096 -> 4096 12.7 and 17.1 (128
// points, which have no form here, as tiles 7.3, 8.8 and 17.5).
// Its code is kept short, a chunk or two of a row at a time: with eight of them
// (so that all points' loads were on the way at once) 9 points took 7.3 us.
constexpr int kFewWaves = 8, kFewThreads = 64 * kFewWaves, kFewPoints = 64, kFusedPoints = 32, kFusedBytes = 36 * 1024;
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
        // one point: by the whole block; more: a wave each.  A lane takes kHeld
        // chunks of the row at a time
        const bool one = p.rows == 1;
        const int step = one ? kFewThreads : 64, first = one ? tid : lane, points = (int)p.rows;
        auto form = [&](auto held) {
            constexpr int kHeld = decltype(held)::value;
            float v[kHeld][kChunk];
            for (int r = one ? 0 : wave; r < points; r += kFewWaves) {
                const X *row_at = (const X *)p.x + r * p.ldx;
                auto load = [&](int c) {
                    auto k = [&](int h) { return (c + h * step) * kChunk; };
                    load_chunks<X>(p.n_in, [&](int h) { return row_at + k(h); }, [&](int h) { return p.n_in - k(h); }, v);
                };
                uint32_t top = 0;
                for (int c = first; c < chunks; c += step * kHeld) {
                    load(c);
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
                for (int c = first; c < chunks; c += step * kHeld) {
                    if (chunks > step * kHeld)
                        load(c);
#pragma unroll
                    for (int h = 0; h < kHeld; ++h) {
                        const int at = c + h * step;
                        if (at == 0)
                            scales[r] = sc.scale;
                        if (at < chunks)
                            *(uint2 *)(codes + r * pitch + at * kChunk) = sc.codes(v[h]);
                    }
                }
            }
        };
        if (chunks <= step)
            form(std::integral_constant<int, 1>());
        else
            form(std::integral_constant<int, 2>());
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
        const float scale = FUSED ? scales[b * 16 + point] : p.s[r];
        float v = scaled<true>(sum, scale, p.t[n], p.b[n]);
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
    else if (FUSED || a.rows <= 32)
        few_kernel<X, Y, 2, FUSED><<<grid, kFewThreads, 0, stream>>>(a);
    else if constexpr (!FUSED)
        few_kernel<X, Y, 4, FUSED><<<grid, kFewThreads, 0, stream>>>(a);
}

template <typename Y>
void launch_product(const Linear8Args &a, hipStream_t stream) {
    if (a.rows <= kFewPoints)
        return launch_few<float, Y, false>(a, stream);   // x is not read
    nt::shared_lines(a.y, a.ldy * (int64_t)sizeof(Y)) ? launch_tiled<Y, true>(a, stream) : launch_tiled<Y, false>(a, stream);
}

// ---- narrow layers --------------------------------------------------------------
//
// Up to SLABS * 64 inputs and many points: a block takes its points' rows whole,
// forms their codes in LDS, and goes through all outputs with them, so that the
// codes never lie in memory, which is what bounds these products.  The weights
// come as fragments straight from the L2, a slab ahead.
template <typename Y, int SLABS, int WA, int WB, int NA, int NB>
struct Narrow {
    static constexpr int kPoints = 16 * NB * WB, kRows = kPoints / 4, kOuts = 16 * NA * WA;
    static constexpr int kCodes = kPoints / 16 * SLABS * 1024, kOut = 4 * 16 * nt::Out<Y, NA>::kRow;
    static constexpr int kFit = 160 * 1024 / (kCodes + kOut);
    // 64 points of fp32 results have no room in a quarter of a CU's registers:
    // 65,536 x 256 <- 256 in fp32 takes 32.9 us with four blocks of them a CU, 27.1
    // with three
    static constexpr int kMost = sizeof(Y) == 4 && NB == 4 ? 3 : 4;
    static constexpr int kPerCu = kPoints == 128 ? 2 : kFit < kMost ? kFit : kMost;
    static_assert(WA * WB == 4 && kPerCu >= 2, "four waves, two blocks");
};

template <typename X, typename Y, int SLABS, int WA, int WB, int NA, int NB>
__global__ void __launch_bounds__(256, (Narrow<Y, SLABS, WA, WB, NA, NB>::kPerCu)) narrow_kernel(Linear8Args p) {
    typedef Narrow<Y, SLABS, WA, WB, NA, NB> N;
    constexpr int kPoints = N::kPoints, kRows = N::kRows, kOuts = N::kOuts, kBatch = 8;
    typedef nt::Out<Y, NA> Out;
    __shared__ __align__(1024) char codes[N::kCodes];
    __shared__ __align__(16) char out[N::kOut];      // the points' scales first
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t p0 = (int64_t)blockIdx.x * kPoints;
    float *scales = (float *)out;

    // codes: 2^lanes_log lanes per row, a chunk each
    const int chunks = p.slabs * (kSlabBytes / kChunk);
    int lanes_log = 3;
    while ((1 << lanes_log) < chunks)
        ++lanes_log;
    const int lanes = 1 << lanes_log, per = 64 >> lanes_log, c = lane & (lanes - 1), k = c * kChunk;
    for (int r0 = wave * kRows; r0 < wave * kRows + kRows; r0 += per * kBatch) {
        float v[kBatch][kChunk];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int64_t r = min(p0 + min(r0 + i * per + (lane >> lanes_log), kPoints - 1), p.rows - 1);
            load_chunk((const X *)p.x + r * p.ldx + k, p.n_in - k, v[i]);
        }
        uint32_t top[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
            top[i] = top_bits(v[i]);
        for (int d = lanes / 2; d > 0; d /= 2)
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                top[i] = max(top[i], (uint32_t)__shfl_xor((int)top[i], d));
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const RowScale sc(top[i]);
            const int r = r0 + i * per + (lane >> lanes_log);
            if (r < wave * kRows + kRows) {
                if (c == 0)
                    scales[r] = sc.scale;
                if (c < chunks)
                    *(uint2 *)(codes + blocked_offset(r, k, p.slabs)) = sc.codes(v[i]);
            }
        }
    }
    __syncthreads();

    const int wa = wave / WB, wb = wave % WB, row = lane & 15;
    const int at = row * kSlabBytes + (((lane >> 4) ^ chunk_turn(row)) * 16);
    float s[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
        s[b] = scales[(wb * NB + b) * 16 + row];
    __syncthreads();                                   // the scales' place is the results' now

    const int last = (p.n_out - 1) / 16;               // 16 outputs
    auto weights = [&](int pass, int slab, u32x4 (&a)[NA]) {
#pragma unroll
        for (int t = 0; t < NA; ++t)
            a[t] = *(const u32x4 *)(p.w + ((int64_t)min(pass * (kOuts / 16) + wa * NA + t, last) * p.slabs + slab) * 1024 + at);
    };
    auto go = [&](auto far) {
        u32x4 a[NA], next[NA];
        weights(0, 0, a);
        const int passes = (p.n_out + kOuts - 1) / kOuts;
        for (int pass = 0; pass < passes; ++pass) {
            i32x4 acc[NA][NB] = {};
            for (int slab = 0; slab < p.slabs; ++slab) {
                const bool more = slab + 1 < p.slabs;
                weights(more ? pass : min(pass + 1, passes - 1), more ? slab + 1 : 0, next);
                u32x4 b[NB];
#pragma unroll
                for (int u = 0; u < NB; ++u)
                    b[u] = *(const u32x4 *)(codes + ((wb * NB + u) * p.slabs + slab) * 1024 + at);
#pragma unroll
                for (int u = 0; u < NB; ++u)
#pragma unroll
                    for (int t = 0; t < NA; ++t)
                        acc[t][u] = nt::I8::mul(a[t], b[u], acc[t][u]);
#pragma unroll
                for (int t = 0; t < NA; ++t)
                    a[t] = next[t];
            }
            const int64_t a0 = (int64_t)pass * kOuts + wa * NA * 16;
            if (a0 < p.n_out)
                Out::template store<NB, false>(out + wave * 16 * Out::kRow, lane, (Y *)p.y, p.ldy, a0, p.n_out, p0 + wb * NB * 16, p.rows,
                                        [&](int t, int64_t n, int u, float (&v)[4]) {
                                            const f32x4 sc = *(const f32x4 *)(p.t + n), bias = *(const f32x4 *)(p.b + n);
#pragma unroll
                                            for (int e = 0; e < 4; ++e) {
                                                v[e] = scaled<decltype(far)::value>(acc[t][u][e], s[u], sc[e], bias[e]);
                                                if (p.relu)
                                                    v[e] = relu_keep_nan(v[e]);
                                            }
                                        },
                                        [](int, int, u32x4 &) {});
        }
    };
    if (any_far(s))
        go(std::true_type());
    else
        go(std::false_type());
}

template <typename X, typename Y, int SLABS, int WA, int WB, int NB>
void launch_narrow_tile(const Linear8Args &a, hipStream_t stream) {
    constexpr int kPoints = Narrow<Y, SLABS, WA, WB, 4, NB>::kPoints;
    narrow_kernel<X, Y, SLABS, WA, WB, 4, NB><<<dim3((uint32_t)((a.rows + kPoints - 1) / kPoints)), 256, 0, stream>>>(a);
}

// Points of a block: 64, of which four share a CU; with few outputs and enough
// rows for as many larger blocks 128 (device us, 64 and 128, and with the codes
// in memory: 262144 x 64 <- 64 27.2, 20.2, 28.9; 131072 x 64 <- 64 13.3, 9.8,
// 19.9; 262144 x 128 <- 128 38.1, 34.3, 45.5; 100000 x 128 <- 128 16.2, 17.9,
// 23.1; 65521 x 50 <- 201 in fp32 18.6, 21.2, 23.3; against the rule 131072 x
// 100 <- 300 54.4, 82.2, 63.7).
template <typename X, typename Y, int SLABS>
void launch_narrow(const Linear8Args &a, hipStream_t stream) {
    const bool many = a.rows >= 131072;
    if (a.n_out <= 64)
        many ? launch_narrow_tile<X, Y, SLABS, 1, 4, 2>(a, stream) : launch_narrow_tile<X, Y, SLABS, 1, 4, 1>(a, stream);
    else if (a.n_out <= 128)
        many ? launch_narrow_tile<X, Y, SLABS, 2, 2, 4>(a, stream) : launch_narrow_tile<X, Y, SLABS, 2, 2, 2>(a, stream);
    else
        launch_narrow_tile<X, Y, SLABS, 4, 1, 4>(a, stream);
}

bool few_fused(int64_t rows, int32_t n_in) {
    return rows <= kFusedPoints && rows * fused_pitch(slabs_of(n_in)) <= kFusedBytes;
}
// Device us this way and with the codes in memory, in bf16:
//   16384 x 512 <- 512     23.6  20.0      24576 x 512 <- 512    26.6  26.7
//   32768 x 512 <- 512     28.9  30.0      65536 x 512 <- 512    40.1  49.6
//   32768 x 1024 <- 256    27.4  32.5      65536 x 1024 <- 256   45.0  54.1
//   32768 x 1024 <- 512    44.7  40.6      65536 x 1024 <- 512   64.8  73.8
//   32768 x 1500 <- 512    79.6  57.2      65536 x 1500 <- 512    160   110
//   16384 x 64 <- 64        5.5   7.2      16384 x 1024 <- 256   23.5  19.8
// (in fp32 32768 x 1024 <- 512 48.7 and 52.6)
constexpr int64_t kNarrowPoints = 32768;
bool narrow(int64_t rows, int32_t n_in, int32_t n_out) { return rows >= kNarrowPoints && rows <= (1 << 30) && n_in <= 512 && n_out <= 1024; }

template <typename X, typename Y>
void launch_as(const Linear8Args &a, hipStream_t stream) {
    if (few_fused(a.rows, a.n_in))
        launch_few<X, Y, true>(a, stream);
    else if (narrow(a.rows, a.n_in, a.n_out))
        a.slabs <= 4 ? launch_narrow<X, Y, 4>(a, stream) : launch_narrow<X, Y, 8>(a, stream);
    else
        launch_product<Y>(a, stream);
}

}  // namespace

int64_t linear8_scratch_rows(int64_t rows, int32_t n_in, int32_t n_out) {
    return narrow(rows, n_in, n_out) ? kNarrowPoints - 1 : rows;
}

hipError_t launch_linear8(const Linear8Args &a, int32_t x_dtype, int32_t y_dtype, hipStream_t stream) {
    if (!few_fused(a.rows, a.n_in) && !narrow(a.rows, a.n_in, a.n_out)) {
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
