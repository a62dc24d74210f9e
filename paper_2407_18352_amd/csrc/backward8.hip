// The backward pass of a linear layer whose input was kept in 8 bits:
//   dw = dy^T a, db = the sum of dy's rows, dx = (dy W) where the codes are not 0.
// A kept value (8 significant bits times a power of two) is exact in bf16, so
// dw's products are exact on v_mfma_f32_16x16x32_bf16 and summed in fp32.  An
// fp32 operand is the exact sum of three bf16 terms: three products for dw,
// for dx those six of nine whose terms' ranks sum to at most 2.
#include "dense8_nt.hpp"

namespace hpacml {

namespace {

constexpr int kThreads = 256;             // of the kernels that lay operands out and join parts
constexpr int64_t kMaxBlocks = 1 << 16;   // they loop beyond them

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

// planes of W's transpose [n_in][n_out], blocked, zero beyond n_out
template <typename T>
__global__ void __launch_bounds__(kThreads) transpose_kernel(const T *__restrict__ W, int64_t ldw, int32_t n_out,
                                                             int32_t n_in, char *__restrict__ out, int32_t slabs) {
    const int64_t plane = blocked_bytes(n_in, slabs), pitch = (int64_t)slabs * (kSlabBytes / 2);
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n_in * pitch; i += (int64_t)gridDim.x * kThreads) {
        const int64_t k = i / pitch, j = i - k * pitch;
        char *at = out + blocked_offset(k, 2 * j, slabs);
        if constexpr (sizeof(T) == 4) {
            uint16_t t[3] = {0, 0, 0};
            if (j < n_out)
                split3(W[j * ldw + k], t);
            for (int q = 0; q < 3; ++q)
                *(uint16_t *)(at + q * plane) = t[q];
        } else {
            *(uint16_t *)at = j < n_out ? W[j * ldw + k] : (uint16_t)0;
        }
    }
}

// ---- dx -------------------------------------------------------------------------

struct DxArgs {
    nt::Operand wt, g;          // W's transpose [n_in][n_out], blocked, and dy, in rows
    const uint8_t *codes;       // NULL: everything is let through
    void *dx;
    int64_t ld_codes, lddx;
    int32_t n_in, terms;
    uint32_t in_tiles, point_tiles;
};

template <typename X, int WA, int WB, int NA, int NB>
__global__ void __launch_bounds__(64 * WA * WB) dx_kernel(DxArgs p) {
    typedef nt::Tile<nt::Bf16, WA, WB, NA, NB> T;
    __shared__ __align__(1024) char lds[T::kLds];
    const nt::TileAt at = nt::tile_at(blockIdx.x, gridDim.x, p.in_tiles, p.point_tiles);
    const int64_t a0 = at.out * T::kA, b0 = at.point * T::kB;
    f32x4 acc[NA][NB] = {};
    T t;
    t.template run<false>(p.wt, p.g, a0, b0, p.terms, lds, acc);
    t.store((X *)p.dx, p.lddx, a0, p.n_in, b0, p.g.rows, lds,
            [&](int a, int64_t, int b, int64_t, float (&v)[4]) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = acc[a][b][e];
            },
            [&](int64_t r, int64_t k, u32x4 &u) {
                if (!p.codes)
                    return;
                // rows of codes are whole blocks of channels: all of these exist
                const uint8_t *c = p.codes + r * p.ld_codes + k;
                if constexpr (sizeof(X) == 2) {
                    const uint2 q = *(const uint2 *)c;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t two = (e < 2 ? q.x : q.y) >> (16 * (e & 1));
                        u[e] &= (two & 0xFFu ? 0x0000FFFFu : 0u) | (two & 0xFF00u ? 0xFFFF0000u : 0u);
                    }
                } else {
                    const uint32_t q = *(const uint32_t *)c;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        u[e] = (q >> (8 * e)) & 0xFFu ? u[e] : 0u;
                }
            });
}

// ---- dw and db ------------------------------------------------------------------
//
// The sum runs over the rows, along which neither operand is contiguous: both
// go to LDS as they lie, [row][column] in bf16, and the fragments come out
// transposed (ds_read_tr16_b64: 16 lanes read 4 rows x 16 columns and get one
// column's 4 rows each).  dy is loaded straight to LDS; the codes pass through
// registers, where they become bf16 values.  Slabs of 64 rows, double-buffered:
// during a slab the next one's dy loads, its codes (loaded a slab earlier) are
// converted and written, and the codes of the one after are fetched.
//
// A row of a slab is pairs of 16-byte chunks (16 columns); pair p is stored at
// p ^ turn(row), so that the rows a transposing read touches at one pair lie
// on different banks.
struct DwArgs {
    const char *g;              // dy's planes
    int64_t g_pitch, g_width;   // bytes; columns from the width on read as 0
    int64_t g_plane;
    hpacml8_checkpoint c;
    float *dw, *db;             // parts: dw [splits][n_out][n_in], db [splits][n_out]; NULL: not wanted
    int64_t rows_per_split;
    int32_t n_out, planes;
    uint32_t out_tiles, in_tiles;
};

template <bool RELU, int WA, int WB, int NA, int NB>
struct DwTile {
    static constexpr int kWaves = WA * WB, kThreads = 64 * kWaves, kRows = 64;
    static constexpr int kA = 16 * NA * WA, kB = 16 * NB * WB;          // outputs, channels
    static constexpr int kPitchA = 2 * kA, kPitchB = 2 * kB;            // bytes of an LDS row
    static constexpr int kBufA = kRows * kPitchA, kBufB = kRows * kPitchB, kBuf = kBufA + kBufB;
    static constexpr int kLoadsA = kBufA / (1024 * kWaves);             // direct loads of a wave per slab
    static constexpr int kChunks = kRows * kB / 16 / kThreads;          // 16 codes each, per thread and slab
    static_assert(kLoadsA >= 1 && kChunks >= 1 && kChunks * 16 * kThreads == kRows * kB, "whole shares");

    // which pair of an LDS row column pair 0 is at
    template <int PAIRS>
    static __device__ __forceinline__ int turn(int row) {
        return ((row & 3) | ((row >> 1) & 4)) & (PAIRS - 1);
    }
    // fragment of 16 columns from `col` on, 32 rows from `row` on: lane l gets column l % 16, rows 8 (l / 16) + 0..7
    template <int PITCH>
    static __device__ __forceinline__ bf16x8 fragment(const char *buf, int row, int col, int lane) {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 *Lds;
        const int r = row + (lane >> 4) * 8 + ((lane & 15) >> 2);
        const char *a = buf + r * PITCH + (((col >> 4) ^ turn<PITCH / 32>(r)) * 32) + (lane & 3) * 8;
        const char *b = buf + (r + 4) * PITCH + (((col >> 4) ^ turn<PITCH / 32>(r + 4)) * 32) + (lane & 3) * 8;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)a), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)b);
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        return __builtin_bit_cast(bf16x8, (s16x8){lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    }
};

template <bool RELU, int WA, int WB, int NA, int NB>
__global__ void __launch_bounds__(64 * WA * WB) dw_kernel(DwArgs p) {
    typedef DwTile<RELU, WA, WB, NA, NB> T;
    __shared__ __align__(1024) char lds[2 * T::kBuf];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wa = wave / WB, wb = wave % WB;

    // the tiles of one part of the rows follow one another on one XCD
    const uint32_t blocks = gridDim.x, xcd = blockIdx.x & 7, per = blocks >> 3, more = blocks & 7;
    const uint32_t id = xcd * per + min(xcd, more) + (blockIdx.x >> 3), tiles = p.out_tiles * p.in_tiles;
    const uint32_t part = id / tiles, tile = id - part * tiles;
    const int j0 = (int)(tile / p.in_tiles) * T::kA, k0 = (int)(tile % p.in_tiles) * T::kB;
    const int64_t from = part * p.rows_per_split, to = min(from + p.rows_per_split, p.c.rows);
    const int slabs = to > from ? (int)((to - from + T::kRows - 1) / T::kRows) : 0, total = slabs * p.planes;

    // dy: lane's place in a direct load, and the column that belongs there
    const uint32_t base = nt::lds_offset(lds);
    auto load_g = [&](int s, int buf) {
        const int plane = p.planes - 1 - s / slabs;          // the smallest terms first
        const int64_t r0 = from + (int64_t)(s % slabs) * T::kRows;
        const char *g = p.g + plane * p.g_plane;
#pragma unroll
        for (int i = 0; i < T::kLoadsA; ++i) {
            const int at = (i * T::kWaves + wave) * 1024 + lane * 16;
            const int row = at / T::kPitchA, chunk = at % T::kPitchA / 16;
            const int col = ((chunk >> 1) ^ T::template turn<T::kPitchA / 32>(row)) * 32 + (chunk & 1) * 16 + j0 * 2;   // bytes
            const void *src = g + (r0 + row) * p.g_pitch + col;
            if (r0 + row >= to || col >= p.g_width)
                src = nt::zero_chunk;
            nt::load_to_lds(src, base + buf * T::kBuf + (i * T::kWaves + wave) * 1024);
        }
    };
    // codes: 16 columns of a row each
    u32x4 code[T::kChunks];
    uint32_t byte[T::kChunks];
    const int code_cols = (p.c.width + 31) / 32 * 32;
    auto load_x = [&](int s) {
        const int64_t r0 = from + (int64_t)(s % slabs) * T::kRows;
#pragma unroll
        for (int i = 0; i < T::kChunks; ++i) {
            const int at = i * T::kThreads + threadIdx.x, row = at / (T::kB / 16);
            const int64_t r = min(r0 + row, to - 1);
            int col = k0 + at % (T::kB / 16) * 16;
            col = col < code_cols ? col : 0;                 // beyond the width: any codes
            code[i] = *(const u32x4 *)((const uint8_t *)p.c.codes + r * p.c.ld_codes + col);
            byte[i] = r0 + row < to ? ((const uint8_t *)p.c.exps)[r * p.c.ld_exps + col / 32] : 0u;   // 0: 2^e reads as 0
        }
    };
    auto write_x = [&](int buf) {
#pragma unroll
        for (int i = 0; i < T::kChunks; ++i) {
            const int at = i * T::kThreads + threadIdx.x, row = at / (T::kB / 16), pair = at % (T::kB / 16);
            const float s = block_scale(byte[i]);
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t q = code[i][e / 2] >> (16 * (e & 1));
                const float lo = block_value<RELU>(q & 0xFFu, s), hi = block_value<RELU>((q >> 8) & 0xFFu, s);
                // exact in bf16: the high halves
                w[e] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo), 0x07060302u);
            }
            char *to_lds = lds + buf * T::kBuf + T::kBufA + row * T::kPitchB + ((pair ^ T::template turn<T::kPitchB / 32>(row)) * 32);
            ((u32x4 *)to_lds)[0] = u32x4{w[0], w[1], w[2], w[3]};
            ((u32x4 *)to_lds)[1] = u32x4{w[4], w[5], w[6], w[7]};
        }
    };

    f32x4 acc[NA][NB] = {}, sum[NA] = {};
    const bool sums = p.db && k0 == 0 && wb == 0;
    const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u});
    if (total > 0) {
        load_g(0, 0);
        load_x(0);
        write_x(0);
        if (total > 1)
            load_x(1);
    }
    for (int s = 0; s < total; ++s) {
        nt::wait_loads<0>();
        nt::barrier();
        const char *buf = lds + (s & 1) * T::kBuf;
        if (s + 1 < total) {
            load_g(s + 1, (s + 1) & 1);
            write_x((s + 1) & 1);
            if (s + 2 < total)
                load_x(s + 2);
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            bf16x8 a[NA], b[NB];
#pragma unroll
            for (int t = 0; t < NA; ++t)
                a[t] = T::template fragment<T::kPitchA>(buf, ks * 32, (wa * NA + t) * 16, lane);
#pragma unroll
            for (int t = 0; t < NB; ++t)
                b[t] = T::template fragment<T::kPitchB>(buf + T::kBufA, ks * 32, (wb * NB + t) * 16, lane);
#pragma unroll
            for (int t = 0; t < NA; ++t)
#pragma unroll
                for (int u = 0; u < NB; ++u)
                    acc[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[t], b[u], acc[t][u], 0, 0, 0);
            if (sums) {
#pragma unroll
                for (int t = 0; t < NA; ++t)
                    sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[t], ones, sum[t], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < NA; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int j = j0 + (wa * NA + t) * 16 + (lane >> 4) * 4 + e;
            if (j >= p.n_out)
                continue;
            if (sums && (lane & 15) == 0)
                p.db[(int64_t)part * p.n_out + j] = sum[t][e];
            if (p.dw) {
#pragma unroll
                for (int u = 0; u < NB; ++u) {
                    const int k = k0 + (wb * NB + u) * 16 + (lane & 15);
                    if (k < p.c.width)
                        p.dw[((int64_t)part * p.n_out + j) * p.c.width + k] = acc[t][u][e];
                }
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
    return dim3((uint32_t)(n < 1 ? 1 : n < kMaxBlocks ? n : kMaxBlocks));
}
size_t whole(size_t b) { return (b + 255) / 256 * 256; }

int64_t tiles_of(int64_t a, int64_t b, int64_t tile) { return (a + tile - 1) / tile * ((b + tile - 1) / tile); }

// Tile of dw: the largest that a gradient of this size fills.
int dw_tile(int32_t n_out, int32_t n_in) {
    return n_out <= 64 || n_in <= 64 ? 64 : tiles_of(n_out, n_in, 256) < 16 ? 128 : 256;
}

template <typename X, int WA, int WB, int NA, int NB>
void launch_dx_tile(const DxArgs &a, hipStream_t st) {
    typedef nt::Tile<nt::Bf16, WA, WB, NA, NB> T;
    DxArgs d = a;
    d.in_tiles = (uint32_t)((a.n_in + T::kA - 1) / T::kA);
    const int64_t step = nt::rows_per_launch(d.in_tiles, T::kB);
    for (int64_t r = 0; r < a.g.rows; r += step) {
        d.g.rows = a.g.rows - r < step ? a.g.rows - r : step;
        d.g.base = a.g.base + r * a.g.pitch;
        d.codes = a.codes ? a.codes + r * a.ld_codes : nullptr;
        d.dx = (X *)a.dx + r * a.lddx;
        d.point_tiles = (uint32_t)((d.g.rows + T::kB - 1) / T::kB);
        dx_kernel<X, WA, WB, NA, NB><<<dim3(d.in_tiles * d.point_tiles), T::kThreads, 0, st>>>(d);
    }
}

template <typename X>
void launch_dx(const DxArgs &d, hipStream_t st) {
    if (tiles_of(d.g.rows, d.n_in, 256) >= 512 && d.wt.width >= 2048)
        launch_dx_tile<X, 4, 2, 4, 8>(d, st);
    else if (tiles_of(d.g.rows, d.n_in, 128) >= 256 && d.n_in > 64)
        launch_dx_tile<X, 2, 2, 4, 4>(d, st);
    else
        launch_dx_tile<X, 2, 2, 2, 2>(d, st);
}

template <bool RELU>
void launch_dw(const DwArgs &d, uint32_t blocks, int tile, hipStream_t st) {
    if (tile == 256)
        dw_kernel<RELU, 4, 2, 4, 8><<<blocks, 512, 0, st>>>(d);
    else if (tile == 128)
        dw_kernel<RELU, 2, 2, 4, 4><<<blocks, 256, 0, st>>>(d);
    else
        dw_kernel<RELU, 2, 2, 2, 2><<<blocks, 256, 0, st>>>(d);
}

}  // namespace

Backward8Plan backward8_plan(const hpacml8_checkpoint &c, const void *dy, int32_t dtype, int64_t lddy, int32_t n_out,
                             bool want_dw, bool want_dx) {
    Backward8Plan p{};
    p.planes = dtype == HPACML_F32 ? 3 : 1;
    p.direct = dtype == HPACML_BF16 && ((uintptr_t)dy & 15) == 0 && lddy % 8 == 0 && n_out % 8 == 0;
    p.slabs = (int32_t)slabs_of(2 * n_out);
    p.pitch = (int64_t)p.slabs * (kSlabBytes / 2);
    p.tile = dw_tile(n_out, c.width);
    p.splits = 1;
    if (want_dw) {
        // one round of the chip: a block of the largest tile fills a CU's LDS,
        // two of the middle one and four of the smallest do
        const int64_t tiles = tiles_of(n_out, c.width, p.tile), least = p.tile == 64 ? 256 : 512;
        int64_t splits = (p.tile == 256 ? 256 : p.tile == 128 ? 512 : 1024) / tiles;
        const int64_t most = c.rows / least;
        splits = splits < most ? splits : most;
        splits = splits < 1 ? 1 : splits;
        p.rows_per_split = ((c.rows + splits - 1) / splits + 63) / 64 * 64;
        p.splits = p.rows_per_split ? (int32_t)((c.rows + p.rows_per_split - 1) / p.rows_per_split) : 1;
    }
    size_t at = 0;
    p.off_dy = at;
    if (!p.direct)
        at += whole((size_t)p.planes * c.rows * p.pitch * 2);
    p.off_wt = at;
    if (want_dx)
        at += whole((size_t)p.planes * blocked_bytes(c.width, p.slabs));
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
    uint16_t *planes = (uint16_t *)(a.scratch + p.off_dy);
    char *wt = a.scratch + p.off_wt;
    nt::Operand g{(const char *)planes, rows, p.pitch * 2, p.pitch * 2, rows * p.pitch * 2};
    if (p.direct)
        g = {(const char *)a.dy, rows, a.lddy * 2, (int64_t)a.n_out * 2, 0};
    else if (rows > 0 && f32)
        planes_kernel<float><<<blocks_for(rows * p.pitch), kThreads, 0, st>>>((const float *)a.dy, a.lddy, rows, a.n_out, planes, p.pitch);
    else if (rows > 0)
        planes_kernel<uint16_t><<<blocks_for(rows * p.pitch), kThreads, 0, st>>>((const uint16_t *)a.dy, a.lddy, rows, a.n_out, planes, p.pitch);
    if (a.dx && rows > 0) {
        if (f32)
            transpose_kernel<float><<<blocks_for(a.c.width * p.pitch), kThreads, 0, st>>>((const float *)a.W, a.ldw, a.n_out, a.c.width, wt, p.slabs);
        else
            transpose_kernel<uint16_t><<<blocks_for(a.c.width * p.pitch), kThreads, 0, st>>>((const uint16_t *)a.W, a.ldw, a.n_out, a.c.width, wt, p.slabs);
        DxArgs d{};
        d.wt = {wt, a.c.width, (int64_t)p.slabs * 1024, (int64_t)p.slabs * kSlabBytes, blocked_bytes(a.c.width, p.slabs)};
        d.g = g;
        d.codes = a.c.act == HPACML_ACT_RELU ? (const uint8_t *)a.c.codes : nullptr;
        d.dx = a.dx;
        d.ld_codes = a.c.ld_codes;
        d.lddx = a.lddx;
        d.n_in = a.c.width;
        d.terms = p.planes;
        if (f32)
            launch_dx<float>(d, st);
        else
            launch_dx<uint16_t>(d, st);
    }
    if (a.dw || a.db) {
        DwArgs d{};
        d.g = g.base;
        d.g_pitch = g.pitch;
        d.g_width = g.width;
        d.g_plane = g.plane;
        d.c = a.c;
        d.dw = a.dw ? (float *)(a.scratch + p.off_dw) : nullptr;
        d.db = a.db ? (float *)(a.scratch + p.off_db) : nullptr;
        d.rows_per_split = p.rows_per_split;
        d.n_out = a.n_out;
        d.planes = p.planes;
        d.out_tiles = (uint32_t)((a.n_out + p.tile - 1) / p.tile);
        d.in_tiles = a.dw ? (uint32_t)((a.c.width + p.tile - 1) / p.tile) : 1;
        const uint32_t blocks = d.out_tiles * d.in_tiles * p.splits;
        if (a.c.act == HPACML_ACT_RELU)
            launch_dw<true>(d, blocks, p.tile, st);
        else
            launch_dw<false>(d, blocks, p.tile, st);
        if (d.dw)
            join_kernel<<<blocks_for((int64_t)a.n_out * a.c.width), kThreads, 0, st>>>(d.dw, p.splits, a.n_out, a.c.width, a.dw, a.lddw, a.accumulate);
        if (d.db)
            join_kernel<<<blocks_for(a.n_out), kThreads, 0, st>>>(d.db, p.splits, 1, a.n_out, a.db, a.n_out, a.accumulate);
    }
    return hipGetLastError();
}

}  // namespace hpacml
