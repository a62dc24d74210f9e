// The backward pass of a linear layer whose input was kept in 8 bits:
//   dw = dy^T a, db = the sum of dy's rows, dx = (dy W) where the codes are not 0.
// A kept value (8 significant bits times a power of two) is exact in bf16, so
// dw's products are exact on v_mfma_f32_16x16x32_bf16 and summed in fp32.  An
// fp32 operand is the exact sum of three bf16 terms: three products for dw,
// for dx those six of nine whose terms' ranks sum to at most 2.
#include <type_traits>

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
__global__ void __launch_bounds__(64 * WA * WB, 2) dx_kernel(DxArgs p) {
    typedef nt::Product<nt::Bf16, X, false, WA, WB, NA, NB> T;
    __shared__ __align__(1024) char lds[T::kLds];
    T t;
    t.run(p.wt, p.g, p.in_tiles, p.point_tiles, p.terms, lds, [&](const f32x4 (&acc)[NA][NB], int64_t a0, int64_t b0) {
        // the codes of the values that this lane stores, all asked for at
        // once.  Rows of codes are whole blocks of channels: all of a piece's exist.
        constexpr int kPieces = T::kChunks / 4;
        uint2 code[NB][kPieces];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const typename T::Piece at = t.piece(b, i, a0, b0);
                if (p.codes && at.point < p.g.rows && at.out < p.n_in) {
                    const uint8_t *c = p.codes + at.point * p.ld_codes + at.out;
                    code[b][i] = sizeof(X) == 2 ? *(const uint2 *)c : uint2{*(const uint32_t *)c, 0u};
                } else {
                    code[b][i] = uint2{~0u, ~0u};
                }
            }
        t.store((X *)p.dx, p.lddx, a0, p.n_in, b0, p.g.rows,
                [&](int a, int64_t, int b, float (&v)[4]) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        v[e] = acc[a][b][e];
                },
                [&](int b, int i, u32x4 &u) {
                    const uint2 q = code[b][i];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (sizeof(X) == 2) {
                            const uint32_t two = (e < 2 ? q.x : q.y) >> (16 * (e & 1));
                            u[e] &= (two & 0xFFu ? 0x0000FFFFu : 0u) | (two & 0xFF00u ? 0xFFFF0000u : 0u);
                        } else {
                            u[e] = (q.x >> (8 * e)) & 0xFFu ? u[e] : 0u;
                        }
                    }
                });
    });
}

// ---- dw and db ------------------------------------------------------------------
//
// The sum runs over the rows, along which neither operand is contiguous: both
// go to LDS as they lie, [row][column] in bf16, and the fragments come out
// transposed (ds_read_tr16_b64: 16 lanes read 4 rows x 16 columns and get one
// column's 4 rows each).  Slabs of 32 rows, one matrix instruction's depth.
// Everything comes from memory by direct loads: dy to where its fragments are
// read, the codes and their exponents to a place of the thread's own, from
// where it takes them two slabs later, turns them into bf16 values and writes
// those among the fragments.  During slab s (whose dy fragments are in
// registers) a wave reads slab s's value fragments two ahead of their use and
// slab s + 1's dy fragments, converts slab s + 2's codes, and asks for slab
// s + 4's dy and slab s + 5's codes: three slabs pass before a load is waited
// for.  One barrier per slab.
//
// A row of a slab is pairs of 16-byte chunks (16 columns); pair p is stored at
// p ^ turn(row), so that the rows a transposing read touches at one pair lie
// on different banks, and its two chunks change places with swap(p, row), so
// that the threads that write one chunk each do not meet on half the banks.
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

template <int WA, int WB, int NA, int NB>
struct DwTile {
    static constexpr int kWaves = WA * WB, kThreads = 64 * kWaves, kRows = 32;
    static constexpr int kA = 16 * NA * WA, kB = 16 * NB * WB;          // outputs, channels
    static constexpr int kPitchG = 2 * kA, kPitchX = 2 * kB;            // bytes of an LDS row
    static constexpr int kG = kRows * kPitchG, kX = kRows * kPitchX;    // one slab's
    static constexpr int kRingG = 4, kRingX = 3, kRingCodes = 4;
    static constexpr int kCodes = kThreads * 16, kExps = kThreads * 4;  // 16 codes and an exponent per thread
    static constexpr int kAtX = kRingG * kG, kAtCodes = kAtX + kRingX * kX, kAtExps = kAtCodes + kRingCodes * kCodes;
    static constexpr int kLds = kAtExps + kRingCodes * kExps;
    static constexpr int kLoadsG = kG / (1024 * kWaves), kLoads = kLoadsG + 2;
    static constexpr int kActive = kRows * kB / 16;                     // threads with codes of their own
    static_assert(kLoadsG >= 1 && kActive <= kThreads && kLds <= 160 * 1024, "shares of a slab");

    template <int PITCH>
    static __device__ __forceinline__ int turn(int row) {
        return ((row & 3) | ((row >> 1) & 4)) & (PITCH / 32 - 1);
    }
    static __device__ __forceinline__ int swap(int pair, int row) { return ((pair >> 3) + row) & 1; }
    // byte of a slab where column pair `pair`, chunk `half` of `row` is stored
    template <int PITCH>
    static __device__ __forceinline__ int place(int row, int pair, int half) {
        return row * PITCH + (pair ^ turn<PITCH>(row)) * 32 + (half ^ swap(pair, row)) * 16;
    }
    // where a lane begins to read the fragment of column pair `pair`: lane l
    // gets column l % 16, rows 8 (l / 16) + 0..3; rows + 4..7 are 4 * PITCH on
    // (turn and swap are the same there)
    template <int PITCH>
    static __device__ __forceinline__ int fragment_at(int pair, int lane) {
        const int row = (lane >> 4) * 8 + ((lane & 15) >> 2), eighth = lane & 3;
        return place<PITCH>(row, pair, eighth >> 1) + (eighth & 1) * 8;
    }
    template <int PITCH>
    static __device__ __forceinline__ bf16x8 fragment(const char *at) {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        typedef __attribute__((address_space(3))) s16x4 *Lds;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)at);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(at + 4 * PITCH));
        return __builtin_bit_cast(bf16x8, (s16x8){lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    }
};

template <bool RELU, int WA, int WB, int NA, int NB>
__global__ void __launch_bounds__(64 * WA * WB) dw_kernel(DwArgs p) {
    typedef DwTile<WA, WB, NA, NB> T;
    __shared__ __align__(1024) char lds[T::kLds];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wa = wave / WB, wb = wave % WB;

    // the tiles of one part of the rows follow one another on one XCD
    const uint32_t blocks = gridDim.x, xcd = blockIdx.x & 7, per = blocks >> 3, more = blocks & 7;
    const uint32_t id = xcd * per + min(xcd, more) + (blockIdx.x >> 3), tiles = p.out_tiles * p.in_tiles;
    const uint32_t part = id / tiles, tile = id - part * tiles;
    const int j0 = (int)(tile / p.in_tiles) * T::kA, k0 = (int)(tile % p.in_tiles) * T::kB;
    const int64_t from = part * p.rows_per_split, to = min(from + p.rows_per_split, p.c.rows);
    const int slabs = to > from ? (int)((to - from + T::kRows - 1) / T::kRows) : 0, total = slabs * p.planes;

    f32x4 acc[NA][NB] = {};
    float sum[NA] = {};
    const bool sums = p.db && k0 == 0 && wb == 0;

    if (total > 0) {
        const uint32_t base = nt::lds_offset(lds);
        // dy: the column that belongs where this lane's bytes of a load land
        int g_row[T::kLoadsG], g_col[T::kLoadsG];
#pragma unroll
        for (int i = 0; i < T::kLoadsG; ++i) {
            const int at = (i * T::kWaves + wave) * 1024 + lane * 16, row = at / T::kPitchG, chunk = at % T::kPitchG / 16;
            const int pair = (chunk >> 1) ^ T::template turn<T::kPitchG>(row);
            g_row[i] = row;
            g_col[i] = j0 * 2 + pair * 32 + ((chunk & 1) ^ T::swap(pair, row)) * 16;
        }
        // codes: this thread's row and 16 columns
        const int x_id = tid % T::kActive, x_row = x_id / (T::kB / 16), x_pair = x_id % (T::kB / 16);
        int x_col = k0 + x_pair * 16;
        x_col = x_col < (p.c.width + 31) / 32 * 32 ? x_col : 0;     // beyond the width: any codes
        const int x_at = T::kAtX + T::template place<T::kPitchX>(x_row, x_pair, 0);
        const int x_other = T::kAtX + T::template place<T::kPitchX>(x_row, x_pair, 1);

        // the slabs loaded next, past the end the last one again or zeros (so
        // that every step has the same loads under way)
        int g_slab = 0, g_plane = p.planes - 1, g_slot = 0, x_slab = 0, x_slot = 0;   // the smallest terms first
        auto load_g = [&](int i) {
            const int64_t r = from + (int64_t)g_slab * T::kRows + g_row[i];
            const char *src = p.g + g_plane * p.g_plane + r * p.g_pitch + g_col[i];
            nt::load_to_lds(nt::chosen(r < to && g_col[i] < p.g_width && g_plane >= 0, src), base + g_slot * T::kG + (i * T::kWaves + wave) * 1024);
        };
        auto next_g = [&]() {
            g_slot = g_slot + 1 == T::kRingG ? 0 : g_slot + 1;
            if (++g_slab == slabs) {
                g_slab = 0;
                --g_plane;
            }
        };
        auto x_source = [&]() { return min(from + (int64_t)x_slab * T::kRows + x_row, to - 1); };
        auto load_codes = [&]() {
            nt::load_to_lds((const uint8_t *)p.c.codes + x_source() * p.c.ld_codes + x_col,
                            base + T::kAtCodes + x_slot * T::kCodes + wave * 1024);
        };
        auto load_exps = [&]() {
            nt::load_byte_to_lds((const uint8_t *)p.c.exps + x_source() * p.c.ld_exps + (x_col >> 5),
                                 base + T::kAtExps + x_slot * T::kExps + wave * 256);
        };
        auto next_x = [&]() {
            x_slot = x_slot + 1 == T::kRingCodes ? 0 : x_slot + 1;
            x_slab = x_slab + 1 == slabs ? 0 : x_slab + 1;
        };

        // codes to values: slab c_slab (its row may lie past the end: zeros)
        int c_slab = 0, c_slot = 0, w_slot = 0;
        u32x4 code;
        float scale;
        uint32_t word[8];
        auto take = [&]() {
            code = *(const u32x4 *)(lds + T::kAtCodes + c_slot * T::kCodes + tid * 16);
            uint32_t e = *(const uint32_t *)(lds + T::kAtExps + c_slot * T::kExps + tid * 4);
            asm("" : "+v"(e));                    // read it without a branch
            scale = from + (int64_t)c_slab * T::kRows + x_row < to ? block_scale(e & 0xFFu) : 0.f;
        };
        auto convert = [&](int e) {
            const uint32_t w = code[e / 2], q = w >> (16 * (e & 1));
            const float lo = block_value<RELU>(q & 0xFFu, scale), hi = block_value<RELU>((q >> 8) & 0xFFu, scale);
            // exact in bf16: the high halves
            word[e] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo), 0x07060302u);
        };
        auto put = [&]() {
            if (T::kActive == T::kThreads || tid < T::kActive) {
                *(u32x4 *)(lds + x_at + w_slot * T::kX) = u32x4{word[0], word[1], word[2], word[3]};
                *(u32x4 *)(lds + x_other + w_slot * T::kX) = u32x4{word[4], word[5], word[6], word[7]};
            }
            c_slot = c_slot + 1 == T::kRingCodes ? 0 : c_slot + 1;
            w_slot = w_slot + 1 == T::kRingX ? 0 : w_slot + 1;
            c_slab = c_slab + 1 == slabs ? 0 : c_slab + 1;
        };

        // fragments
        int a_at[NA], b_at[NB], a_slot = 0, b_slot = 0;
#pragma unroll
        for (int t = 0; t < NA; ++t)
            a_at[t] = T::template fragment_at<T::kPitchG>(wa * NA + t, lane);
#pragma unroll
        for (int u = 0; u < NB; ++u)
            b_at[u] = T::kAtX + T::template fragment_at<T::kPitchX>(wb * NB + u, lane);
        bf16x8 a[2][NA], b[4];
        auto read_a = [&](int t) { return T::template fragment<T::kPitchG>(lds + a_at[t] + a_slot * T::kG); };
        auto read_b = [&](int u, int slot) { return T::template fragment<T::kPitchX>(lds + b_at[u] + slot * T::kX); };
        auto next_slot = [](int slot, int ring) { return slot + 1 == ring ? 0 : slot + 1; };

        // first: the place in `b` of the slab's first fragment
        auto step = [&](auto first, const bf16x8 (&now)[NA], bf16x8 (&next)[NA]) {
            constexpr int kFirst = decltype(first)::value;
            nt::wait_loads<2 * T::kLoads>();      // what the step before the last two asked for
            nt::barrier();
            const int after = next_slot(b_slot, T::kRingX);
#pragma unroll
            for (int u = 0; u < NB; ++u) {
                // fragments two tiles ahead; past the last, the next slab's first
                b[(kFirst + u + 2) & 3] = u + 2 < NB ? read_b(u + 2, b_slot) : read_b(u + 2 - NB, after);
#pragma unroll
                for (int t = u * NA / NB; t < (u + 1) * NA / NB; ++t)
                    next[t] = read_a(t);
                if (u == 0)
                    take();
                constexpr int kWords = (8 + NB - 2) / (NB - 1);
#pragma unroll
                for (int e = (u - 1) * kWords; e < u * kWords; ++e)
                    if (e >= 0 && e < 8)
                        convert(e);
#pragma unroll
                for (int i = u * T::kLoads / NB; i < (u + 1) * T::kLoads / NB; ++i) {
                    if (i < T::kLoadsG)
                        load_g(i);
                    else if (i == T::kLoadsG)
                        load_codes();
                    else
                        load_exps();
                }
#pragma unroll
                for (int t = 0; t < NA; ++t)
                    acc[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(now[t], b[(kFirst + u) & 3], acc[t][u], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            put();
            if (sums) {
                // eight rows at a time, so that few roundings follow one another
#pragma unroll
                for (int t = 0; t < NA; ++t) {
                    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
                    const bf16x2 ones = __builtin_bit_cast(bf16x2, 0x3F803F80u);
                    float v = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; e += 2)
                        v = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{now[t][e], now[t][e + 1]}, ones, v, false);
                    sum[t] += v;
                }
            }
            next_g();
            next_x();
            a_slot = next_slot(a_slot, T::kRingG);
            b_slot = after;
        };

        // slabs 0..3 of dy and 0..3 of the codes, of which 0 and 1 are converted here
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            load_codes();
            load_exps();
            next_x();
        }
#pragma unroll
        for (int i = 0; i < T::kRingG; ++i) {
#pragma unroll
            for (int l = 0; l < T::kLoadsG; ++l)
                load_g(l);
            next_g();
        }
        nt::wait_loads<0>();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            take();
#pragma unroll
            for (int e = 0; e < 8; ++e)
                convert(e);
            put();
        }
        __builtin_amdgcn_sched_barrier(0);
        load_codes();                             // slab 4, where slab 0's were
        load_exps();
        next_x();
        nt::wait_loads<63>();
        nt::barrier();
#pragma unroll
        for (int t = 0; t < NA; ++t)
            a[0][t] = read_a(t);
        a_slot = 1;
        b[0] = read_b(0, 0);
        b[1] = read_b(1, 0);
        for (int s = 0; s < total; s += 2) {
            step(std::integral_constant<int, 0>(), a[0], a[1]);
            if (s + 1 >= total)
                break;
            step(std::integral_constant<int, NB & 3>(), a[1], a[0]);
        }
        nt::wait_loads<0>();
    }
#pragma unroll
    for (int t = 0; t < NA; ++t) {
        if (sums) {
            // lane l holds output l % 16's rows 8 (l / 16) + 0..7
            float v = sum[t];
            v += __shfl_xor(v, 16);
            v += __shfl_xor(v, 32);
            const int j = j0 + (wa * NA + t) * 16 + lane;
            if (lane < 16 && j < p.n_out)
                p.db[(int64_t)part * p.n_out + j] = v;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int j = j0 + (wa * NA + t) * 16 + (lane >> 4) * 4 + e;
            if (p.dw && j < p.n_out) {
#pragma unroll
                for (int u = 0; u < NB; ++u) {
                    const int k = k0 + (wb * NB + u) * 16 + (lane & 15);
                    if (k < p.c.width)
                        p.dw[((int64_t)part * p.n_out + j) * p.c.width + k] = acc[t][u][e];
                }
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
void launch_dx_tile(DxArgs d, hipStream_t st) {
    typedef nt::Product<nt::Bf16, X, false, WA, WB, NA, NB> T;
    d.in_tiles = (uint32_t)((d.n_in + T::kA - 1) / T::kA);
    d.point_tiles = (uint32_t)((d.g.rows + T::kB - 1) / T::kB);
    dx_kernel<X, WA, WB, NA, NB>
        <<<nt::blocks_for_tiles((int64_t)d.in_tiles * d.point_tiles, T::kPerCu), T::kThreads, 0, st>>>(d);
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
    p.direct = dtype == HPACML_BF16 && ((uintptr_t)dy & 15) == 0 && lddy % 8 == 0 && lddy < (1 << 22) && n_out % 32 == 0;
    p.slabs = (int32_t)slabs_of(2 * n_out);
    p.pitch = (int64_t)p.slabs * (kSlabBytes / 2);
    p.tile = dw_tile(n_out, c.width);
    p.splits = 1;
    if (want_dw) {
        // one round of the chip: a block of the largest tile fills a CU's LDS,
        // two of the middle one and three of the smallest do
        const int64_t tiles = tiles_of(n_out, c.width, p.tile), least = p.tile == 64 ? 256 : 512;
        int64_t splits = (p.tile == 256 ? 256 : p.tile == 128 ? 512 : 768) / tiles;
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
