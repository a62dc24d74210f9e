// The backward pass of a linear layer whose input was kept in 8 bits:
//   dw = dy^T a, db = the sum of dy's rows, dx = (dy W) where the codes are not 0.
// A kept value (8 significant bits times a power of two) is exact in bf16, so
// dw's products are exact on v_mfma_f32_16x16x32_bf16 and summed in fp32.  An
// fp32 operand is the exact sum of three bf16 terms: three products for dw,
// for dx those six of nine whose terms' ranks sum to at most 2.
//
// Few rows take one launch (backward8_few.hip); otherwise up to four follow one
// another.  131,072 rows of 2048 <- 2048 in bf16: W laid out 8 us, dx 0.9 ms, dw
// 1.05-1.15 ms (1.0 PFLOP/s; the matrix cores work in 43% of its cycles, held up
// by the conversion of the codes between them), parts joined 14 us.  262,144
// rows of 256 <- 256: 5, 65, 68 and 7 us; dx and dw are bound by memory (337 MB
// at 5.2 TB/s; 203 MB at 3.0 TB/s).
#include <type_traits>

#include "dense8_nt.hpp"
#include "dense8_rows.hpp"

namespace hpacml {

namespace {

constexpr int kThreads = 256;             // of the kernels that lay operands out and join parts
constexpr int64_t kMaxBlocks = 1 << 16;   // they loop beyond them

// What the products read, laid out in scratch by one launch: dy's planes
// [planes][rows][pitch], zero beyond n_out (unless dy is read in place), and
// the planes of W's transpose [n_in][n_out], blocked, zero beyond n_out
// (unless dx is not wanted).
template <typename T>
struct LayoutArgs {
    const T *dy;
    int64_t lddy, rows, pitch;
    uint16_t *planes;
    uint32_t row_blocks;        // blocks that lay out dy; the others W
    const T *W;
    int64_t ldw;
    char *wt;
    int32_t n_out, n_in, slabs, cols_log;
};
constexpr int kTurn = 64;       // channels of a block of W, by one slab's outputs

// a chunk of eight values as bf16, or as its three terms
__device__ __forceinline__ void store_planes(char *at, int64_t plane, const float (&v)[kChunk], float) {
    uint32_t w[4][3];
#pragma unroll
    for (int e = 0; e < kChunk; e += 2)
        split3(v[e], v[e + 1], w[e / 2]);
#pragma unroll
    for (int q = 0; q < 3; ++q)
        *(u32x4 *)(at + q * plane) = u32x4{w[0][q], w[1][q], w[2][q], w[3][q]};
}
__device__ __forceinline__ void store_planes(char *at, int64_t, const float (&v)[kChunk], uint16_t) {
    *(u32x4 *)at = u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
}

template <typename T>
__global__ void __launch_bounds__(kThreads) layout_kernel(LayoutArgs<T> p) {
    __shared__ float tile[kSlabBytes / 2][kTurn + 1];
    const int tid = threadIdx.x;
    float v[kChunk];
    if (blockIdx.x < p.row_blocks) {
        const int col = tid & ((1 << p.cols_log) - 1), per = kThreads >> p.cols_log, chunks = (int)(p.pitch / kChunk);
        for (int64_t r = (int64_t)blockIdx.x * per + (tid >> p.cols_log); r < p.rows; r += (int64_t)p.row_blocks * per)
            for (int at = col; at < chunks; at += 1 << p.cols_log) {
                load_chunk(p.dy + r * p.lddy + at * kChunk, p.n_out - at * kChunk, v);
                store_planes((char *)(p.planes + r * p.pitch + at * kChunk), p.rows * p.pitch * 2, v, T{});
            }
        return;
    }
    const int id = (int)(blockIdx.x - p.row_blocks), slab = id % p.slabs, k0 = id / p.slabs * kTurn;
    float w[kSlabBytes / 2 * kTurn / kThreads];
#pragma unroll
    for (int n = 0; n < kSlabBytes / 2 * kTurn / kThreads; ++n) {
        const int i = n * kThreads + tid, out = slab * (kSlabBytes / 2) + i / kTurn, k = k0 + i % kTurn;
        w[n] = out < p.n_out && k < p.n_in ? load_value(p.W + (int64_t)out * p.ldw + k) : 0.f;
    }
#pragma unroll
    for (int n = 0; n < kSlabBytes / 2 * kTurn / kThreads; ++n)
        tile[(n * kThreads + tid) / kTurn][tid % kTurn] = w[n];
    __syncthreads();
    const int k = tid / 4, c = tid % 4;      // eight outputs of a channel
    if (k0 + k < p.n_in) {
#pragma unroll
        for (int e = 0; e < kChunk; ++e)
            v[e] = tile[c * kChunk + e][k];
        store_planes(p.wt + blocked_offset(k0 + k, slab * kSlabBytes + c * 16, p.slabs), blocked_bytes(p.n_in, p.slabs), v, T{});
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

template <typename X, bool MERGE, int WA, int WB, int NA, int NB>
__global__ void __launch_bounds__(64 * WA * WB, 2) dx_kernel(DxArgs p) {
    typedef nt::Product<nt::Bf16, X, false, MERGE, WA, WB, NA, NB> T;
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
                const auto at = t.piece(b, i, a0, b0);
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
    float *dw, *db;             // of the first part; NULL: not wanted
    int64_t lddw, dw_part, db_part;   // pitch of dw, and from a part to the next
    int64_t rows_per_split;
    int32_t n_out, planes, accumulate;
    uint32_t out_tiles, in_tiles;
};

// PL: planes of dy that a slab takes at once.  Three at once convert the codes
// once and have three times as much under way, but the largest tile has no
// room for them in LDS and goes through the rows once for each.
template <int PL, int WA, int WB, int NA, int NB>
struct DwTile {
    static constexpr int kWaves = WA * WB, kThreads = 64 * kWaves, kRows = 32;
    static constexpr int kA = 16 * NA * WA, kB = 16 * NB * WB;          // outputs, channels
    static constexpr int kPitchG = 2 * kA, kPitchX = 2 * kB;            // bytes of an LDS row
    static constexpr int kPlane = kRows * kPitchG, kG = PL * kPlane, kX = kRows * kPitchX;    // one slab's
    static constexpr int kRingG = 4, kRingX = 3, kRingCodes = 4;
    static constexpr int kCodes = kThreads * 16, kExps = kThreads * 4;  // 16 codes and an exponent per thread
    static constexpr int kAtX = kRingG * kG, kAtCodes = kAtX + kRingX * kX, kAtExps = kAtCodes + kRingCodes * kCodes;
    static constexpr int kLds = kAtExps + kRingCodes * kExps;
    static constexpr int kLoadsG = kG / (1024 * kWaves), kLoads = kLoadsG + 2;   // direct loads of a wave
    static constexpr int kPerCu = 160 * 1024 / kLds;
    static constexpr int kActive = kRows * kB / 16;                     // threads with codes of their own
    static_assert(kLoadsG >= 1 && kActive <= kThreads && kLds <= 160 * 1024, "shares of a slab");

    template <int PITCH>
    static __device__ __forceinline__ int turn(int row) {
        return ((row & 3) | ((row >> 1) & 4)) & (PITCH / 32 - 1);
    }
    static __device__ __forceinline__ int swap(int pair, int row) { return ((pair >> 2) + row) & 1; }
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

template <bool RELU, int PL, int WA, int WB, int NA, int NB>
__global__ void __launch_bounds__(64 * WA * WB) dw_kernel(DwArgs p) {
    typedef DwTile<PL, WA, WB, NA, NB> T;
    __shared__ __align__(1024) char lds[T::kLds];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wa = wave / WB, wb = wave % WB;

    // the tiles of one part of the rows follow one another on one XCD
    const uint32_t blocks = gridDim.x, xcd = blockIdx.x & 7, per = blocks >> 3, more = blocks & 7;
    const uint32_t id = xcd * per + min(xcd, more) + (blockIdx.x >> 3), tiles = p.out_tiles * p.in_tiles;
    const uint32_t part = id / tiles, tile = id - part * tiles;
    const int j0 = (int)(tile / p.in_tiles) * T::kA, k0 = (int)(tile % p.in_tiles) * T::kB;
    const int64_t from = part * p.rows_per_split, to = min(from + p.rows_per_split, p.c.rows);
    const int slabs = to > from ? (int)((to - from + T::kRows - 1) / T::kRows) : 0, total = slabs * (p.planes / PL);

    f32x4 acc[NA][NB] = {};
    float sum[NA] = {};
    const bool sums = p.db && k0 == 0 && wb == 0;

    if (total > 0) {
        const uint32_t base = nt::lds_offset(lds);
        const int rows = (int)(to - from);
        // dy: the row and column that belong where this lane's bytes of a load
        // land; where there is no such row or column, zeros (a column past the
        // last has a row past every last)
        const char *g_at[T::kLoadsG];
        int g_row[T::kLoadsG], g_plane = p.planes - PL;      // (the first of PL) the smallest terms first
        int64_t g_first[T::kLoadsG];
#pragma unroll
        for (int i = 0; i < T::kLoadsG; ++i) {
            const int at = (i * T::kWaves + wave) * 1024 + lane * 16, row = at % T::kPlane / T::kPitchG, chunk = at % T::kPitchG / 16;
            const int pair = (chunk >> 1) ^ T::template turn<T::kPitchG>(row);
            const int col = j0 * 2 + pair * 32 + ((chunk & 1) ^ T::swap(pair, row)) * 16;
            g_row[i] = col < p.g_width ? row : INT32_MAX;
            g_first[i] = at / T::kPlane * p.g_plane + (from + row) * p.g_pitch + col;
            g_at[i] = p.g + g_plane * p.g_plane + g_first[i];
        }
        // codes: this thread's row and 16 columns
        const int x_id = tid % T::kActive, x_row = x_id / (T::kB / 16), x_pair = x_id % (T::kB / 16);
        int x_col = k0 + x_pair * 16;
        x_col = x_col < (p.c.width + 31) / 32 * 32 ? x_col : 0;     // beyond the width: any codes
        const int64_t x_first = min(from + x_row, to - 1);
        const char *const codes_first = (const char *)p.c.codes + x_first * p.c.ld_codes + x_col;
        const char *const exps_first = (const char *)p.c.exps + x_first * p.c.ld_exps + (x_col >> 5);
        const char *codes_at = codes_first, *exps_at = exps_first;
        const int x_at = T::kAtX + T::template place<T::kPitchX>(x_row, x_pair, 0);
        const int x_other = T::kAtX + T::template place<T::kPitchX>(x_row, x_pair, 1);

        // What is loaded next, and how many rows are left there.  After the
        // last slab come the next plane's, and after the last plane zeros and
        // any codes: every step has the same loads under way.
        int g_left = rows, g_slot = 0, x_left = rows, x_slot = 0;
        auto load_g = [&](int i) {
            nt::load_to_lds(nt::chosen(g_row[i] < g_left, g_at[i]), base + g_slot * T::kG + (i * T::kWaves + wave) * 1024);
        };
        auto next_g = [&]() {
            g_slot = g_slot + 1 == T::kRingG ? 0 : g_slot + 1;
            g_left -= T::kRows;
#pragma unroll
            for (int i = 0; i < T::kLoadsG; ++i)
                g_at[i] += T::kRows * p.g_pitch;
            if (g_left <= 0) {
                g_plane -= PL;
                g_left = g_plane < 0 ? 0 : rows;
#pragma unroll
                for (int i = 0; i < T::kLoadsG; ++i)
                    g_at[i] = p.g + g_plane * p.g_plane + g_first[i];
            }
        };
        // (a row past the last reads the part's first again; it counts as zeros)
        auto load_codes = [&]() {
            nt::load_to_lds(x_row < x_left ? codes_at : codes_first, base + T::kAtCodes + x_slot * T::kCodes + wave * 1024);
        };
        auto load_exps = [&]() {
            nt::load_byte_to_lds(x_row < x_left ? exps_at : exps_first, base + T::kAtExps + x_slot * T::kExps + wave * 256);
        };
        auto next_x = [&]() {
            x_slot = x_slot + 1 == T::kRingCodes ? 0 : x_slot + 1;
            x_left -= T::kRows;
            codes_at += T::kRows * p.c.ld_codes;
            exps_at += T::kRows * p.c.ld_exps;
            if (x_left <= 0) {
                x_left = rows;
                codes_at = codes_first;
                exps_at = exps_first;
            }
        };

        // codes to values, zeros past the last row
        int c_left = rows, c_slot = 0, w_slot = 0;
        u32x4 code;
        float scale;
        uint32_t word[8];
        auto take = [&]() {
            code = *(const u32x4 *)(lds + T::kAtCodes + c_slot * T::kCodes + tid * 16);
            uint32_t e = *(const uint32_t *)(lds + T::kAtExps + c_slot * T::kExps + tid * 4);
            asm("" : "+v"(e));                    // read it without a branch
            scale = x_row < c_left ? block_scale(e & 0xFFu, p.planes) : 0.f;
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
            c_left = c_left <= T::kRows ? rows : c_left - T::kRows;
        };

        // fragments
        int a_at[NA], b_at[NB], a_slot = 0, b_slot = 0;
#pragma unroll
        for (int t = 0; t < NA; ++t)
            a_at[t] = T::template fragment_at<T::kPitchG>(wa * NA + t, lane);
#pragma unroll
        for (int u = 0; u < NB; ++u)
            b_at[u] = T::kAtX + T::template fragment_at<T::kPitchX>(wb * NB + u, lane);
        bf16x8 a[2][PL * NA], b[4];      // a: plane by plane
        auto read_a = [&](int t) { return T::template fragment<T::kPitchG>(lds + a_at[t % NA] + t / NA * T::kPlane + a_slot * T::kG); };
        auto read_b = [&](int u, int slot) { return T::template fragment<T::kPitchX>(lds + b_at[u] + slot * T::kX); };
        auto next_slot = [](int slot, int ring) { return slot + 1 == ring ? 0 : slot + 1; };

        // first: the place in `b` of the slab's first fragment
        auto step = [&](auto first, const bf16x8 (&now)[PL * NA], bf16x8 (&next)[PL * NA]) {
            constexpr int kFirst = decltype(first)::value;
            nt::wait_loads<2 * T::kLoads>();      // what the step before the last two asked for
            nt::barrier();
            const int after = next_slot(b_slot, T::kRingX);
#pragma unroll
            for (int u = 0; u < NB; ++u) {
                // fragments two tiles ahead; past the last, the next slab's first
                b[(kFirst + u + 2) & 3] = u + 2 < NB ? read_b(u + 2, b_slot) : read_b(u + 2 - NB, after);
#pragma unroll
                for (int t = u * PL * NA / NB; t < (u + 1) * PL * NA / NB; ++t)
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
                for (int t = PL * NA - 1; t >= 0; --t)
                    acc[t % NA][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[(kFirst + u) & 3], now[t], acc[t % NA][u], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            put();
            if (sums) {
                // eight rows at a time, so that few roundings follow one another
#pragma unroll
                for (int t = PL * NA - 1; t >= 0; --t) {
                    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
                    const bf16x2 ones = __builtin_bit_cast(bf16x2, 0x3F803F80u);
                    float v = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; e += 2)
                        v = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{now[t][e], now[t][e + 1]}, ones, v, false);
                    sum[t % NA] += v;
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
        for (int t = 0; t < PL * NA; ++t)
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
    // acc[t][u]: channels 4 (lane / 16) + e of output lane % 16
    float *dw = p.dw ? p.dw + part * p.dw_part : nullptr;
    const bool four = ((uintptr_t)dw & 15) == 0 && p.lddw % 4 == 0;
#pragma unroll
    for (int t = 0; t < NA; ++t) {
        if (sums) {
            // lane l holds output l % 16's rows 8 (l / 16) + 0..7
            float v = sum[t];
            v += __shfl_xor(v, 16);
            v += __shfl_xor(v, 32);
            const int j = j0 + (wa * NA + t) * 16 + lane;
            if (lane < 16 && j < p.n_out) {
                float *to_db = p.db + part * p.db_part + j;
                *to_db = p.accumulate ? *to_db + v : v;
            }
        }
        const int j = j0 + (wa * NA + t) * 16 + (lane & 15);
        if (!dw || j >= p.n_out)
            continue;
#pragma unroll
        for (int u = 0; u < NB; ++u) {
            const int k = k0 + (wb * NB + u) * 16 + (lane >> 4) * 4;
            float *out = dw + j * p.lddw + k;
            f32x4 v = acc[t][u];
            if (four && k + 4 <= p.c.width) {
                *(f32x4 *)out = p.accumulate ? *(const f32x4 *)out + v : v;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (k + e < p.c.width)
                        out[e] = p.accumulate ? out[e] + v[e] : v[e];
            }
        }
    }
}

// dw [n_out][lddw] and db [n_out] (+)= the sums over their parts, which lie
// after one another; four at a time where rows keep the alignment (FOUR).
struct JoinArgs {
    const float *dw_parts, *db_parts;
    float *dw, *db;               // NULL: not wanted
    int64_t lddw;
    int32_t splits, n_out, n_in, accumulate;
};
// V: four values where rows keep the alignment, or one.  PARTS threads share a
// sum where there are many parts: each adds every PARTS-th, and the first adds
// theirs (always in the same order).
template <typename V, int PARTS>
__global__ void __launch_bounds__(kThreads) join_kernel(JoinArgs p) {
    constexpr int kPer = sizeof(V) / 4, kSums = kThreads / PARTS;
    __shared__ V share[PARTS][kSums];
    const int lane = threadIdx.x % kSums, first = threadIdx.x / kSums;
    auto total = [&](auto *parts, int64_t i, int64_t all) {
        typedef std::remove_cv_t<std::remove_reference_t<decltype(*parts)>> T;
        T v = {};
        if (i < all) {
            const T *at = parts + i;
            int s = first;
            for (; s + 3 * PARTS < p.splits; s += 4 * PARTS) {
                T w[4];
#pragma unroll
                for (int n = 0; n < 4; ++n)
                    w[n] = at[(s + n * PARTS) * all];
#pragma unroll
                for (int n = 0; n < 4; ++n)
                    v += w[n];
            }
            for (; s < p.splits; s += PARTS)
                v += at[s * all];
        }
        if (PARTS > 1) {
            T(*to)[kSums] = (T(*)[kSums])share;
            __syncthreads();
            to[first][lane] = v;
            __syncthreads();
            if (first == 0)
#pragma unroll
                for (int n = 1; n < PARTS; ++n)
                    v += to[n][lane];
        }
        return v;
    };
    const int64_t row = p.n_in / kPer, all = p.dw ? p.n_out * row : 0, step = (int64_t)gridDim.x * kSums;
    for (int64_t i0 = (int64_t)blockIdx.x * kSums; i0 < all; i0 += step) {
        const int64_t i = i0 + lane;
        const V v = total((const V *)p.dw_parts, i, all);
        if (first == 0 && i < all) {
            V *o = (V *)(p.dw + i / row * p.lddw) + i % row;
            *o = p.accumulate ? *o + v : v;
        }
    }
    for (int64_t i0 = (int64_t)blockIdx.x * kSums; p.db && i0 < p.n_out; i0 += step) {
        const int64_t i = i0 + lane;
        const float v = total(p.db_parts, i, p.n_out);
        if (first == 0 && i < p.n_out)
            p.db[i] = p.accumulate ? p.db[i] + v : v;
    }
}

dim3 blocks_for(int64_t items) {
    const int64_t n = (items + kThreads - 1) / kThreads;
    return dim3((uint32_t)(n < 1 ? 1 : n < kMaxBlocks ? n : kMaxBlocks));
}
size_t whole(size_t b) { return (b + 255) / 256 * 256; }

// log2 of the chunks a row of a block of threads covers: 4 .. 256
int cols_log(int64_t chunks) {
    int l = 2;
    while (((int64_t)1 << l) < chunks && (1 << l) < kThreads)
        ++l;
    return l;
}

template <typename T>
void launch_layout(const Backward8Args &a, const Backward8Plan &p, uint16_t *planes, char *wt, hipStream_t st) {
    LayoutArgs<T> l{(const T *)a.dy, a.lddy, p.direct ? 0 : a.c.rows, p.pitch, planes, 0, (const T *)a.W, a.ldw, wt, a.n_out,
                    a.c.width, p.slabs, cols_log(p.pitch / kChunk)};
    const int64_t per = kThreads >> l.cols_log, blocks = (l.rows + per - 1) / per;
    l.row_blocks = (uint32_t)(blocks < 8192 ? blocks : 8192);
    const uint32_t turn = a.dx ? (uint32_t)((a.c.width + kTurn - 1) / kTurn * p.slabs) : 0;
    if (l.row_blocks + turn > 0)
        layout_kernel<T><<<l.row_blocks + turn, kThreads, 0, st>>>(l);
}

template <typename X, bool MERGE, int WA, int WB, int NA, int NB>
void launch_dx_tile(DxArgs d, hipStream_t st) {
    typedef nt::Product<nt::Bf16, X, false, MERGE, WA, WB, NA, NB> T;
    d.in_tiles = (uint32_t)((d.n_in + T::kA - 1) / T::kA);
    d.point_tiles = (uint32_t)((d.g.rows + T::kB - 1) / T::kB);
    dx_kernel<X, MERGE, WA, WB, NA, NB>
        <<<nt::blocks_for_tiles((int64_t)d.in_tiles * d.point_tiles, T::kPerCu), T::kThreads, 0, st>>>(d);
}

template <typename X, bool MERGE>
void launch_dx(const DxArgs &d, hipStream_t st) {
    switch (nt::tile_for(d.n_in, d.g.rows, d.wt.width / kSlabBytes * (d.terms * (d.terms + 1) / 2))) {
    case nt::Size::k64x64: return launch_dx_tile<X, MERGE, 2, 2, 2, 2>(d, st);
    case nt::Size::k128x128: return launch_dx_tile<X, MERGE, 2, 2, 4, 4>(d, st);
    case nt::Size::k128x256: return launch_dx_tile<X, MERGE, 2, 4, 4, 4>(d, st);
    case nt::Size::k256x256: return launch_dx_tile<X, MERGE, 4, 2, 4, 8>(d, st);
    }
}

template <bool RELU, int PL, int WA, int WB, int NA, int NB>
void launch_dw_tile(DwArgs d, int splits, hipStream_t st) {
    typedef DwTile<PL, WA, WB, NA, NB> T;
    d.out_tiles = (uint32_t)((d.n_out + T::kA - 1) / T::kA);
    d.in_tiles = d.dw ? (uint32_t)((d.c.width + T::kB - 1) / T::kB) : 1;
    dw_kernel<RELU, PL, WA, WB, NA, NB><<<d.out_tiles * d.in_tiles * splits, T::kThreads, 0, st>>>(d);
}

template <bool RELU>
void launch_dw(const DwArgs &d, const Backward8Plan &p, hipStream_t st) {
    switch (p.dw.tile) {   // of kDwTiles
    case 0: return launch_dw_tile<RELU, 1, 4, 2, 4, 8>(d, p.dw.splits, st);
    case 1: return launch_dw_tile<RELU, 1, 4, 2, 4, 4>(d, p.dw.splits, st);
    case 2: return launch_dw_tile<RELU, 1, 2, 4, 4, 4>(d, p.dw.splits, st);
    case 3: return launch_dw_tile<RELU, 1, 2, 2, 4, 4>(d, p.dw.splits, st);
    case 4: return launch_dw_tile<RELU, 1, 2, 2, 2, 2>(d, p.dw.splits, st);
    case 5: return launch_dw_tile<RELU, 3, 2, 2, 4, 4>(d, p.dw.splits, st);
    case 6: return launch_dw_tile<RELU, 3, 2, 2, 2, 2>(d, p.dw.splits, st);
    }
}

template <typename V>
void launch_join(const JoinArgs &j, hipStream_t st) {
    const int64_t sums = (int64_t)j.n_out * (j.n_in * 4 / (int)sizeof(V));
    if (j.splits >= 16)
        join_kernel<V, 16><<<blocks_for(sums * 16), kThreads, 0, st>>>(j);
    else
        join_kernel<V, 1><<<blocks_for(sums), kThreads, 0, st>>>(j);
}

}  // namespace

Backward8Plan backward8_plan(const hpacml8_checkpoint &c, const void *dy, int32_t dtype, int64_t lddy, int32_t n_out,
                             bool want_dw, bool want_dx) {
    Backward8Plan p{};
    p.few = few_rows(c.rows, n_out, c.width);   // (the scratch asked for does not depend on it)
    p.planes = dtype == HPACML_F32 ? 3 : 1;
    // dw reads whole 16-byte chunks of dy's rows, dx whole slabs, both with 32-bit offsets in a tile
    p.direct = dtype == HPACML_BF16 && ((uintptr_t)dy & 15) == 0 && lddy % 8 == 0 && lddy < (1 << 22) &&
               n_out % (want_dx ? 32 : 8) == 0;
    p.slabs = (int32_t)slabs_of(2 * n_out);
    p.pitch = (int64_t)p.slabs * (kSlabBytes / 2);
    p.dw = want_dw ? choose_dw(c.rows, n_out, c.width, p.planes) : DwForm{0, 1, 0};
    size_t at = 0;
    p.off_dy = at;
    if (!p.direct)
        at += whole((size_t)p.planes * c.rows * p.pitch * 2);
    p.off_wt = at;
    if (want_dx)
        at += whole((size_t)p.planes * blocked_bytes(c.width, p.slabs));
    p.off_dw = at;
    if (want_dw && p.dw.splits > 1)
        at += whole((size_t)p.dw.splits * n_out * c.width * 4);
    p.off_db = at;
    if (want_dw && p.dw.splits > 1)
        at += whole((size_t)p.dw.splits * n_out * 4);
    p.bytes = at;
    return p;
}

hipError_t launch_backward8(const Backward8Args &a, const Backward8Plan &p, hipStream_t st) {
    if (p.few)
        return launch_backward8_few(a, st);
    const int64_t rows = a.c.rows;
    const bool f32 = a.dtype == HPACML_F32;
    uint16_t *planes = (uint16_t *)(a.scratch + p.off_dy);
    char *wt = a.scratch + p.off_wt;
    if (rows > 0)
        f32 ? launch_layout<float>(a, p, planes, wt, st) : launch_layout<uint16_t>(a, p, planes, wt, st);
    nt::Operand g{(const char *)planes, rows, p.pitch * 2, p.pitch * 2, rows * p.pitch * 2};
    if (p.direct)
        g = {(const char *)a.dy, rows, a.lddy * 2, (int64_t)a.n_out * 2, 0};
    if (a.dx && rows > 0) {
        DxArgs d{};
        d.wt = {wt, a.c.width, (int64_t)p.slabs * 1024, (int64_t)p.slabs * kSlabBytes, blocked_bytes(a.c.width, p.slabs)};
        d.g = g;
        d.codes = a.c.act == HPACML_ACT_RELU ? (const uint8_t *)a.c.codes : nullptr;
        d.dx = a.dx;
        d.ld_codes = a.c.ld_codes;
        d.lddx = a.lddx;
        d.n_in = a.c.width;
        d.terms = p.planes;
        const bool shared = nt::shared_lines(a.dx, a.lddx * (f32 ? 4 : 2));
        if (f32)
            shared ? launch_dx<float, true>(d, st) : launch_dx<float, false>(d, st);
        else
            shared ? launch_dx<uint16_t, true>(d, st) : launch_dx<uint16_t, false>(d, st);
    }
    if (a.dw || a.db) {
        const bool join = p.dw.splits > 1;
        DwArgs d{};
        d.g = g.base;
        d.g_pitch = g.pitch;
        d.g_width = g.width;
        d.g_plane = g.plane;
        d.c = a.c;
        d.dw = join && a.dw ? (float *)(a.scratch + p.off_dw) : a.dw;
        d.db = join && a.db ? (float *)(a.scratch + p.off_db) : a.db;
        d.lddw = join ? a.c.width : a.lddw;
        d.dw_part = (int64_t)a.n_out * a.c.width;
        d.db_part = a.n_out;
        d.accumulate = join ? 0 : a.accumulate;
        d.rows_per_split = p.dw.rows_per_split;
        d.n_out = a.n_out;
        d.planes = p.planes;
        a.c.act == HPACML_ACT_RELU ? launch_dw<true>(d, p, st) : launch_dw<false>(d, p, st);
        if (join) {
            const JoinArgs j{d.dw, d.db, a.dw, a.db, a.lddw, p.dw.splits, a.n_out, a.c.width, a.accumulate};
            if (a.c.width % 4 == 0 && ((uintptr_t)a.dw & 15) == 0 && a.lddw % 4 == 0)
                launch_join<f32x4>(j, st);
            else
                launch_join<float>(j, st);
        }
    }
    return hipGetLastError();
}

}  // namespace hpacml
