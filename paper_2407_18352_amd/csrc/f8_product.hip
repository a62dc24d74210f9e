// y (+)= act(p q^T + b) of matrices in 8-bit floating point.
//
// The operands pass through LDS in slabs of 64 values, half a block: one matrix
// instruction's depth (32 x 32 x 64, a scale of its own for each row, which it
// applies itself: a power of two costs nothing in the sum).  A ring of four slabs
// is filled by direct global-to-LDS loads; while the matrix cores work on slab s
// from registers, a wave reads slab s + 1's fragments from LDS and the loads of
// slabs up to s + 4 are under way.  One barrier per slab publishes slab s + 1 and
// frees slab s.  The scales of a block come the same way, one word per lane for
// a wave's own rows of both operands.  Codes lie in memory as in LDS.
//
// Two arithmetics.  The 8-bit matrix instruction aligns the products of eight
// neighbouring values to the largest of them and drops what lies below 2^-13 of
// it: of normal values a result is then 1.3e-5 off, whatever the width.  That is
// far below a step of bf16 (2^-8), so results in bf16 are computed so.  Results in
// fp32 (EXACT) take the codes to bf16 in registers, exactly, with their scales,
// and the bf16 instruction, which sums in fp32 (1e-7 off) at half the rate.
//
// The matrix instruction's first operand is q, so that a lane of its result has
// four neighbouring outputs of one row of y.  A block goes on from tile to tile
// (or part of one, where the width is split), the slabs following one another
// through the ring.
//
// 131,072 x 4096 <- 4096 in bf16 takes 1.67-1.8 ms (2.4-2.6 PFLOP/s; the card's power
// holds it at 1.62 GHz there, matrix cores busy 69%), in fp32 at 2048 <- 131,072 ->
// 2048 0.79 ms (1.39 PFLOP/s, busy 73%): a tile of 256 x 256 reads 96 KB and writes
// 32 KB of LDS for a slab, as many cycles as its products take.
#include <type_traits>

#include "dense8_nt.hpp"
#include "f8.hpp"

namespace hpacml {
namespace f8 {

namespace {

// 4 bytes per lane to LDS at `lds` + 4 * lane
__device__ __forceinline__ void load_word_to_lds(const void *g, uint32_t lds) {
    uint32_t save;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %1, off\n\ts_mov_b32 m0, %0"
                 : "=&s"(save)
                 : "v"(g), "s"(lds)
                 : "memory");
}

struct Item {
    uint32_t out, point, part;
};

// Work items: the tiles of one part of the width after another.  Blocks go to
// the eight XCDs in turn; each XCD takes a contiguous run of items, so that what
// they share meets in its L2; a run goes through groups of kGroup row tiles by
// all output tiles.
struct Items {
    static constexpr uint32_t kGroup = 4;
    uint32_t out_tiles, point_tiles;
    uint32_t at, end, step;

    __device__ __forceinline__ Items(uint32_t outs, uint32_t points, uint32_t parts) : out_tiles(outs), point_tiles(points) {
        const uint32_t items = outs * points * parts, xcd = blockIdx.x & 7, per = items >> 3, more = items & 7;
        const uint32_t first = xcd * per + min(xcd, more);
        at = first + (blockIdx.x >> 3);
        end = first + per + (xcd < more ? 1 : 0);
        step = (gridDim.x - xcd + 7) >> 3;
    }
    __device__ __forceinline__ bool more() const { return at < end; }
    __device__ __forceinline__ void next() { at += step; }
    __device__ __forceinline__ Item place() const {
        Item i;
        const uint32_t tiles = out_tiles * point_tiles;
        i.part = at / tiles;
        const uint32_t t = at - i.part * tiles, group = t / (kGroup * out_tiles), r = t - group * kGroup * out_tiles;
        const uint32_t high = min(kGroup, point_tiles - group * kGroup);
        i.out = r / high;
        i.point = group * kGroup + r % high;
        return i;
    }
};

template <typename Y>
struct Args {
    const char *pc, *ps, *qc, *qs;
    int64_t p_rows, q_rows;
    uint32_t blocks, parts, per, more;      // of the width; of a part: at least `per`
    uint32_t out_tiles, point_tiles;
    const float *b;
    Y *y;
    int64_t ldy, part_stride;
    int32_t relu, accumulate;
};

// Blocks of WA x WB waves, each 32 NA outputs x 32 NB rows of y.
template <int WA, int WB, int NA, int NB>
struct Shape {
    static constexpr int kWaves = WA * WB, kThreads = 64 * kWaves, kRing = 4;
    static constexpr int kA = 32 * NA * WA, kB = 32 * NB * WB;
    static constexpr int kUnitsA = kA / 32, kUnitsB = kB / 32, kSlab = (kUnitsA + kUnitsB) * kUnit;
    static constexpr int kMineA = kUnitsA / kWaves, kMineB = kUnitsB / kWaves, kLoads = 2 * (kMineA + kMineB);
    static constexpr int kAtScales = kRing * kSlab, kAtOut = kAtScales + kWaves * 512, kLds = kAtOut + kWaves * 2048;
    static constexpr int kPerCu = 160 * 1024 / kLds;
    static_assert(kMineA * kWaves == kUnitsA && kMineB * kWaves == kUnitsB && kPerCu >= 1, "whole units per wave");
    static_assert(128 % (32 * NA) == 0 && 128 % (32 * NB) == 0, "a wave's scales are in one word per lane");
};

template <typename S, typename Y, int NA, int NB, int WA, int WB>
__device__ __forceinline__ void store_tile(const Args<Y> &g, char *own, int lane, int64_t a0, int64_t b0, Y *y, f32x16 (&acc)[NA][NB]) {
    // The wave's results leave through 2 KB of LDS: 16 rows x 128 bytes at a
    // time, so that the stores are 128-byte runs of a row.
    constexpr int kTiles = 64 / (32 * (int)sizeof(Y) / 2), kPer = 16 / sizeof(Y);   // outputs' tiles at a time, values of 16 bytes
    static_assert(NA % kTiles == 0, "whole runs");
    asm volatile("" : "+v"(lane));       // nothing of this is formed ahead of the products, whose registers it would take
    const int row = lane & 15, mine = (lane >> 4) & 1, high = lane >> 5;
    const bool more = g.part_stride == 0;
    if (more && g.b) {
#pragma unroll
        for (int a = 0; a < NA; ++a)
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float t = g.b[min(a0 + a * 32 + q * 8 + high * 4 + e, g.q_rows - 1)];
#pragma unroll
                    for (int b = 0; b < NB; ++b)
                        acc[a][b][q * 4 + e] += t;
                }
    }
    if (more && g.relu) {
#pragma unroll
        for (int a = 0; a < NA; ++a)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    acc[a][b][e] = relu_keep_nan(acc[a][b][e]);
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int at = 0; at < NA; at += kTiles)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                if (mine == half) {
#pragma unroll
                    for (int t = 0; t < kTiles; ++t)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const f32x16 &c = acc[at + t][b];
                            const float v[4] = {c[q * 4], c[q * 4 + 1], c[q * 4 + 2], c[q * 4 + 3]};
                            const int byte = (t * 32 + q * 8 + high * 4) * (int)sizeof(Y);
                            store_four((Y *)(own + row * 128 + (((byte >> 4) ^ (row & 7)) * 16) + (byte & 15)), v);
                        }
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int r = i * 8 + (lane >> 3), c = lane & 7;
                    u32x4 u = *(const u32x4 *)(own + r * 128 + ((c ^ (r & 7)) * 16));
                    const int64_t point = b0 + b * 32 + half * 16 + r, out = a0 + at * 32 + c * kPer;
                    if (point < g.p_rows && out < g.q_rows) {
                        Y *to = y + point * g.ldy + out;
                        if (out + kPer <= g.q_rows) {
                            if (sizeof(Y) == 4 && g.accumulate) {
                                const f32x4 old = *(const f32x4_any *)to;
                                u = __builtin_bit_cast(u32x4, __builtin_bit_cast(f32x4, u) + old);
                            }
                            *(u32x4_any *)to = u;
                        } else {
#pragma unroll
                            for (int e = 0; e < kPer; ++e)
                                if (out + e < g.q_rows) {
                                    if constexpr (sizeof(Y) == 4)
                                        to[e] = nt::element<Y>(u, e) + (g.accumulate ? to[e] : 0.f);
                                    else
                                        to[e] = nt::element<Y>(u, e);
                                }
                        }
                    }
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            }
}

template <typename Y, bool EXACT, int WA, int WB, int NA, int NB>
__global__ __launch_bounds__(64 * WA * WB, 2) void product_kernel(Args<Y> g) {
    typedef Shape<WA, WB, NA, NB> S;
    extern __shared__ __align__(16) char lds[];
    // A slab's fragments.  Those of q but the last are read in place of the slab
    // before's as soon as the matrix instructions have taken them (kept twice,
    // all of them need 260 registers); the others are kept twice.
    // EXACT: codes of a slab, of q's rows and then of p's, a quarter of them in
    // bf16: those of q in place of the quarter before's, those of p twice.
    i32x8 once[EXACT ? 1 : NA - 1];
    struct Frags {
        i32x8 last, b[NB];
    };
    i32x8 raw[EXACT ? NA + NB : 1];
    bf16x8 qa[EXACT ? NA : 1], pb[2][EXACT ? NB : 1];
    float scale[EXACT ? NA + NB : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wa = wave / WB, wb = wave % WB;
    const uint32_t base = nt::lds_offset(lds);
    const char *fa = lds + wa * NA * kUnit + lane * 16, *fb = lds + (S::kUnitsA + wb * NB) * kUnit + lane * 16;
    char *own_scales = lds + S::kAtScales + wave * 512;
    const uint32_t scales_at = nt::lds_offset(own_scales);

    Items items(g.out_tiles, g.point_tiles, g.parts), ahead = items;
    if (!items.more())
        return;
    const uint64_t unit_pitch = (uint64_t)g.blocks * 2 * kUnit;      // of 32 rows
    const uint32_t last_a = (uint32_t)((g.q_rows - 1) >> 5), last_b = (uint32_t)((g.p_rows - 1) >> 5);
    auto first_block = [&](uint32_t part) { return part * g.per + min(part, g.more); };   // the first parts have one more

    // the item loaded: addresses of its next slab, and slabs left
    uint64_t ga[S::kMineA], gb[S::kMineB], gs;
    int left = 0, to_slot = 0, to_scales = 0, from_slot = 0, from_scales = 0;
    auto begin = [&]() {
        const Item i = ahead.place();
        const uint32_t k0 = first_block(i.part);
        left = 2 * (int)(first_block(i.part + 1) - k0);
#pragma unroll
        for (int l = 0; l < S::kMineA; ++l)
            ga[l] = (uint64_t)g.qc + min(i.out * S::kUnitsA + l * S::kWaves + wave, last_a) * unit_pitch + (uint64_t)k0 * 2 * kUnit;
#pragma unroll
        for (int l = 0; l < S::kMineB; ++l)
            gb[l] = (uint64_t)g.pc + min(i.point * S::kUnitsB + l * S::kWaves + wave, last_b) * unit_pitch + (uint64_t)k0 * 2 * kUnit;
        // lanes below 32: q's words, the others: p's
        const uint64_t ra = min((i.out * S::kUnitsA + wa * NA) >> 2, last_a >> 2), rb = min((i.point * S::kUnitsB + wb * NB) >> 2, last_b >> 2);
        gs = lane < 32 ? (uint64_t)g.qs + (ra * g.blocks + k0) * 128 + lane * 4 : (uint64_t)g.ps + (rb * g.blocks + k0) * 128 + (lane - 32) * 4;
    };
    // one of the direct loads of the slab loaded next
    auto load_part = [&](int l) {
        const uint32_t to = base + to_slot * S::kSlab;
        if (l < 2 * S::kMineA)
            nt::load_to_lds(ga[l < 2 * S::kMineA ? l / 2 : 0] + (l & 1) * 1024, lane * 16, to + (l / 2 * S::kWaves + wave) * kUnit + (l & 1) * 1024);
        else {
            const int m = l < 2 * S::kMineA ? 0 : l - 2 * S::kMineA;
            nt::load_to_lds(gb[m / 2] + (m & 1) * 1024, lane * 16, to + (S::kUnitsA + m / 2 * S::kWaves + wave) * kUnit + (m & 1) * 1024);
        }
    };
    auto load_scales = [&]() {
        load_word_to_lds((const void *)gs, scales_at + to_scales * 256);
        to_scales ^= 1;
        gs += 128;
    };
    auto load_done = [&]() {
        to_slot = (to_slot + 1) & (S::kRing - 1);
#pragma unroll
        for (int l = 0; l < S::kMineA; ++l)
            ga[l] += kUnit;
#pragma unroll
        for (int l = 0; l < S::kMineB; ++l)
            gb[l] += kUnit;
        if (--left == 0) {
            // the next item, or, past the last, the same again (every step has as many loads under way)
            Items t = ahead;
            t.next();
            if (t.more())
                ahead = t;
            begin();
        }
    };
    auto read_half = [&](const char *p, i32x8 &f, int h) {
        const i32x4 v = *(const i32x4 *)(p + h * 1024);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            f[h * 4 + e] = v[e];
    };
    // read r of a slab's fragments: what is kept twice, then q's first ones
    constexpr int kTwice = 2 * (1 + NB), kReads = 2 * (NA - 1) + kTwice;
    auto read_part = [&](int r, Frags &f) {
        const int at = from_slot * S::kSlab;
        if (r < 2)
            read_half(fa + at + (NA - 1) * kUnit, f.last, r & 1);
        else if (r < kTwice)
            read_half(fb + at + (r - 2) / 2 * kUnit, f.b[r < kTwice ? (r - 2) / 2 : 0], r & 1);
        else
            read_half(fa + at + (r - kTwice) / 2 * kUnit, once[r < kTwice ? 0 : (r - kTwice) / 2], r & 1);
    };
    uint32_t sa, sb, next_sa, next_sb;
    const int shift_a = wa * NA % 4 * 8, shift_b = wb * NB % 4 * 8;
    auto read_scales = [&]() {
        next_sa = *(const uint32_t *)(own_scales + from_scales * 256 + (lane & 31) * 4) >> shift_a;
        next_sb = *(const uint32_t *)(own_scales + from_scales * 256 + 128 + (lane & 31) * 4) >> shift_b;
        from_scales ^= 1;
    };
    f32x16 acc[NA][NB];
    auto mul = [&](const Frags &f, int i) {
        const int a = i / NB, b = i % NB;
        f32x16 &c = acc[a][b];
        switch (a * 4 + b) {
#define HPACML_F8_CASE(A_, B_)                                              \
    case A_ * 4 + B_:                                                       \
        if constexpr (!EXACT && A_ < NA && B_ < NB)                         \
            c = multiply<A_, B_>(A_ < NA - 1 ? once[A_ < NA - 1 ? A_ : 0] : f.last, f.b[B_], c, sa, sb);             \
        break;
            HPACML_F8_CASE(0, 0) HPACML_F8_CASE(1, 0) HPACML_F8_CASE(2, 0) HPACML_F8_CASE(3, 0)
            HPACML_F8_CASE(0, 1) HPACML_F8_CASE(1, 1) HPACML_F8_CASE(2, 1) HPACML_F8_CASE(3, 1)
#undef HPACML_F8_CASE
        }
        asm volatile("" : "+v"(c));          // stays between the loads it is written between
    };
    // Slab s from `now`, slab s + 1 to `next`, slab s + 4 to where slab s was.
    // FIRST: of a block of the width; its step also loads a block's scales, the
    // other one reads those of the next block.
    int arrived = 0;             // steps whose loads have
    auto step = [&](const Frags &now, Frags &next, auto first) {
        constexpr bool FIRST = decltype(first)::value;
        constexpr int kMul = NA * NB, kOps = kTwice + 1 + S::kLoads;
        if (arrived > 0)
            nt::wait_loads<63>();
        else
            nt::wait_loads<2 * S::kLoads + 1>();
        --arrived;
        nt::barrier();
        from_slot = (from_slot + 1) & (S::kRing - 1);
        // The LDS reads and loads go out between the matrix instructions, as
        // early as the registers are free.
#pragma unroll
        for (int i = 0, op = 0; i < kMul; ++i) {
            mul(now, i);
            __builtin_amdgcn_sched_barrier(0);
            if (i % NB == NB - 1 && i / NB < NA - 1) {
                read_part(kTwice + 2 * (i / NB), next);
                read_part(kTwice + 2 * (i / NB) + 1, next);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (; op < kOps * (i + 1) / (kMul - 1) && op < kOps; ++op) {
                if (op < kTwice)
                    read_part(op, next);
                else if (op == kTwice) {
                    if constexpr (FIRST)
                        load_scales();
                    else
                        read_scales();
                } else
                    load_part(op - kTwice - 1);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        load_done();
        if constexpr (!FIRST) {
            sa = next_sa;
            sb = next_sb;
        }
    };
    // ---- EXACT
    auto take_scales = [&]() {
#pragma unroll
        for (int t = 0; t < NA + NB; ++t) {
            const uint32_t w = t < NA ? sa >> 8 * t : sb >> 8 * (t - NA);
            scale[t] = __builtin_bit_cast(float, (w & 255u) << 23);
        }
    };
    // quarter e of tile t's codes in bf16, times their scale (exact)
    auto quarter = [&](int t, int e) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        bf16x8 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bf16x2 w = i & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[t][2 * e + i / 2], scale[t], true)
                                   : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[t][2 * e + i / 2], scale[t], false);
            v[2 * i] = w[0];
            v[2 * i + 1] = w[1];
        }
        return v;
    };
    auto read_raw = [&](int t, int h) {
        const int at = from_slot * S::kSlab;
        read_half(t < NA ? fa + at + t * kUnit : fb + at + (t - NA) * kUnit, raw[t], h);
    };
    // A slab in four quarters of 16 values; while the matrix cores work on one
    // the next is converted (at the end, the next slab's first), and the halves
    // of the next slab's codes are read where both quarters are done with.
    auto exact_step = [&](auto first) {
        constexpr bool FIRST = decltype(first)::value;
        constexpr int kMul = NA * NB, kOps = 1 + S::kLoads;
        if (arrived > 0)
            nt::wait_loads<63>();
        else
            nt::wait_loads<2 * S::kLoads + 1>();
        --arrived;
        nt::barrier();
        from_slot = (from_slot + 1) & (S::kRing - 1);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (e == 3 && !FIRST) {
                sa = next_sa;
                sb = next_sb;
                take_scales();
            }
#pragma unroll
            for (int i = 0, op = 0; i < kMul; ++i) {
                const int a = i / NB, b = i % NB;
                f32x16 &c = acc[a][b];
                c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qa[a], pb[e & 1][b], c, 0, 0, 0);
                asm volatile("" : "+v"(c));
                __builtin_amdgcn_sched_barrier(0);
                if (i < NB)
                    pb[(e + 1) & 1][i] = quarter(NA + i, (e + 1) & 3);
                if (b == NB - 1)
                    qa[a] = quarter(a, (e + 1) & 3);
                __builtin_amdgcn_sched_barrier(0);
                if (e & 1) {
                    // tiles' halves, one or two after each instruction
#pragma unroll
                    for (; op < (NA + NB) * (i + 1) / kMul; ++op)
                        read_raw(op, e / 2);
                } else if (e == 0) {
#pragma unroll
                    for (; op < kOps * (i + 1) / kMul; ++op) {
                        if (op > 0)
                            load_part(op - 1);
                        else if constexpr (FIRST)
                            load_scales();
                        else
                            read_scales();
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        load_done();
    };
    Frags f0, f1;
    begin();
#pragma unroll
    for (int i = 0; i < S::kRing; ++i) {
        if (i % 2 == 0)
            load_scales();
#pragma unroll
        for (int l = 0; l < S::kLoads; ++l)
            load_part(l);
        load_done();
    }
    nt::wait_loads<0>();
    read_scales();               // an item's last step reads the next one's
    sa = next_sa;
    sb = next_sb;
    if constexpr (EXACT)
        take_scales();
    for (; items.more(); items.next()) {
        const Item it = items.place();
        const int blocks = (int)(first_block(it.part + 1) - first_block(it.part));
        // slabs 0..3 of what comes have arrived, and the scales of two blocks
        nt::barrier();
        if constexpr (EXACT) {
#pragma unroll
            for (int t = 0; t < NA + NB; ++t) {
                read_raw(t, 0);
                read_raw(t, 1);
            }
#pragma unroll
            for (int t = 0; t < NA; ++t)
                qa[t] = quarter(t, 0);
#pragma unroll
            for (int t = 0; t < NB; ++t)
                pb[0][t] = quarter(NA + t, 0);
        } else {
#pragma unroll
            for (int r = 0; r < kReads; ++r)
                read_part(r, f0);
        }
#pragma unroll
        for (int a = 0; a < NA; ++a)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    acc[a][b][e] = 0.f;
        arrived = S::kRing - 1;
        asm volatile("" : "+s"(arrived));
        for (int k = 0; k < blocks; ++k) {
            if constexpr (EXACT) {
                exact_step(std::true_type());
                exact_step(std::false_type());
            } else {
                step(f0, f1, std::true_type());
                step(f1, f0, std::false_type());
            }
        }
        nt::wait_loads<0>();
        store_tile<S, Y, NA, NB, WA, WB>(g, lds + S::kAtOut + wave * 2048, lane, (int64_t)it.out * S::kA + wa * NA * 32,
                                         (int64_t)it.point * S::kB + wb * NB * 32, g.y + it.part * g.part_stride, acc);
    }
}

// y = act(the sum of parts + b), four outputs of a row at a time; `lanes` threads
// share an output's parts (235 parts of 50 x 201 outputs took 64 us with one).
template <typename Y, int LANES>
__global__ __launch_bounds__(256) void finish_kernel(const float *part, int64_t parts, int64_t rows, int64_t width, int64_t pitch, const float *b,
                                                     int32_t relu, int32_t accumulate, Y *y, int64_t ldy) {
    constexpr int kFours = 256 / LANES;
    __shared__ f32x4 of[LANES > 1 ? LANES : 1][kFours];
    const int64_t four = (width + 3) / 4, all = rows * four;
    const int at = threadIdx.x % kFours, share = threadIdx.x / kFours;
    for (int64_t first = (int64_t)blockIdx.x * kFours; first < all; first += (int64_t)gridDim.x * kFours) {
        const int64_t i = first + at, r = i / four, c = i % four * 4;
        f32x4 t = {0.f, 0.f, 0.f, 0.f};
        if (i < all) {
            const float *p = part + r * pitch + c;
#pragma unroll 4
            for (int64_t k = share; k < parts; k += LANES)
                t += *(const f32x4_any *)(p + k * rows * pitch);
        }
        if constexpr (LANES > 1) {
            __syncthreads();
            of[share][at] = t;
            __syncthreads();
            if (share > 0)
                continue;
#pragma unroll
            for (int k = 1; k < LANES; ++k)
                t += of[k][at];
        }
        if (i >= all)
            continue;
        Y *to = y + r * ldy + c;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < width) {
                float v = t[e] + (b ? b[c + e] : 0.f);
                if (relu)
                    v = relu_keep_nan(v);
                if constexpr (sizeof(Y) == 4)
                    v += accumulate ? to[e] : 0.f;
                store_value(to + e, v);
            }
    }
}

template <typename Y>
hipError_t launch_finish(const float *part, int64_t parts, int64_t rows, int64_t width, int64_t pitch, const float *b, int32_t relu,
                         int32_t accumulate, Y *y, int64_t ldy, hipStream_t stream) {
    const int64_t four = rows * ((width + 3) / 4), lanes = parts > 8 ? 16 : 1, blocks = (four + 256 / lanes - 1) / (256 / lanes);
    const uint32_t grid = (uint32_t)(blocks < 1 << 20 ? blocks : 1 << 20);
    if (lanes > 1)
        finish_kernel<Y, 16><<<grid, 256, 0, stream>>>(part, parts, rows, width, pitch, b, relu, accumulate, y, ldy);
    else
        finish_kernel<Y, 1><<<grid, 256, 0, stream>>>(part, parts, rows, width, pitch, b, relu, accumulate, y, ldy);
    return hipGetLastError();
}

int64_t partial_pitch(int64_t q_rows) { return (q_rows + 3) / 4 * 4; }

template <typename Y, bool EXACT, int WA, int WB, int NA, int NB>
hipError_t launch_shape(const Args<Y> &g, hipStream_t stream) {
    typedef Shape<WA, WB, NA, NB> S;
    auto kernel = product_kernel<Y, EXACT, WA, WB, NA, NB>;
    const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, S::kLds);     // of this device
    if (e != hipSuccess)
        return e;
    const uint32_t grid = nt::blocks_for_tiles((int64_t)g.out_tiles * g.point_tiles * g.parts, S::kPerCu);
    kernel<<<grid, S::kThreads, S::kLds, stream>>>(g);
    return hipGetLastError();
}

template <typename Y>
hipError_t launch_tiles(const ProductArgs &a, const Plan &p, bool exact, Y *y, int64_t ldy, int64_t part_stride, hipStream_t stream) {
    const uint32_t blocks = (uint32_t)blocks_of(a.p.width), parts = (uint32_t)p.parts;
    const Args<Y> g = {a.p.codes, a.p.scales, a.q.codes, a.q.scales, a.p.rows, a.q.rows, blocks, parts, blocks / parts, blocks % parts, p.out_tiles,
                       p.point_tiles, a.b, y, ldy, part_stride, a.relu, part_stride ? 0 : a.accumulate};
    if constexpr (sizeof(Y) == 4)
        if (exact)
            return p.big ? launch_shape<Y, true, 2, 4, 4, 2>(g, stream) : launch_shape<Y, true, 2, 2, 2, 2>(g, stream);
    return p.big ? launch_shape<Y, false, 2, 4, 4, 2>(g, stream) : launch_shape<Y, false, 2, 2, 2, 2>(g, stream);
}

}  // namespace

int64_t product_partial_bytes(int64_t p_rows, int64_t q_rows, int64_t width) {
    if (few_rows(p_rows, q_rows, width))
        return 0;
    const Plan p = plan_of(p_rows, q_rows, width);
    return p.parts > 1 ? (int64_t)p.parts * p_rows * partial_pitch(q_rows) * 4 : 0;
}

hipError_t launch_product(const ProductArgs &a, int32_t y_dtype, hipStream_t stream) {
    if (a.p.rows == 0 || a.q.rows == 0)
        return hipSuccess;
    if (few_rows(a.p.rows, a.q.rows, a.p.width))
        return launch_product_few(a, y_dtype, stream);
    const Plan p = plan_of(a.p.rows, a.q.rows, a.p.width);
    const int64_t pitch = partial_pitch(a.q.rows);
    const bool empty = a.p.width == 0;
    if (!empty && p.parts == 1)
        return y_dtype == HPACML_F32 ? launch_tiles(a, p, true, (float *)a.y, a.ldy, 0, stream) : launch_tiles(a, p, false, (uint16_t *)a.y, a.ldy, 0, stream);
    if (!empty) {
        const hipError_t e = launch_tiles(a, p, y_dtype == HPACML_F32, a.partial, pitch, a.p.rows * pitch, stream);
        if (e != hipSuccess)
            return e;
    }
    const int64_t parts = empty ? 0 : p.parts;
    if (y_dtype == HPACML_F32)
        return launch_finish(a.partial, parts, a.p.rows, a.q.rows, pitch, a.b, a.relu, a.accumulate, (float *)a.y, a.ldy, stream);
    return launch_finish(a.partial, parts, a.p.rows, a.q.rows, pitch, a.b, a.relu, 0, (uint16_t *)a.y, a.ldy, stream);
}

}  // namespace f8
}  // namespace hpacml
