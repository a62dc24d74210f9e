// The product both operands of which lie along k: C[a][b] = sum_k A[a][k] B[b][k],
// int8 codes with 32-bit sums or bf16 with fp32 sums.
//
// The operands pass through LDS in slabs of 64 bytes of k (64 codes, 32 bf16:
// one matrix instruction's depth), a ring of four filled by direct
// global-to-LDS loads.  While the matrix cores work on slab s from registers,
// a wave reads slab s + 1's fragments from LDS and the loads of slabs up to
// s + 4 are under way: what a load waits for in the memory system is covered by
// the slabs before it.  One barrier per slab publishes slab s + 1 (its loads
// have been waited for) and frees slab s (its fragments are in registers).
//
// A block computes tiles of C one after another, and the slabs of its tiles
// follow one another through the ring: during a tile's last slabs the next
// tile's first ones load, and they arrive while the results are stored.  (A
// block per tile began and ended every tile with nothing under way: with 256
// blocks in step, 15 us of each 57 us at 4096 codes of k.)
//
// A row of a slab is four 16-byte chunks, chunk c stored at c ^ chunk_turn(row),
// so that the 16 rows a matrix instruction reads at one chunk fall on different
// banks.  An operand that this library lays out itself lies in memory as in LDS:
// a direct load then reads 1 KB in one piece, whatever k is, where rows of a
// power of two would meet in the same few channels of the L2.  From an operand
// in rows each lane fetches the chunk that belongs where its bytes land (the
// direct loads can't permute what they write).  A holds the outputs and B the
// points: a lane of the matrix instruction's result then has four consecutive
// outputs of one point, which is what a row-major store wants.
//
// The direct loads are inline assembly: seeing them, the compiler would make
// every LDS read wait for all of them.  Their completion is waited for by hand.
#pragma once

#include "dense8.hpp"
#include "dense8_rules.hpp"

namespace hpacml {

namespace nt {

struct I8 {
    typedef i32x4 Acc;
    static __device__ __forceinline__ Acc mul(u32x4 a, u32x4 b, Acc c) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
    }
};
struct Bf16 {
    typedef f32x4 Acc;
    static __device__ __forceinline__ Acc mul(u32x4 a, u32x4 b, Acc c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};

// 16 bytes per lane from `g` to LDS at `lds` + 16 * lane (`lds` wave-uniform);
// M0, which carries that address, is put back
__device__ __forceinline__ void load_to_lds(const void *g, uint32_t lds) {
    uint32_t save;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\ts_mov_b32 m0, %0"
                 : "=&s"(save)
                 : "v"(g), "s"(lds)
                 : "memory");
}
// the same from `base` + `offset`, the base wave-uniform
__device__ __forceinline__ void load_to_lds(uint64_t base, uint32_t offset, uint32_t lds) {
    uint32_t save;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b32 m0, %0"
                 : "=&s"(save)
                 : "v"(offset), "s"(base), "s"(lds)
                 : "memory");
}
// one byte per lane, to the low byte of the word at `lds` + 4 * lane
__device__ __forceinline__ void load_byte_to_lds(const void *g, uint32_t lds) {
    uint32_t save;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_ubyte %1, off\n\ts_mov_b32 m0, %0"
                 : "=&s"(save)
                 : "v"(g), "s"(lds)
                 : "memory");
}
// at most N of this wave's vector-memory loads are still under way, and its
// LDS reads are in registers
template <int N>
__device__ __forceinline__ void wait_loads() {
    static_assert(N >= 0 && N < 64, "vmcnt range");
    __builtin_amdgcn_sched_barrier(0);   // the matrix instructions written before it stay before it
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));
}
__device__ __forceinline__ void barrier() { asm volatile("s_barrier" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_offset(const void *p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p;
}

// what a load beyond an operand's width reads
__device__ __align__(16) const uint32_t zero_chunk[4] = {0, 0, 0, 0};

// `g`, or zeros, by selection: the address is computed either way
__device__ __forceinline__ const void *chosen(bool exists, const char *g) {
    asm("" : "+v"(g));
    return exists ? g : (const char *)zero_chunk;
}

// element e of 16 bytes
template <typename Y>
__device__ __forceinline__ Y element(const u32x4 &u, int e) {
    if constexpr (sizeof(Y) == 4) {
        const uint32_t w = u[e];
        return __builtin_bit_cast(Y, w);
    } else {
        const uint32_t w = u[e / 2];
        return (Y)(w >> (16 * (e & 1)));
    }
}

// One operand, in `terms` planes `plane` bytes apart.  BLOCKED: as the LDS
// image has it, 16 rows x 64 bytes after one another (1 KB, chunks swizzled),
// `pitch` bytes per 16 rows; what pads the last rows and slab is there.
// Otherwise rows `pitch` bytes apart.  `width` bytes of k: whole slabs.
struct Operand {
    const char *base;
    int64_t rows, pitch, width, plane;
};

// Block id -> tiles.  Blocks go to the eight XCDs in turn; each XCD takes a
// contiguous run of tiles, its blocks one after another along the run, so that
// what they share meets in its L2; a run goes through groups of kGroup point
// tiles by all output tiles.
constexpr int kGroup = 4;
struct Tiles {
    uint32_t out_tiles, point_tiles;
    uint32_t at, end, step;

    __device__ __forceinline__ Tiles(uint32_t outs, uint32_t points) : out_tiles(outs), point_tiles(points) {
        const uint32_t tiles = outs * points, xcd = blockIdx.x & 7, per = tiles >> 3, more = tiles & 7;
        const uint32_t first = xcd * per + min(xcd, more);
        at = first + (blockIdx.x >> 3);
        end = first + per + (xcd < more ? 1 : 0);
        step = (gridDim.x - xcd + 7) >> 3;
    }
    __device__ __forceinline__ bool more() const { return at < end; }
    __device__ __forceinline__ void next() { at += step; }
    __device__ __forceinline__ void place(uint32_t &out, uint32_t &point) const {
        const uint32_t group = at / (kGroup * out_tiles), r = at - group * kGroup * out_tiles;
        const uint32_t high = min((uint32_t)kGroup, point_tiles - group * kGroup);
        out = r / high;
        point = group * kGroup + r % high;
    }
};
// Blocks for `tiles` tiles when `per_cu` of them share a CU: one round of the
// chip's 256 CUs at most.
inline uint32_t blocks_for_tiles(int64_t tiles, int per_cu) { return (uint32_t)(tiles < 256 * per_cu ? tiles : 256 * per_cu); }

// A wave's results on their way out, as rows of Y, NA * 16 outputs of 16 points
// at a time.  They are turned in LDS, so that the stores are 16-byte pieces of
// long runs of a row, and bypass the caches (a later kernel reads them, if
// any).  131,072 x 1024 -> 1024 in 8 bits, measured with a block per tile: 146
// us so, 187 us through the caches, 227 us with stores as the matrix
// instruction leaves its results.
template <typename Y, int NA>
struct Out {
    static constexpr int kPer = 16 / sizeof(Y), kRow = NA * 16 * sizeof(Y), kChunks = kRow / 16;
    // 16 bytes that a lane stores
    struct Piece {
        int64_t point, out;
        int at;            // in the wave's part of LDS
    };
    // piece i of the 16 points from p0 on, of the outputs from a0 on
    static __device__ __forceinline__ Piece piece(int lane, int i, int64_t a0, int64_t p0) {
        const int at = i * 64 + lane, row = at / kChunks, c = at % kChunks;
        return {p0 + row, a0 + c * kPer, row * kRow + ((c ^ (row & (kChunks - 1))) * 16)};
    }
    // own: the wave's 16 * kRow bytes of LDS.  value(a, n, b, v): the four
    // results of acc[a][b], outputs n.. (a multiple of 4, not above the last).
    // mask(b, i, chunk): changes the 16 bytes that are about to be stored as
    // piece i of acc[..][b].
    // MERGE: for rows that share cache lines (shared_lines): the stores go
    // through the L2, which puts the lines together (fp32 rows of 201: dx of
    // 30,011 rows 22.7 -> 19.6 us).  A form of its own: with a test at each
    // store dx of 262,144 rows, 256 <- 256 in bf16, its inputs read before, took
    // 86 us, not 70.
    template <int NB, bool MERGE, typename Value, typename Mask>
    static __device__ __forceinline__ void store(char *own, int lane, Y *y, int64_t ldy, int64_t a0, int64_t n_out, int64_t b0,
                                                 int64_t rows, Value value, Mask mask) {
        const int64_t last = (n_out - 1) & ~(int64_t)3;
        const int row = lane & 15, grp = lane >> 4;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
            for (int a = 0; a < NA; ++a) {
                float v[4];
                value(a, min(a0 + a * 16 + grp * 4, last), b, v);
                const int byte = (a * 16 + grp * 4) * (int)sizeof(Y);
                store_four((Y *)(own + row * kRow + (((byte >> 4) ^ (row & (kChunks - 1))) * 16) + (byte & 15)), v);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // one wave's LDS accesses are in order
#pragma unroll
            for (int i = 0; i < kChunks / 4; ++i) {
                const Piece p = piece(lane, i, a0, b0 + b * 16);
                u32x4 u = *(const u32x4 *)(own + p.at);
                mask(b, i, u);
                if (p.point < rows && p.out < n_out) {
                    Y *to = y + p.point * ldy + p.out;
                    if (p.out + kPer <= n_out) {
                        if constexpr (MERGE)
                            *(u32x4_any *)to = u;
                        else
                            __builtin_nontemporal_store(u, (u32x4_any *)to);
                    } else {
#pragma unroll
                        for (int e = 0; e < kPer; ++e)
                            if (p.out + e < n_out)
                                to[e] = element<Y>(u, e);
                    }
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
    }
};

inline bool shared_lines(const void *y, int64_t pitch_bytes) { return (((uintptr_t)y | (uint64_t)pitch_bytes) & 63) != 0; }

// Blocks of WA x WB waves, each NA x NB tiles of 16 x 16; results of type Y.
// A is blocked, B is if BLOCKED_B, and comes in rows otherwise.
template <typename Mma, typename Y, bool BLOCKED_B, bool MERGE, int WA, int WB, int NA, int NB>
struct Product {
    static constexpr int kWaves = WA * WB, kThreads = 64 * kWaves, kRing = 4;
    static constexpr int kA = 16 * NA * WA, kB = 16 * NB * WB;
    static constexpr int kBuf = (kA + kB) * kSlabBytes, kLoadsA = kA / (16 * kWaves), kLoadsB = kB / (16 * kWaves);
    static constexpr int kLoads = kLoadsA + kLoadsB;
    static constexpr int kRow = Out<Y, NA>::kRow, kChunks = Out<Y, NA>::kChunks;
    static constexpr int kAtOut = kRing * kBuf, kLds = kAtOut + kWaves * 16 * kRow;
    static constexpr int kPerCu = 160 * 1024 / kLds;
    static_assert(kLoadsA * 16 * kWaves == kA && kLoadsB * 16 * kWaves == kB && kPerCu >= 1, "whole loads per wave");
    typedef typename Mma::Acc Acc;
    struct Frags {
        u32x4 a[NA], b[NB];
    };

    int wave, lane;
    char *lds;

    // `terms`: 1, or 3 planes of each operand of which the products of ranks
    // that sum to at most 2 are taken, the smallest first.  finish(acc, a0,
    // b0): the tile's results; acc[a][b]: outputs a0 + 16 (WA-wave * NA + a) +
    // 4 (lane / 16) + e of point b0 + 16 (WB-wave * NB + b) + lane % 16.
    template <typename Finish>
    __device__ __forceinline__ void run(const Operand &A, const Operand &B, uint32_t out_tiles, uint32_t point_tiles, int terms,
                                        char *shared, Finish finish) {
        lds = shared;
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int row16 = lane >> 2, chunk = (lane & 3) ^ chunk_turn(row16);   // chunk_turn(row) depends on row % 16 alone
        const uint32_t base = lds_offset(lds) + wave * 1024;
        const int wa = wave / WB, wb = wave % WB;
        const int fr = (lane & 15) * kSlabBytes + ((lane >> 4) ^ chunk_turn(lane & 15)) * 16;
        const char *fa = lds + wa * NA * 16 * kSlabBytes + fr, *fb = lds + (kA + wb * NB * 16) * kSlabBytes + fr;
        const int slabs = (int)(A.width / kSlabBytes), total = slabs * (terms * (terms + 1) / 2), pairs = (total + 1) / 2;

        Tiles tiles(out_tiles, point_tiles), ahead = tiles;   // the tile worked on, and the one loaded
        if (!tiles.more())
            return;
        int rank = 0, term = 0, slab = 0, to_slot = 0, from_slot = 0;
        uint64_t ga[kLoadsA], gb;         // first bytes of the tile loaded, in its plane: of each load of A, of B's rows
        uint32_t ob[kLoadsB];             // this lane's offsets from there
        auto begin_plane = [&]() {
            uint32_t out, point;
            ahead.place(out, point);
            const uint64_t a = (uint64_t)(A.base + term * A.plane), b = (uint64_t)(B.base + (rank - term) * B.plane);
            const int64_t b0 = (int64_t)point * kB;
#pragma unroll
            for (int i = 0; i < kLoadsA; ++i)
                ga[i] = a + min((int64_t)out * (kA / 16) + i * kWaves + wave, (A.rows - 1) / 16) * A.pitch;
            gb = b + (BLOCKED_B ? b0 / 16 : b0) * B.pitch;
#pragma unroll
            for (int i = 0; i < kLoadsB; ++i) {
                const int at = i * kWaves + wave, left = (int)min(B.rows - 1 - b0, (int64_t)kB);   // rows after the tile's first
                ob[i] = BLOCKED_B ? (uint32_t)min(at, left / 16) * (uint32_t)B.pitch + lane * 16
                                  : (uint32_t)min(at * 16 + row16, left) * (uint32_t)B.pitch + chunk * 16;
            }
        };
        auto begin_tile = [&]() {
            rank = terms - 1;
            term = 0;
            begin_plane();
        };
        // one of the direct loads of the slab loaded next
        auto load_part = [&](int i) {
            const uint32_t to = base + to_slot * kBuf;
            if (i < kLoadsA)
                load_to_lds(ga[i < kLoadsA ? i : 0] + (uint64_t)slab * 1024, lane * 16, to + i * kWaves * 1024);
            else
                load_to_lds(gb + (uint64_t)slab * (BLOCKED_B ? 1024 : kSlabBytes), ob[i < kLoadsA ? 0 : i - kLoadsA],
                            to + kA * kSlabBytes + (i - kLoadsA) * kWaves * 1024);
        };
        // the slab after it: of this tile, the next, or, past the last, the
        // same tile again (every step has as many loads under way)
        auto load_done = [&]() {
            to_slot = (to_slot + 1) & (kRing - 1);
            if (++slab == slabs) {
                slab = 0;
                if (++term > rank) {
                    term = 0;
                    --rank;
                }
                if (rank >= 0) {
                    if (terms > 1)
                        begin_plane();
                } else {
                    Tiles t = ahead;
                    t.next();
                    if (t.more())
                        ahead = t;
                    begin_tile();
                }
            }
        };
        auto read_part = [&](int i, Frags &f) {
            const int at = from_slot * kBuf;
            if (i < NA)
                f.a[i < NA ? i : 0] = *(const u32x4 *)(fa + at + i * 16 * kSlabBytes);
            else
                f.b[i < NA ? 0 : i - NA] = *(const u32x4 *)(fb + at + (i - NA) * 16 * kSlabBytes);
        };
        Acc acc[NA][NB];
        auto multiply = [&](const Frags &f, int i) {
            acc[i % NA][i / NA] = Mma::mul(f.a[i % NA], f.b[i / NA], acc[i % NA][i / NA]);
        };
        // Slab s of the tile from `now`, slab s + 1 to `next`, the slab loaded
        // next to where slab s was.  Slab s + 1's loads have those of the last
        // two steps behind them, which may still be under way; in a tile's
        // first three steps they have arrived before the last tile's stores,
        // which are not waited for.  The LDS reads and loads go out evenly
        // between the matrix instructions: issued in one block they would
        // hold up the waves, all of which come from the barrier together.
        int arrived = 0;                 // steps whose loads have
        auto step = [&](const Frags &now, Frags &next) {
            constexpr int kOps = NA + NB + kLoads, kMul = NA * NB;
            if (arrived > 0)
                wait_loads<63>();
            else
                wait_loads<(kRing - 2) * kLoads>();
            --arrived;
            barrier();
            from_slot = (from_slot + 1) & (kRing - 1);
#pragma unroll
            for (int i = 0, op = 0; i < kMul; ++i) {
                multiply(now, i);
#pragma unroll
                for (; op < kOps * (i + 1) / kMul; ++op) {
                    if (op < NA + NB)
                        read_part(op, next);
                    else
                        load_part(op - NA - NB);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            load_done();
        };
        Frags f0, f1;
        begin_tile();
#pragma unroll
        for (int i = 0; i < kRing; ++i) {
#pragma unroll
            for (int l = 0; l < kLoads; ++l)
                load_part(l);
            load_done();
        }
        wait_loads<0>();
        for (; tiles.more(); tiles.next()) {
            // slabs 0..3 of the tile have arrived
            barrier();
#pragma unroll
            for (int i = 0; i < NA + NB; ++i)
                read_part(i, f0);
#pragma unroll
            for (int a = 0; a < NA; ++a)
#pragma unroll
                for (int b = 0; b < NB; ++b)
                    acc[a][b] = Acc{0, 0, 0, 0};
            arrived = kRing - 1;
            asm volatile("" : "+s"(arrived));   // one form of the step, not one for each value
            for (int pair = 0; pair < pairs; ++pair) {
                step(f0, f1);            // the last step's fragments are the next tile's; they are read again
                int left = total - 2 * pair;
                asm volatile("" : "+s"(left));   // one way out of the loop: with two, the results are copied
                if (left > 1)
                    step(f1, f0);
            }
            wait_loads<0>();
            uint32_t out, point;
            tiles.place(out, point);
            finish(acc, (int64_t)out * kA, (int64_t)point * kB);
        }
    }
    // the point of acc[..][b], from the tile's first
    __device__ __forceinline__ int point_of(int b) const { return (wave % WB * NB + b) * 16 + (lane & 15); }

    // The results, as rows of Y: see Out.
    typedef Out<Y, NA> O;
    __device__ __forceinline__ typename O::Piece piece(int b, int i, int64_t a0, int64_t b0) const {
        return O::piece(lane, i, a0 + wave / WB * NA * 16, b0 + (wave % WB * NB + b) * 16);
    }
    template <typename Value, typename Mask>
    __device__ __forceinline__ void store(Y *y, int64_t ldy, int64_t a0, int64_t n_out, int64_t b0, int64_t rows, Value value,
                                          Mask mask) const {
        O::template store<NB, MERGE>(lds + kAtOut + wave * 16 * kRow, lane, y, ldy, a0 + wave / WB * NA * 16, n_out,
                                     b0 + wave % WB * NB * 16, rows, value, mask);
    }
};

}  // namespace nt

}  // namespace hpacml
