// The product both operands of which lie along k: C[a][b] = sum_k A[a][k] B[b][k],
// int8 codes with 32-bit sums or bf16 with fp32 sums.
//
// A block computes a tile of C.  The operands pass through LDS in slabs of 64
// bytes of k (64 codes, 32 bf16: one matrix instruction's depth), a ring of
// kRing of them filled by direct global-to-LDS loads.  While the matrix cores
// work on slab s from registers, a wave reads slab s + 1's fragments from LDS
// and the loads of slabs up to s + kRing are under way; what a slab's loads
// have to wait for in the memory system is covered by the slabs before it.
// One barrier per slab publishes slab s + 1 (its loads have been waited for)
// and frees slab s (its fragments are in registers).
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
// Otherwise rows `pitch` bytes apart, of which `width` bytes count (the rest
// of the last slab reads as zero).
struct Operand {
    const char *base;
    int64_t rows, pitch, width, plane;
};

// Blocks of WA x WB waves, each NA x NB tiles of 16 x 16.
template <typename Mma, int WA, int WB, int NA, int NB, int RING = 4>
struct Tile {
    static constexpr int kWaves = WA * WB, kThreads = 64 * kWaves, kRing = RING;
    static constexpr int kA = 16 * NA * WA, kB = 16 * NB * WB;
    static constexpr int kBuf = (kA + kB) * kSlabBytes, kLds = kRing * kBuf;
    static constexpr int kLoadsA = kA / (16 * kWaves), kLoadsB = kB / (16 * kWaves), kLoads = kLoadsA + kLoadsB;
    static_assert(kLoadsA * 16 * kWaves == kA && kLoadsB * 16 * kWaves == kB, "whole loads per wave");
    typedef typename Mma::Acc Acc;
    struct Frags {
        u32x4 a[NA], b[NB];
    };

    int wave, lane;

    // acc[a][b]: outputs a0 + 16 (WA-wave * NA + a) + 4 (lane / 16) + e of
    // point b0 + 16 (WB-wave * NB + b) + lane % 16
    // terms: 1, or 3 planes of each operand of which the products of ranks
    // that sum to at most 2 are taken, the smallest first.  A is BLOCKED.
    template <bool BLOCKED_B>
    __device__ __forceinline__ void run(const Operand &A, const Operand &B, int64_t a0, int64_t b0, int terms, char *lds,
                                        Acc (&acc)[NA][NB]) {
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int row16 = lane >> 2, chunk = (lane & 3) ^ chunk_turn(row16);   // chunk_turn(row) depends on row % 16 alone
        int64_t oa[kLoadsA], ob[kLoadsB];
#pragma unroll
        for (int i = 0; i < kLoadsA; ++i)
            oa[i] = min(a0 / 16 + i * kWaves + wave, (A.rows - 1) / 16) * A.pitch + lane * 16;
#pragma unroll
        for (int i = 0; i < kLoadsB; ++i)
            ob[i] = BLOCKED_B ? min(b0 / 16 + i * kWaves + wave, (B.rows - 1) / 16) * B.pitch + lane * 16
                              : min(b0 + (i * kWaves + wave) * 16 + row16, B.rows - 1) * B.pitch + chunk * 16;
        const uint32_t base = lds_offset(lds) + wave * 1024;
        const int wa = wave / WB, wb = wave % WB;
        const int fr = (lane & 15) * kSlabBytes + ((lane >> 4) ^ chunk_turn(lane & 15)) * 16;
        const char *fa = lds + wa * NA * 16 * kSlabBytes + fr, *fb = lds + (kA + wb * NB * 16) * kSlabBytes + fr;

        const int slabs = (int)((A.width + kSlabBytes - 1) / kSlabBytes);
        const int total = slabs * (terms * (terms + 1) / 2);
        int rank = terms - 1, term = 0, slab = 0, to_slot = 0, from_slot = 0;   // what is loaded and read next
        const char *ga = A.base + term * A.plane, *gb = B.base + (rank - term) * B.plane;
        // one of the direct loads of the slab loaded next
        auto load_part = [&](int i) {
            const uint32_t to = base + to_slot * kBuf;
            const bool of_a = i < kLoadsA;
            const int n = of_a ? i : i - kLoadsA;
            const char *g = of_a ? ga + oa[of_a ? n : 0] + (int64_t)slab * 1024
                                 : gb + ob[of_a ? 0 : n] + (int64_t)slab * (BLOCKED_B ? 1024 : kSlabBytes);
            const bool rest = !BLOCKED_B && !of_a;
            load_to_lds(rest ? chosen(slab * kSlabBytes + chunk * 16 < B.width, g) : g, to + (of_a ? 0 : kA * kSlabBytes) + n * kWaves * 1024);
        };
        auto load_done = [&]() {
            to_slot = to_slot + 1 == kRing ? 0 : to_slot + 1;
            if (++slab == slabs) {
                slab = 0;
                if (++term > rank) {
                    term = 0;
                    --rank;
                }
                ga = A.base + term * A.plane;
                gb = B.base + (rank - term) * B.plane;
            }
        };
        auto load = [&]() {
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                load_part(i);
            load_done();
        };
        auto read_part = [&](int i, Frags &f) {
            const int at = from_slot * kBuf;
            if (i < NA)
                f.a[i < NA ? i : 0] = *(const u32x4 *)(fa + at + i * 16 * kSlabBytes);
            else
                f.b[i < NA ? 0 : i - NA] = *(const u32x4 *)(fb + at + (i - NA) * 16 * kSlabBytes);
        };
        auto read_done = [&]() { from_slot = from_slot + 1 == kRing ? 0 : from_slot + 1; };
        auto read = [&](Frags &f) {
#pragma unroll
            for (int i = 0; i < NA + NB; ++i)
                read_part(i, f);
            read_done();
        };
        auto multiply = [&](const Frags &f, int i) {
            acc[i % NA][i / NA] = Mma::mul(f.a[i % NA], f.b[i / NA], acc[i % NA][i / NA]);
        };
        // Slab s from `now`, slab s + 1 to `next`, slab s + kRing to where
        // slab s was.  Slab s + 1's loads have kRing - 2 slabs behind them
        // that may still be under way.  The LDS reads and loads go out evenly
        // between the matrix instructions: issued in one block they would
        // hold up the waves, all of which come from the barrier together.
        auto step = [&](const Frags &now, Frags &next) {
            constexpr int kOps = NA + NB + kLoads, kMul = NA * NB;
            wait_loads<(kRing - 2) * kLoads>();
            barrier();
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
            read_done();
        };
        // the same near the end, where no more loads follow
        auto last_step = [&](int s, const Frags &now, Frags &next) {
            wait_loads<0>();
            if (s + 1 < total) {
                barrier();
                read(next);
            }
#pragma unroll
            for (int i = 0; i < NA * NB; ++i)
                multiply(now, i);
        };
        Frags f0, f1;
#pragma unroll
        for (int i = 0; i < kRing; ++i)
            if (i < total)
                load();
        if (total >= kRing)
            wait_loads<(kRing - 1) * kLoads>();
        else
            wait_loads<0>();
        barrier();
        read(f0);
        int s = 0;
        for (; s + 1 + kRing < total; s += 2) {
            step(f0, f1);
            step(f1, f0);
        }
        if (s + kRing < total) {
            step(f0, f1);
            ++s;
            f0 = f1;
        }
        for (; s < total; s += 2) {
            last_step(s, f0, f1);
            if (s + 1 < total)
                last_step(s + 1, f1, f0);
        }
    }
    // the point of acc[..][b], from the tile's first
    __device__ __forceinline__ int point_of(int b) const { return (wave % WB * NB + b) * 16 + (lane & 15); }

    // The results, as rows of Y.  value(a, n, b, r, v): the four results of
    // acc[a][b], outputs n.. (a multiple of 4 and below A.rows rounded up to
    // one; past the last ones if the tile is) of point r (not above the last).
    // mask(r, n, chunk): changes the 16 bytes that are about to be stored as
    // outputs n.. of point r.  A wave turns 16 points at a time in LDS, so that
    // its stores are 16-byte pieces of long runs of a row; they bypass the
    // caches (the results are read by a later kernel, if at all): 131,072 x
    // 1024 -> 1024 in 8 bits takes 146 us, 187 us without that, 227 us with
    // stores as the matrix instruction leaves its results.
    template <typename Y, typename Value, typename Mask>
    __device__ __forceinline__ void store(Y *y, int64_t ldy, int64_t a0, int64_t n_out, int64_t b0, int64_t rows, char *lds,
                                          Value value, Mask mask) const {
        constexpr int kPer = 16 / sizeof(Y), kRow = NA * 16 * sizeof(Y), kPitch = kRow + 16, kChunks = kRow / 16;
        static_assert(kWaves * 16 * kPitch <= kLds, "room for the waves' rows");
        const int wa = wave / WB, wb = wave % WB;
        wait_loads<0>();
        barrier();                       // the ring is free
        char *own = lds + wave * 16 * kPitch;
        const int64_t last = (n_out - 1) & ~(int64_t)3;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int64_t p0 = b0 + (wb * NB + b) * 16;
#pragma unroll
            for (int a = 0; a < NA; ++a) {
                float v[4];
                value(a, min(a0 + (wa * NA + a) * 16 + (lane >> 4) * 4, last), b, min(p0 + (lane & 15), rows - 1), v);
                store_four((Y *)(own + (lane & 15) * kPitch) + a * 16 + (lane >> 4) * 4, v);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // one wave's LDS accesses are in order
#pragma unroll
            for (int i = 0; i < kChunks / 4; ++i) {
                const int at = i * 64 + lane, row = at / kChunks, c = at % kChunks;
                u32x4 u = *(const u32x4 *)(own + row * kPitch + c * 16);
                const int64_t r = p0 + row, n = a0 + wa * NA * 16 + c * kPer;
                if (r < rows && n < n_out) {
                    mask(r, n, u);
                    Y *to = y + r * ldy + n;
                    if (n + kPer <= n_out) {
                        __builtin_nontemporal_store(u, (u32x4_any *)to);
                    } else {
#pragma unroll
                        for (int e = 0; e < kPer; ++e)
                            if (n + e < n_out)
                                to[e] = element<Y>(u, e);
                    }
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
    }
};

// Rows of one launch: a launch of more than 2^22 blocks is split (a grid holds
// fewer than 2^32 threads).
inline int64_t rows_per_launch(uint32_t out_tiles, int64_t tile) {
    const int64_t point_tiles = (int64_t)(1 << 22) / out_tiles;
    return (point_tiles < 1 ? 1 : point_tiles) * tile;
}

// Block id -> tile.  Blocks go to the eight XCDs in turn; each XCD takes a
// contiguous run of tiles, so that what its blocks share meets in its L2, and
// a run goes through groups of `kGroup` point tiles by all output tiles.
constexpr int kGroup = 4;
struct TileAt {
    int64_t out, point;
};
__device__ __forceinline__ TileAt tile_at(uint32_t block, uint32_t blocks, uint32_t out_tiles, uint32_t point_tiles) {
    const uint32_t xcd = block & 7, in = block >> 3, per = blocks >> 3, more = blocks & 7;
    const uint32_t t = xcd * per + min(xcd, more) + in;
    const uint32_t group = t / (kGroup * out_tiles), r = t - group * kGroup * out_tiles;
    const uint32_t high = min((uint32_t)kGroup, point_tiles - group * kGroup);
    return {r / high, (int64_t)group * kGroup + r % high};
}

}  // namespace nt

}  // namespace hpacml
