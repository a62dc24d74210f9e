// The product both operands of which lie along k: C[a][b] = sum_k A[a][k] B[b][k],
// int8 codes with 32-bit sums or bf16 with fp32 sums.
//
// A block computes a tile of C.  The operands pass through LDS in slabs of 128
// bytes of k (128 codes, 64 bf16), double-buffered: while the block works on a
// slab, direct global-to-LDS loads bring the next.  A row of a slab is eight
// 16-byte chunks, chunk c stored at c ^ swizzle(row), so that the 16 rows a
// matrix instruction reads at one chunk fall on different banks; the direct
// loads can't permute what they write, so each lane fetches the chunk that
// belongs where its bytes land.  A holds the outputs and B the points: a lane
// of the matrix instruction's result then has four consecutive outputs of one
// point, which is what a row-major store wants.
//
// The direct loads are inline assembly: seeing them, the compiler would make
// every LDS read wait for all of them.  Their completion is waited for by
// hand (all of them, once per slab) before the barrier that publishes a slab.
// That one barrier per slab also keeps the next loads off the buffer until
// every wave has its fragments of it in registers.
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
// this wave's loads have arrived and its LDS reads are in registers
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0070); }
__device__ __forceinline__ void barrier() { asm volatile("s_barrier" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_offset(const void *p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p;
}
__device__ __forceinline__ int swizzle(int row) { return row & 7; }

// what a load beyond an operand's width reads
__device__ __align__(16) const uint32_t zero_chunk[4] = {0, 0, 0, 0};

// One operand: rows `pitch` bytes apart, of which `width` bytes count (the
// rest of the slabs is zero), in `terms` planes `plane` bytes apart.
struct Operand {
    const char *base;
    int64_t rows, pitch, width, plane;
};

// Blocks of WA x WB waves, each NA x NB tiles of 16 x 16.
template <typename Mma, int WA, int WB, int NA, int NB>
struct Tile {
    static constexpr int kWaves = WA * WB, kThreads = 64 * kWaves;
    static constexpr int kA = 16 * NA * WA, kB = 16 * NB * WB;
    static constexpr int kBuf = (kA + kB) * kSlabBytes;
    static constexpr int kLoadsA = kA / (8 * kWaves), kLoadsB = kB / (8 * kWaves);
    static_assert(kLoadsA * 8 * kWaves == kA && kLoadsB * 8 * kWaves == kB, "whole loads per wave");
    typedef typename Mma::Acc Acc;

    const char *pa[kLoadsA], *pb[kLoadsB];
    int wave, lane;

    // acc[a][b]: outputs a0 + 16 (WA-wave * NA + a) + 4 (lane / 16) + e of
    // point b0 + 16 (WB-wave * NB + b) + lane % 16
    // terms: 1, or 3 planes of each operand of which the products of ranks
    // that sum to at most 2 are taken, the smallest first.  EDGE: the
    // operands' widths may end inside a slab.
    template <bool EDGE>
    __device__ __forceinline__ void run(const Operand &A, const Operand &B, int64_t a0, int64_t b0, int terms, char *lds,
                                        Acc (&acc)[NA][NB]) {
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int row8 = lane >> 3, chunk = (lane & 7) ^ swizzle(row8);   // swizzle(row) depends on row % 8 alone
        int64_t oa[kLoadsA], ob[kLoadsB];
#pragma unroll
        for (int i = 0; i < kLoadsA; ++i)
            oa[i] = min(a0 + (i * kWaves + wave) * 8 + row8, A.rows - 1) * A.pitch + chunk * 16;
#pragma unroll
        for (int i = 0; i < kLoadsB; ++i)
            ob[i] = min(b0 + (i * kWaves + wave) * 8 + row8, B.rows - 1) * B.pitch + chunk * 16;
        const uint32_t base = lds_offset(lds);
        const int wa = wave / WB, wb = wave % WB;
        const int fr = (lane & 15) * kSlabBytes, sw = swizzle(lane & 7), grp = lane >> 4;
        const char *fa = lds + wa * NA * 16 * kSlabBytes + fr, *fb = lds + (kA + wb * NB * 16) * kSlabBytes + fr;

        const int slabs = (int)((max(A.width, B.width) + kSlabBytes - 1) / kSlabBytes);
        int rank = terms - 1, term = 0, slab = 0;   // what is loaded next
        const char *ga = A.base + term * A.plane, *gb = B.base + (rank - term) * B.plane;
        auto load = [&](int buf) {
            const uint32_t to = base + buf * kBuf + wave * 1024;
            const int64_t k = (int64_t)slab * kSlabBytes;
#pragma unroll
            for (int i = 0; i < kLoadsA; ++i) {
                const void *g = ga + oa[i] + k;
                if (EDGE && k + chunk * 16 >= A.width)
                    g = zero_chunk;
                load_to_lds(g, to + i * kWaves * 1024);
            }
#pragma unroll
            for (int i = 0; i < kLoadsB; ++i) {
                const void *g = gb + ob[i] + k;
                if (EDGE && k + chunk * 16 >= B.width)
                    g = zero_chunk;
                load_to_lds(g, to + (kA * kSlabBytes) + i * kWaves * 1024);
            }
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
        const int total = slabs * (terms * (terms + 1) / 2);
        load(0);
        for (int s = 0; s < total; ++s) {
            wait_loads();
            barrier();
            const int cur = (s & 1) * kBuf;
            if (s + 1 < total)
                load((s + 1) & 1);
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                const int at = cur + (((ks * 4 + grp) ^ sw) * 16);
                u32x4 a[NA], b[NB];
#pragma unroll
                for (int t = 0; t < NA; ++t)
                    a[t] = *(const u32x4 *)(fa + at + t * 16 * kSlabBytes);
#pragma unroll
                for (int t = 0; t < NB; ++t)
                    b[t] = *(const u32x4 *)(fb + at + t * 16 * kSlabBytes);
#pragma unroll
                for (int u = 0; u < NB; ++u)
#pragma unroll
                    for (int t = 0; t < NA; ++t)
                        acc[t][u] = Mma::mul(a[t], b[u], acc[t][u]);
            }
        }
    }
    // first output and point of this lane's acc[t][u]
    __device__ __forceinline__ int out_of(int t) const { return (wave / WB * NA + t) * 16 + (lane >> 4) * 4; }
    __device__ __forceinline__ int point_of(int u) const { return (wave % WB * NB + u) * 16 + (lane & 15); }
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
