// Which kernel a product of matrices in 8-bit floating point takes: rules on its
// sizes, host arithmetic alone.
#pragma once

#include <stdint.h>

#include "hpacmlt.h"

namespace hpacml {
namespace f8 {

constexpr int kBlock = HPACMLT_BLOCK;
constexpr int64_t blocks_of(int64_t width) { return (width + kBlock - 1) / kBlock; }

// Whether a product of few rows is computed in one launch, whose blocks take 16
// outputs and pass over the width 32, 16 or 8 blocks of it at a time (for up to
// 16, 32 and 64 rows).  It is the faster one while that is short: up to three
// passes, counted once for every 4096 outputs (a block on each CU).  In
// microseconds, so and with codes of x and tiles, bf16: one row, 4096 -> 4096
// (one pass) 7.6 and 13.6, 8192 -> 4096 (two) 10.9 and 16.6, 4096 -> 8192 (two)
// 13.3 and 16.7, 16,384 -> 512 (four) 15.7 and 13.2, 1024 -> 65,536 (sixteen) 59
// and 19; 32 rows, 6144 -> 4096 (three) 17.6 and 18.7, 8192 -> 4096 (four) 21.4 and
// 19.0; 64 rows, 2048 -> 4096 (two) 12.1 and 15.6, 4096 -> 64 (four) 19.4 and 13.5.
inline bool few_rows(int64_t p_rows, int64_t q_rows, int64_t width) {
    const int64_t at_once = p_rows <= 16 ? 32 : p_rows <= 32 ? 16 : 8;
    return p_rows <= 64 && width > 0 && q_rows <= 3 * 4096 && (blocks_of(width) + at_once - 1) / at_once * ((q_rows + 4095) / 4096) <= 3;
}

// Tiles of 256 x 256 read less LDS for a product, tiles of 128 x 128 fill the
// chip with less and are shorter to begin and end.  Measured, large against small:
// 4096^3 56 and 65 us, 65,536 x 512 x 512 27 and 29 us; 2048^3, where the large
// ones have to split the width, 37 and 13 us; 20,000 x 1000 x 300 22 and 18 us;
// 2048 x 2048 x 131,072 in fp32, split in four, 780 and 1134 us; 256 x 256 x
// 262,144 56 and 46 us (the parts' join).  So large tiles where there is one for
// each CU and a width of four blocks, or parts of 64 blocks and more.
// A part has four blocks of the width at least: 128 x 4096 x 4096 25 us without
// that, 19 us with it.
struct Plan {
    bool big;
    uint32_t out_tiles, point_tiles;
    int32_t parts;
};
inline Plan plan_for(int64_t p_rows, int64_t q_rows, int64_t width, bool big) {
    Plan p;
    p.big = big;
    const int64_t side = big ? 256 : 128;
    p.out_tiles = (uint32_t)((q_rows + side - 1) / side);
    p.point_tiles = (uint32_t)((p_rows + side - 1) / side);
    const int64_t tiles = (int64_t)p.out_tiles * p.point_tiles, blocks = blocks_of(width), chip = big ? 256 : 512;
    const int64_t parts = tiles >= chip / 2 || tiles == 0 ? 1 : chip / tiles, most = blocks < 8 ? 1 : blocks / 4;
    p.parts = (int32_t)(parts > most ? most : parts);
    return p;
}
inline Plan plan_of(int64_t p_rows, int64_t q_rows, int64_t width) {
    const int64_t blocks = blocks_of(width);
    if (p_rows > 128 && q_rows > 128) {
        const Plan p = plan_for(p_rows, q_rows, width, true);
        if (((int64_t)p.out_tiles * p.point_tiles >= 256 && blocks >= 4) || blocks / p.parts >= 64)
            return p;
    }
    return plan_for(p_rows, q_rows, width, false);
}

}  // namespace f8
}  // namespace hpacml
