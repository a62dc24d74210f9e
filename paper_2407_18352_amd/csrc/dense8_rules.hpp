// Which form of a kernel a call of the 8-bit dense layers takes, by its sizes
// alone.  Host arithmetic.
#pragma once

#include <stdint.h>

#include <cmath>

namespace hpacml {

namespace nt {

// The tile (outputs x points) of a product: the largest that leaves no CU
// without one, by these times (us, 8-bit products):
//   rows x out <- in       64 x 64  128 x 128  128 x 256  256 x 256
//   4096 x 256 <- 256          4.6        7.5        8.1       13.8
//   262144 x 64 <- 64         15.0       23.0       18.5       35.0
//   4096 x 1024 <- 1024       11.7       10.9       12.5       20.5
//   1024 x 4096 <- 4096       29.1       23.5       29.5       46.9
//   65536 x 256 <- 256        17.9       15.8       13.8       15.1
//   16384 x 512 <- 512        14.0       11.6       10.5       16.6
//   16384 x 1024 <- 1024      37.0       26.8       24.0       23.3
//   4096 x 4096 <- 4096      109.0       70.7       73.3       59.4
//   65536 x 4096 <- 4096      2620       1280       1026        899
// The largest needs more tiles where k is short, and outputs of which it does
// not pad more than a quarter away (with the launch that forms the codes):
//   65536 x 2048 <- 512        190        147        141        127
//   131072 x 1280 <- 64        110         96         93         87
//   100000 x 256 <- 600         90         84         87         83
//   100000 x 300 <- 600         99         97         98        119
//   100000 x 300 <- 2048       258        225        215        241
//   65536 x 640 <- 2048        230        176        170        173
// and the same in bf16, dx of (rows, its outputs <- its inputs):
//   262144 x 256 <- 256        123         93         87         79
//   65536 x 2048 <- 64         146        112        108         91
//   200000 x 300 <- 128         91         78         77         91
enum class Size { k64x64, k128x128, k128x256, k256x256 };
inline Size tile_for(int64_t n_out, int64_t rows, int64_t slabs) {
    auto tiles = [&](int64_t outs, int64_t points) { return (n_out + outs - 1) / outs * ((rows + points - 1) / points); };
    const bool many = tiles(256, 256) >= (slabs >= 16 ? 200 : 384);
    return n_out <= 64 || tiles(64, 64) <= 512                     ? Size::k64x64
           : tiles(128, 128) <= 256                                ? Size::k128x128
           : many && 8 * tiles(256, 256) <= 5 * tiles(128, 256)    ? Size::k256x256
                                                                   : Size::k128x256;
}

}  // namespace nt

// How dw is computed: the tile (outputs x channels), the planes at once, and
// the parts of the rows.  More parts shorten the blocks' loops and lengthen the
// join (a part of dw is written and read: n_out * n_in * 8 bytes at about 4.5
// TB/s); at most as many as the chip holds at once.  The tile is the one whose
// time is least by the times measured for a slab of 32 rows in a full chip, at
// 131,072 rows: 1.10, 0.67, 0.68, 0.79 and 0.47 us (the larger tiles need
// fewer of them), with three planes at once 1.9 and 0.9 us.
struct DwForm {
    int32_t tile;           // of kDwTiles
    int32_t splits;         // parts of the rows that sum into dw apart
    int64_t rows_per_split;
};
struct DwTileTimes {
    int outs, channels, planes, at_once;
    double slab_us;
};
constexpr DwTileTimes kDwTiles[] = {{256, 256, 1, 256, 1.10}, {256, 128, 1, 256, 0.67}, {128, 256, 1, 256, 0.68},
                                    {128, 128, 1, 512, 0.79}, {64, 64, 1, 768, 0.47},   {128, 128, 3, 256, 1.9},
                                    {64, 64, 3, 512, 0.9}};
constexpr double kStartUs = 4;     // until a block's first slabs are there; and of another launch

inline DwForm choose_dw(int64_t rows, int32_t n_out, int32_t n_in, int planes) {
    DwForm p{};
    const double slabs = (double)((rows + 31) / 32), part_us = (double)n_out * n_in * 8 / 4.5e6;
    double best = 0;
    for (int i = 0; i < (int)(sizeof(kDwTiles) / sizeof(kDwTiles[0])); ++i) {
        const DwTileTimes &t = kDwTiles[i];
        if (t.planes > planes)
            continue;
        const double tiles = (double)((n_out + t.outs - 1) / t.outs) * ((n_in + t.channels - 1) / t.channels);
        const double us = t.slab_us * (planes / t.planes), most = std::floor(t.at_once / tiles);
        double splits = std::floor(std::sqrt(slabs * us / (part_us + 0.02)) + 0.5);
        splits = std::fmax(1, std::fmin(splits, std::fmin(most, slabs)));
        const double rounds = std::ceil(tiles * splits / t.at_once);
        const double time = rounds * (kStartUs + std::ceil(slabs / splits) * us) + (splits > 1 ? kStartUs + splits * part_us : 0);
        if (i == 0 || time < best) {
            best = time;
            p.tile = i;
            p.splits = (int32_t)splits;
        }
    }
    p.rows_per_split = ((rows + p.splits - 1) / p.splits + 31) / 32 * 32;
    p.splits = p.rows_per_split ? (int32_t)((rows + p.rows_per_split - 1) / p.rows_per_split) : 1;
    return p;
}

// One launch for dx, dw and db (backward8_few.hip), or operands laid out, dx,
// dw and their join apart.  What counts is the number of 32 x 32 results, a
// block each; that launch reads an operand again for every 32 results across.
// Device us, one launch and the general form, of (rows) outputs <- inputs:
//                                 fp32           bf16
//   (256) 64 <- 64              4.7   16.7      4.3  13.0
//   (256) 512 <- 512 (384)      8.5   34.4      6.0  18.0
//   (1024) 256 <- 256 (320)    13.1   27.4     10.6  16.3
//   (256) 64 <- 2048 (640)      7.2   17.7      6.2  13.9
//   (1024) 512 <- 512 (768)    19.0   41.1     13.8  21.6
//   (1) 1024 <- 1024 (1056)     9.4   46.5      7.1  16.2
//   (512) 64 <- 2048 (1152)    11.8   20.1      9.9  15.1
//   (256) 1024 <- 1024 (1280)  19.1   58.0     13.3  19.2
// and beyond the limits, where they cross:
//   (512) 1024 <- 1024 (1536)  30.2   60.2     20.9  28.6
//   (1024) 1024 <- 1024 (2048) 62.7   65.4     37.6  35.2
//   (1024) 1024 <- 2048 (4096)  118   82.2     88.0  41.1
//   (256) 2048 <- 2048 (4608)  66.5   91.2     46.7  36.1
//   (1500) 64 <- 64            15.9   18.3     13.5  14.2
//   (2048) 64 <- 64            20.6   18.1     17.4  14.4
//   (2048) 512 <- 512 (1280)   44.9   45.9     25.3  24.6
//   (4096) 64 <- 64            36.8   18.1     31.6  15.6
inline bool few_rows(int64_t rows, int32_t n_out, int32_t n_in) {
    auto tiles = [](int64_t n) { return (n + 31) / 32; };
    return rows <= 1024 && tiles(n_in) * (tiles(rows) + tiles(n_out)) <= 1280;
}

}  // namespace hpacml
