// Sums of columns.  A block takes 64 columns and a run of rows, sixteen rows at a
// time; its sum is in 64 bits and rounded once, so that hundreds of partial results
// add one rounding, or two where runs are joined by a second launch.
// One thread per column and all the rows took 58 us for 235 rows of 201 and 408
// us for 1024 rows of 2048: latency.  Sixteen threads a column, and for more than
// 512 rows runs of them in a first launch, bring that to a few microseconds.
#include "columns.hpp"

namespace hpacml {

namespace {

constexpr int64_t kOneRun = 512, kRun = 128;     // rows that one launch takes; of a run otherwise, at least
constexpr int64_t kMostRuns = 256;

int64_t runs_of(int64_t rows) {
    const int64_t runs = (rows + kRun - 1) / kRun;
    return rows <= kOneRun ? 1 : runs > kMostRuns ? kMostRuns : runs;
}

// a.room: where the sums of the runs go, NULL: the run is all there is
__global__ __launch_bounds__(1024) void sums_kernel(ColumnSums a, int64_t run) {
    __shared__ double of[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t first = (int64_t)blockIdx.y * run, last = min(first + run, a.rows);
    for (int64_t c0 = (int64_t)blockIdx.x * 64; c0 < a.width; c0 += (int64_t)gridDim.x * 64) {
        const int64_t c = c0 + lane;
        double t = 0;
        if (c < a.width)
#pragma unroll 8
            for (int64_t r = first + wave; r < last; r += 16)
                t += a.part[r * a.pitch + c];
        of[wave][lane] = t;
        __syncthreads();
        if (wave == 0 && c < a.width) {
#pragma unroll
            for (int w = 1; w < 16; ++w)
                t += of[w][lane];
            const float s = (float)t;
            if (a.room)
                a.room[blockIdx.y * a.width + c] = s;
            else if (float *to = c < a.split ? a.out : a.more) {
                const int64_t at = c < a.split ? c : c - a.split;
                to[at] = a.accumulate ? to[at] + s : s;
            }
        }
        __syncthreads();
    }
}

}  // namespace

int64_t column_sums_room(int64_t rows, int64_t width) { return runs_of(rows) > 1 ? runs_of(rows) * width : 0; }

hipError_t launch_column_sums(const ColumnSums &a, hipStream_t stream) {
    if (a.width == 0)
        return hipSuccess;
    const int64_t runs = runs_of(a.rows);
    const int64_t tiles = (a.width + 63) / 64;
    const uint32_t across = (uint32_t)(tiles < 1 << 16 ? tiles : 1 << 16);      // a launch has fewer than 2^32 threads
    ColumnSums last = a;
    if (runs > 1) {
        const int64_t run = (a.rows + runs - 1) / runs;
        sums_kernel<<<dim3(across, (uint32_t)runs), 1024, 0, stream>>>(a, run);
        last.part = a.room;
        last.rows = runs;
        last.pitch = a.width;
    }
    last.room = nullptr;
    sums_kernel<<<across, 1024, 0, stream>>>(last, last.rows);
    return hipGetLastError();
}

}  // namespace hpacml
