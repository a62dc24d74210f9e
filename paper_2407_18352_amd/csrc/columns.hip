// Sums of columns.  A block takes 64 columns and a run of rows, four rows at a
// time; sums are in 64 bits, so that a thousand partial results add no error.
// One thread per column and all the rows took 58 us for 235 rows of 201 and 408
// us for 1024 rows of 2048: latency.  Runs of 32 rows in a first launch bring
// that to a few microseconds.
#include "columns.hpp"

namespace hpacml {

namespace {

constexpr int64_t kRun = 32;              // rows of a run, at least
constexpr int64_t kMostRuns = 256;

int64_t runs_of(int64_t rows) {
    const int64_t runs = (rows + kRun - 1) / kRun;
    return runs < 2 ? 1 : runs > kMostRuns ? kMostRuns : runs;
}

__global__ __launch_bounds__(256) void sums_kernel(const float *part, int64_t rows, int64_t width, int64_t pitch, int64_t run, float *out,
                                                   int64_t ldo, int32_t accumulate) {
    __shared__ double of[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane, first = (int64_t)blockIdx.y * run, last = min(first + run, rows);
    double t = 0;
    if (c < width)
#pragma unroll 8
        for (int64_t r = first + wave; r < last; r += 4)
            t += part[r * pitch + c];
    of[wave][lane] = t;
    __syncthreads();
    if (wave == 0 && c < width) {
        const float s = (float)((of[0][lane] + of[1][lane]) + (of[2][lane] + of[3][lane]));
        float *to = out + blockIdx.y * ldo + c;
        *to = accumulate ? *to + s : s;
    }
}

}  // namespace

int64_t column_sums_room(int64_t rows, int64_t width) { return runs_of(rows) > 1 ? runs_of(rows) * width : 0; }

hipError_t launch_column_sums(const float *part, int64_t rows, int64_t width, int64_t pitch, float *out, int32_t accumulate, float *room,
                              hipStream_t stream) {
    if (width == 0)
        return hipSuccess;
    const int64_t runs = runs_of(rows);
    const uint32_t across = (uint32_t)((width + 63) / 64);
    if (runs > 1) {
        const int64_t run = (rows + runs - 1) / runs;
        sums_kernel<<<dim3(across, (uint32_t)runs), 256, 0, stream>>>(part, rows, width, pitch, run, room, width, 0);
        sums_kernel<<<across, 256, 0, stream>>>(room, runs, width, width, runs, out, 0, accumulate);
    } else
        sums_kernel<<<across, 256, 0, stream>>>(part, rows, width, pitch, rows, out, 0, accumulate);
    return hipGetLastError();
}

}  // namespace hpacml
