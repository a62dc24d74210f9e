// Sums of the columns of a matrix of partial results, in a fixed order.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hpacml {

// Of `rows` rows of `width` columns, `pitch` floats apart, the sums of the first
// `split` columns (+)= to `out`, those of the others to `more` (either may be
// NULL: not wanted).  Many rows are joined in two launches, through `room`:
// column_sums_room floats.
struct ColumnSums {
    const float *part;
    int64_t rows, width, pitch;
    float *out, *more;
    int64_t split;
    int32_t accumulate;
    float *room;
};
int64_t column_sums_room(int64_t rows, int64_t width);
hipError_t launch_column_sums(const ColumnSums &a, hipStream_t stream);

}  // namespace hpacml
