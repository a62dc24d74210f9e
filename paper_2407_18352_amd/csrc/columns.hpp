// Sums of the columns of a matrix of partial results, in a fixed order.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hpacml {

// out[c] (+)= sum over `rows` rows of part[r * pitch + c].  Many rows are joined
// in two launches, through `room`: column_sums_room floats.
int64_t column_sums_room(int64_t rows, int64_t width);
hipError_t launch_column_sums(const float *part, int64_t rows, int64_t width, int64_t pitch, float *out, int32_t accumulate, float *room,
                              hipStream_t stream);

}  // namespace hpacml
