// Group norm with an activation on channels-last records: operands, launchers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hpacml {

struct GroupNorm {
    const void *x;
    int64_t ldx, images, points;
    int32_t channels, groups;
    const float *gamma, *beta;       // or NULL
    float eps;
    int32_t act;
    float *mean, *rstd;              // [images][groups]: written (NULL: not wanted), read by the backward pass
    void *y;                         // y, or the backward pass's dx (NULL: not wanted)
    int64_t ldy;
    const void *dy;                  // backward only, as what follows
    int64_t lddy;
    float *dgamma, *dbeta;           // or NULL
    int32_t accumulate;
    char *scratch;
};
int64_t group_norm_scratch(int32_t dtype, int64_t images, int64_t points, int32_t channels, int32_t groups, bool backward);
hipError_t launch_group_norm(const GroupNorm &a, int32_t dtype, hipStream_t stream);
hipError_t launch_group_norm_backward(const GroupNorm &a, int32_t dtype, hipStream_t stream);

}  // namespace hpacml
