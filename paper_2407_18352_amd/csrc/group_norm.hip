// Group norm with an activation, channels last, and its backward pass.
//
// Three forms, by size.  Where an image is one point (a hidden layer's activations), a few
// lanes of a wave hold a group of it in registers: one reading, one launch
// (rows_*).  Where a group of an image fits the registers of a block, the same
// with a block (held_*).  Otherwise three launches (parts_*): sums of every channel over runs
// of an image's points, which a second launch joins to the groups' statistics,
// and the results, from a second reading (of what the first left in the
// Infinity Cache, up to 256 MB).  A thread has the same few neighbouring
// channels throughout, so that their parameters are in registers, and the sums
// that the parameters' gradients are made of stay apart until the end.
//
// Statistics: sums in 64 bits of what the values are more than one of them, and
// of its squares (Moments); in parts those of every channel and run, which are
// joined as (mean, deviation), so that no difference of large sums occurs.
#include "group_norm_device.hpp"

namespace hpacml {

int64_t group_norm_scratch(int32_t dtype, int64_t images, int64_t points, int32_t channels, int32_t groups, bool backward) {
    if (images == 0)
        return 0;
    int64_t need = norm_rows_scratch(dtype, images, points, channels, groups, backward);
    if (need < 0)
        need = norm_held_scratch(dtype, images, points, channels, groups, backward);
    return need < 0 ? norm_parts_scratch(dtype, images, points, channels, groups, backward) : need;
}

namespace {

hipError_t launch(const GroupNorm &a, int32_t dtype, bool backward, hipStream_t stream) {
    if (norm_rows_scratch(dtype, a.images, a.points, a.channels, a.groups, backward) >= 0)
        return launch_norm_rows(a, dtype, backward, stream);
    if (norm_held_scratch(dtype, a.images, a.points, a.channels, a.groups, backward) >= 0)
        return launch_norm_held(a, dtype, backward, stream);
    return launch_norm_parts(a, dtype, backward, stream);
}

}  // namespace

hipError_t launch_group_norm(const GroupNorm &a, int32_t dtype, hipStream_t stream) {
    return a.images ? launch(a, dtype, false, stream) : hipSuccess;
}

hipError_t launch_group_norm_backward(const GroupNorm &a, int32_t dtype, hipStream_t stream) {
    if (a.images)
        return launch(a, dtype, true, stream);
    return a.accumulate ? hipSuccess : launch_parameters(a, nullptr, 0, nullptr, stream);
}

}  // namespace hpacml
