// The norm of many gradients, and clipping: what the kernels read.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hpacml {

// A run of one gradient's values.
struct GradChunk {
    const void *from;
    void *to;
    int32_t count;
    int32_t types;        // bit 0: from is bf16, bit 1: to is bf16
};

constexpr int kGradBlocks = 1024;        // partial results at most
constexpr size_t kGradScratch = kGradBlocks * 8;

// Values of a chunk in a set of `total`: enough chunks for the chip, and not
// more than a block's work is worth.
inline int64_t grad_chunk(int64_t total) {
    const int64_t per = total / 8192 / 1024 * 1024;
    return per < 2048 ? 2048 : per > 32768 ? 32768 : per;
}

// kind: HPACMLT_NORM_*.  partial: kGradScratch bytes.
hipError_t launch_grad_norm(const GradChunk *chunks, int64_t n, int32_t kind, float *norm, void *partial, hipStream_t stream);
hipError_t launch_grad_clip(const GradChunk *chunks, int64_t n, int32_t kind, double most, float *norm, void *partial, hipStream_t stream);

}  // namespace hpacml
