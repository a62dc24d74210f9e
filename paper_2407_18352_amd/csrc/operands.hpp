// The operands of one call of the companion ABIs, checked on the host: types,
// pitches, device memory of the current device, ranges, and overlaps.
#pragma once

#include <hip/hip_runtime.h>

#include "hpacml.h"
#include "span.hpp"

namespace hpacml {

inline hpacml_status status_of(hipError_t e) {
    return e == hipSuccess ? HPACML_OK : e == hipErrorOutOfMemory ? HPACML_E_NOMEM : HPACML_E_DEVICE;
}

inline bool is_type(int32_t t) { return t == HPACML_F32 || t == HPACML_BF16; }
inline int64_t size_of(int32_t t) { return t == HPACML_F32 ? 4 : 2; }
inline bool is_act(int32_t a) { return a == HPACML_ACT_IDENTITY || a == HPACML_ACT_RELU; }
constexpr int64_t kMaxRows = INT32_MAX, kMaxPitch = INT32_MAX;

// The operands of one call.  `add` checks one: aligned device memory of the
// current device, inside its allocation.
struct Operands {
    static constexpr int kMost = 16;
    Span s[kMost];
    int n = 0, device = -1;
    hpacml_status status = HPACML_OK;

    Operands() {
        if (hipGetDevice(&device) != hipSuccess) {
            (void)hipGetLastError();
            status = HPACML_E_DEVICE;
        }
    }
    // rows of `width` elements of `elem` bytes, `ld` elements apart
    void add(const void *p, int64_t rows, int64_t width, int64_t ld, int64_t elem, int64_t align, bool written) {
        if (status != HPACML_OK || rows == 0 || width == 0)
            return;
        if (!p || ((uintptr_t)p & (uintptr_t)(align - 1)) != 0) {
            status = HPACML_E_INVAL;
            return;
        }
        const Span v{(const char *)p, rows, ld * elem, width * elem, written};
        hipPointerAttribute_t attr;
        hipDeviceptr_t base = nullptr;
        size_t size = 0;
        if (hipPointerGetAttributes(&attr, p) != hipSuccess ||
            (attr.type != hipMemoryTypeDevice && attr.type != hipMemoryTypeManaged) || attr.device != device ||
            hipMemGetAddressRange(&base, &size, (hipDeviceptr_t)p) != hipSuccess) {
            (void)hipGetLastError();
            status = HPACML_E_INVAL;
            return;
        }
        if (!inside(v, (const char *)base, size)) {
            status = HPACML_E_RANGE;
            return;
        }
        s[n++] = v;
    }
    hpacml_status check() {
        for (int i = 0; status == HPACML_OK && i < n; ++i)
            for (int j = 0; j < i; ++j)
                if ((s[i].written || s[j].written) && !disjoint(s[i], s[j]))
                    status = HPACML_E_ALIAS;
        return status;
    }
};

inline bool pitch_ok(int64_t ld, int64_t width) { return ld >= width && ld <= kMaxPitch; }

}  // namespace hpacml
