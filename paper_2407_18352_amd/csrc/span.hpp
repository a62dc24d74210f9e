// Matrix operands as ranges of addresses: whether one lies inside its
// allocation, and whether two have an element in common.  Host arithmetic;
// nothing is dereferenced.
#pragma once

#include <stdint.h>

namespace hpacml {

// `rows` (at least 1) rows of `width` (at least 1) bytes, `pitch` bytes apart.
struct Span {
    const char *at;
    int64_t rows, pitch, width;
    bool written;
    // of a span inside its allocation
    const char *end() const { return at + (rows - 1) * pitch + width; }
};

// Inside the `size` bytes from `base` on.  Rows times pitch may pass 64 bits
// (2^31 rows of 2^31 fp32 values), so it is not formed.
inline bool inside(const Span &s, const char *base, uint64_t size) {
    const uint64_t before = (uint64_t)((uintptr_t)s.at - (uintptr_t)base);
    if (s.at < base || before > size || (uint64_t)s.width > size - before)
        return false;
    const uint64_t room = size - before - (uint64_t)s.width;
    return s.rows == 1 || (uint64_t)s.pitch <= room / (uint64_t)(s.rows - 1);
}

// No element in common, of spans inside their allocations: ranges that do not
// meet, or rows of equal pitch that keep to columns of their own.
inline bool disjoint(const Span &a, const Span &b) {
    if (a.end() <= b.at || b.end() <= a.at)
        return true;
    if (a.pitch != b.pitch)
        return false;
    int64_t r = (b.at - a.at) % a.pitch;
    if (r < 0)
        r += a.pitch;
    return a.width <= r && r + b.width <= a.pitch;
}

}  // namespace hpacml
