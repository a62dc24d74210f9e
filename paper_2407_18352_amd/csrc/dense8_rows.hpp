// Rows of values, eight at a time: a lane takes eight consecutive values (16
// bytes of bf16 or 32 of fp32) from any address (the hardware loads and stores
// 16 bytes at an element's alignment).  Only the chunk that crosses a row's
// end goes value by value.
#pragma once

#include "dense8.hpp"

namespace hpacml {

constexpr int kChunk = 8;

// chunk at `p`, of which the first n values exist (the others become 0); n may
// be negative, value n - 1 is the row's last in any case
__device__ __forceinline__ void load_chunk(const float *p, int n, float (&v)[kChunk]) {
    if (n >= kChunk) {
        const f32x4 a = ((const f32x4_any *)p)[0], b = ((const f32x4_any *)p)[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = a[e];
            v[4 + e] = b[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < kChunk; ++e)
            v[e] = p[min(e, n - 1)];
#pragma unroll
        for (int e = 0; e < kChunk; ++e)
            v[e] = e < n ? v[e] : 0.f;
    }
}
__device__ __forceinline__ void load_chunk(const uint16_t *p, int n, float (&v)[kChunk]) {
    if (n >= kChunk) {
        const u32x4 a = *(const u32x4_any *)p;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = __builtin_bit_cast(float, a[e] << 16);
            v[2 * e + 1] = __builtin_bit_cast(float, a[e] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int e = 0; e < kChunk; ++e)
            v[e] = bf16_bits_value(p[min(e, n - 1)]);
#pragma unroll
        for (int e = 0; e < kChunk; ++e)
            v[e] = e < n ? v[e] : 0.f;
    }
}
// N chunks of rows of `width` values at once: all their loads go out before
// the first is waited for (load_chunk's branch makes each wait for its own).
// Chunk h is at at(h) and has left(h) values in front of its row's end; where
// that is less than a chunk the row's last eight values are read and moved
// down.  N chunks one by one where a row has no eight values.
template <typename T, int N, typename At, typename Left>
__device__ __forceinline__ void load_chunks(int width, At at, Left left, float (&v)[N][kChunk]) {
    if (width < kChunk) {
#pragma unroll
        for (int h = 0; h < N; ++h)
            load_chunk(at(h), left(h), v[h]);
        return;
    }
    constexpr int kParts = sizeof(T) / 2;
    u32x4 raw[N][kParts];
#pragma unroll
    for (int h = 0; h < N; ++h) {
        const T *p = at(h) + min(left(h) - kChunk, 0);
#pragma unroll
        for (int i = 0; i < kParts; ++i)
            raw[h][i] = ((const u32x4_any *)p)[i];
    }
#pragma unroll
    for (int h = 0; h < N; ++h) {
#pragma unroll
        for (int e = 0; e < kChunk; ++e) {
            const uint32_t w = raw[h][sizeof(T) == 4 ? e / 4 : 0][sizeof(T) == 4 ? e % 4 : e / 2];
            v[h][e] = __builtin_bit_cast(float, sizeof(T) == 4 ? w : e % 2 ? w & 0xFFFF0000u : w << 16);
        }
        const int down = kChunk - left(h);
        if (__any(down > 0)) {
#pragma unroll
            for (int d = 4; d > 0; d /= 2)
#pragma unroll
                for (int e = 0; e < kChunk; ++e) {
                    const float from = e + d < kChunk ? v[h][e + d] : 0.f;
                    v[h][e] = down > 0 && (down & d) ? from : v[h][e];
                }
#pragma unroll
            for (int e = 0; e < kChunk; ++e)
                v[h][e] = down >= kChunk ? 0.f : v[h][e];
        }
    }
}
__device__ __forceinline__ void store_chunk(float *p, int n, const float (&v)[kChunk]) {
    if (n >= kChunk) {
        ((f32x4_any *)p)[0] = f32x4{v[0], v[1], v[2], v[3]};
        ((f32x4_any *)p)[1] = f32x4{v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
        for (int e = 0; e < kChunk; ++e)
            if (e < n)
                p[e] = v[e];
    }
}
__device__ __forceinline__ void store_chunk(uint16_t *p, int n, const float (&v)[kChunk]) {
    if (n >= kChunk) {
        u32x4 a;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            a[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
        *(u32x4_any *)p = a;
    } else {
#pragma unroll
        for (int e = 0; e < kChunk; ++e)
            if (e < n)
                p[e] = bf16_bits(v[e]);
    }
}

// largest magnitude as bits: an infinity is above every number, a NaN above it
__device__ __forceinline__ uint32_t top_bits(const float (&v)[kChunk]) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < kChunk; ++e)
        m = max(m, __builtin_bit_cast(uint32_t, v[e]) & 0x7FFFFFFFu);
    return m;
}
template <int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
#pragma unroll
    for (int d = LANES / 2; d > 0; d /= 2)
        v = max(v, (uint32_t)__shfl_xor((int)v, d));
    return v;
}

// Scale and codes of a row whose largest magnitude has the bits `top`.  A row
// that counts as zeros has scale 0 and codes 0; one with an infinity or a NaN
// has scale NaN and codes 0.
struct RowScale {
    float scale, inv;
    bool live;
    __device__ __forceinline__ explicit RowScale(uint32_t top) {
        const float amax = __builtin_bit_cast(float, top);
        const bool finite = top < 0x7F800000u;
        live = finite && amax >= 0x1p-119f;
        inv = live ? 127.f / amax : 0.f;
        scale = !finite ? __builtin_nanf("") : live ? amax / 127.f : 0.f;
    }
    __device__ __forceinline__ uint2 codes(const float (&v)[kChunk]) const {
        uint32_t q[2] = {0, 0};
        if (live) {
#pragma unroll
            for (int e = 0; e < kChunk; ++e)
                q[e / 4] |= ((uint32_t)(int32_t)rintf(v[e] * inv) & 0xFFu) << (8 * (e % 4));
        }
        return uint2{q[0], q[1]};
    }
};

}  // namespace hpacml
