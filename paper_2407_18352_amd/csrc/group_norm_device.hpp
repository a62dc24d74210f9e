// What the forms of group norm share: values and activations, sums of lanes, the
// parameters' gradients; their plans and launchers.
#pragma once

#include <type_traits>

#include "columns.hpp"
#include "dense8.hpp"
#include "group_norm.hpp"
#include "hpacmlt.h"

namespace hpacml {

// By the exponential's and the reciprocal's own instructions: z log2(e) is
// rounded to 2^-24 of itself, which moves the result by |z| 2^-24 (1 - result) of
// it, less than the roundings around it.  expf and a division take some thirty
// instructions a value, and the backward pass of 134 million values is bound by
// its arithmetic as much as by memory (1024 images of 1024 points x 128 channels in
// bf16: 409 us with them, 379 without).
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504088896f)); }

// A kernel has one activation: asked at every value, it kept the compiler from
// putting a value's instructions between another's (65,536 x 512 in bf16 51 us, 40 without).
template <int ACT>
__device__ __forceinline__ float activation(float z) {
    if (ACT == HPACML_ACT_RELU)
        return relu_keep_nan(z);
    return ACT == HPACMLT_ACT_SILU ? z * sigmoid(z) : z;
}
// z is asked for in units that save an instruction: of kUnit<ACT> * z
template <int ACT>
constexpr float kUnit = ACT == HPACMLT_ACT_SILU ? 1.44269504088896f : 1.f;
// g = dy act'(z); a SiLU's slope is s (1 + z (1 - s)), s the sigmoid
template <int ACT>
__device__ __forceinline__ float activation_gradient(float dy, float z) {
    if (ACT == HPACML_ACT_RELU)
        return z <= 0.f ? 0.f : dy;
    if (ACT == HPACMLT_ACT_SILU) {
        constexpr float kLn2 = 0.693147180559945f;
        const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-z));
        return dy * s * __builtin_fmaf(z, __builtin_fmaf(-s, kLn2, kLn2), 1.f);
    }
    return dy;
}

// f(an integral constant of act)
template <typename F>
inline hipError_t with_activation(int32_t act, F f) {
    return act == HPACML_ACT_RELU     ? f(std::integral_constant<int, HPACML_ACT_RELU>())
           : act == HPACMLT_ACT_SILU ? f(std::integral_constant<int, HPACMLT_ACT_SILU>())
                                      : f(std::integral_constant<int, HPACML_ACT_IDENTITY>());
}

// Sums over `lanes` (a power of two) neighbouring lanes.  Up to 16 of them by
// operand permutations of the vector unit, which leave LDS alone; the mirrored
// orders serve, as what they exchange is the same in all lanes of a part.
template <int CONTROL>
__device__ __forceinline__ float permuted(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CONTROL, 15, 15, true));
}
template <int CONTROL>
__device__ __forceinline__ double permuted(double v) {
    typedef int Words __attribute__((ext_vector_type(2)));
    Words w = __builtin_bit_cast(Words, v);
    w[0] = __builtin_amdgcn_update_dpp(0, w[0], CONTROL, 15, 15, true);
    w[1] = __builtin_amdgcn_update_dpp(0, w[1], CONTROL, 15, 15, true);
    return __builtin_bit_cast(double, w);
}
template <typename N>
__device__ __forceinline__ N join_lanes(N t, int lanes) {
    if (lanes > 1)
        t += permuted<0xB1>(t);        // 1 0 3 2
    if (lanes > 2)
        t += permuted<0x4E>(t);        // 2 3 0 1
    if (lanes > 4)
        t += permuted<0x141>(t);       // eight mirrored
    if (lanes > 8)
        t += permuted<0x140>(t);       // sixteen mirrored
    if (lanes > 16)
        t += __shfl_xor(t, 16);
    if (lanes > 32)
        t += __shfl_xor(t, 32);
    return t;
}

// 1 / sqrt(v) of v >= 2^-126, from a rounding to fp32 (2^-24 of v) and its
// reciprocal root (1 ulp): the power of two is taken out, as v may be beyond fp32.
__device__ __forceinline__ float reciprocal_root(double v) {
    const int half = __builtin_amdgcn_frexp_exp(v) >> 1;        // (0 of an infinity and a NaN)
    return __builtin_amdgcn_ldexpf(__builtin_amdgcn_rsqf((float)__builtin_amdgcn_ldexp(v, -2 * half)), -half);
}

// A group's statistics from one reading: sums of v - pivot and of its square in
// 64 bits, where the difference and, but for one rounding, the square are exact.
// pivot, one of the group's values, is at most sqrt(n) standard deviations
// from the mean, so that squares / n less the square of sum / n loses no more
// than n of 2^53, however far from zero the values lie; of equal values both
// sums are 0.  (In 32 bits the mean's rounding was taken for a spread: a group
// of 1e5 had a deviation of 8e-3, and squares passed the range from 1.8e19 on.)
struct Moments {
    double sum = 0, squares = 0;
    __device__ __forceinline__ void add(float v, double pivot) {
        const double d = (double)v - pivot;
        sum += d;
        squares = __builtin_fma(d, d, squares);
        asm volatile("" : "+v"(sum), "+v"(squares));        // one after another: side by side, all the differences took registers
    }
    // share: 1 / n
    __device__ __forceinline__ double variance(double share) const {
        const double m = sum * share, v = __builtin_fma(squares, share, -m * m);
        return v < 0 ? 0 : v;                                    // (a NaN stays one)
    }
};

// What a thread sums a channel's gradients in, a few points' sum at a time.  It
// may have a thousand points, whose sum in 32 bits is off by 5e-7 of the values'
// own spread: with few channels more than that of a result that happens to be
// small.  64 bits for up to four channels a thread (131072 images of 1000 points,
// one channel: 362 us with either); of eight channels and more the errors even
// out, and the registers are needed.
template <int V>
using Total = typename std::conditional<V <= 4, double, float>::type;

// V neighbouring values: 16 or 8 bytes in one access, or one value.
template <typename T, int V>
struct Values {
    static constexpr int kBytes = V * (int)sizeof(T);
    typedef uint32_t Word __attribute__((ext_vector_type(kBytes >= 8 ? kBytes / 4 : 2)));
    typedef Word __attribute__((aligned(sizeof(T)))) Any;
    static __device__ __forceinline__ void load(const T *p, float (&v)[V]) {
        if constexpr (V == 1)
            v[0] = load_value(p);
        else {
            const Word w = *(const Any *)p;
            unpack(w, v);
        }
    }
    static __device__ __forceinline__ void unpack(Word w, float (&v)[V]) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if constexpr (sizeof(T) == 4) {
                const uint32_t u = w[e];
                v[e] = __builtin_bit_cast(float, u);
            } else
                v[e] = __builtin_bit_cast(float, e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
        }
    }
    // as they lie in memory
    typedef typename std::conditional<V == 1, T, Word>::type Held;
    static __device__ __forceinline__ Held hold(const T *p) {
        if constexpr (V == 1)
            return *p;
        else
            return *(const Any *)p;
    }
    static __device__ __forceinline__ void values(Held w, float (&v)[V]) {
        if constexpr (V == 1)
            v[0] = load_value(&w);
        else
            unpack(w, v);
    }
    static __device__ __forceinline__ Word words(const float (&v)[V]) {
        Word w;
#pragma unroll
        for (int e = 0; e < kBytes / 4; ++e) {
            if constexpr (sizeof(T) == 4)
                w[e] = __builtin_bit_cast(uint32_t, v[e]);
            else
                w[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
        }
        return w;
    }
    static __device__ __forceinline__ void store(T *p, const float (&v)[V]) {
        if constexpr (V == 1)
            store_value(p, v[0]);
        else
            *(Any *)p = words(v);
    }
    // past the caches
    static __device__ __forceinline__ void store_past(T *p, const float (&v)[V]) {
        if constexpr (V == 1)
            store_value(p, v[0]);
        else
            __builtin_nontemporal_store(words(v), (Any *)p);
    }
};

// The V values at p, or `none` each.  (One branch around all loads: with one for
// each, every load waited for the one before.)
template <int V>
__device__ __forceinline__ void load_parameters(const float *p, float none, float (&v)[V]) {
    if (p) {
#pragma unroll
        for (int e = 0; e < V; ++e)
            v[e] = p[e];
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
            v[e] = none;
    }
}

// dbeta and dgamma from rows of partial sums, [2][channels] each
inline hipError_t launch_parameters(const GroupNorm &a, const float *part, int64_t rows, float *room, hipStream_t stream) {
    if (!a.dgamma && !a.dbeta)
        return hipSuccess;
    return launch_column_sums({part, rows, 2 * a.channels, 2 * a.channels, a.dbeta, a.dgamma, a.channels, a.accumulate, room}, stream);
}

// The forms.  *_scratch: bytes, or -1 where the sizes do not have the form.
int64_t norm_rows_scratch(int32_t dtype, int64_t images, int64_t points, int32_t channels, int32_t groups, bool backward);
hipError_t launch_norm_rows(const GroupNorm &a, int32_t dtype, bool backward, hipStream_t stream);
int64_t norm_held_scratch(int32_t dtype, int64_t images, int64_t points, int32_t channels, int32_t groups, bool backward);
hipError_t launch_norm_held(const GroupNorm &a, int32_t dtype, bool backward, hipStream_t stream);
int64_t norm_parts_scratch(int32_t dtype, int64_t images, int64_t points, int32_t channels, int32_t groups, bool backward);
hipError_t launch_norm_parts(const GroupNorm &a, int32_t dtype, bool backward, hipStream_t stream);

}  // namespace hpacml
