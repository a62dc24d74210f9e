// Group norm of images whose groups fit a block's registers: one reading, one
// launch.  1024 images of 1024 points x 128 channels in bf16, SiLU, take 136 us (3.9
// TB/s; 163 with two joins, of sums in 32 bits).  Their gradients take 229 us (3.5
// TB/s): the activation's gradient takes as many cycles as the loads, and there is
// room for the registers of two blocks a CU.  Three launches, each value read twice,
// took 379 us.  Results go past the caches (4096 images of 64 points x 256 channels in
// bf16 57 us, 59.5 through them, with a reader behind 96 either way; of 2 MB 8.5 and
// 13.8 either way), those of the gradients do not (229 us, 234 past them).
#include "group_norm_device.hpp"

namespace hpacml {

namespace {

// ---- images whose groups fit a block's registers -----------------------------------------

// A block holds a run of neighbouring groups of one image: `across` vectors of
// each point, `high` points at a time, up to I of them a thread.  It goes from
// image to image with the same channels.
struct Held {
    int32_t groups, across, high;      // of a run; vectors of a run; points at a time
    int32_t runs, strides;             // of a row; blocks of the same run
};

// Sums of `t` over the threads of each of the run's groups.  Thread t has
// vector t % across of the run; a group is `each` vectors.  of: a pair per
// thread, then one per group.  Groups' sums are taken by 32 threads each.
template <typename Pair>
__device__ __forceinline__ Pair join_groups(Pair t, const Held &h, int each, int group, bool here, Pair *of, Pair *of_group) {
    __syncthreads();
    of[threadIdx.x] = t;
    __syncthreads();
    const int entries = h.high * each;
    for (int g = threadIdx.x >> 5; g < h.groups; g += blockDim.x >> 5) {
        Pair s = {0, 0};
        for (int i = threadIdx.x & 31; i < entries; i += 32) {
            const Pair o = of[i / each * h.across + g * each + i % each];
            s.x += o.x;
            s.y += o.y;
        }
        s.x = join_lanes(s.x, 32);
        s.y = join_lanes(s.y, 32);
        if ((threadIdx.x & 31) == 0)
            of_group[g] = s;
    }
    __syncthreads();
    return here ? of_group[group] : Pair{0, 0};
}

// Neighbouring runs of one image go to the same XCD at the same time: they share
// cache lines.
struct HeldPlace {
    int run, stride;
    __device__ __forceinline__ HeldPlace(const Held &h) {
        const uint32_t per = gridDim.x >> 3, more = gridDim.x & 7, xcd = blockIdx.x & 7;
        const uint32_t at = xcd * per + min(xcd, more) + (blockIdx.x >> 3);
        run = at % h.runs;
        stride = at / h.runs;
    }
};

constexpr int kHeldThreads = 512;

template <typename T, int V, int I, int ACT>
__global__ __launch_bounds__(kHeldThreads) void held_forward_kernel(GroupNorm a, Held h) {
    extern __shared__ double2 sums[];
    double2 *sums_of_group = sums + blockDim.x;
    const HeldPlace at(h);
    const int per = a.channels / a.groups, each = per / V, v = threadIdx.x % h.across, r = threadIdx.x / h.across;
    const int group = v / each, c = at.run * h.groups * per + v * V;
    const bool here = r < h.high;
    const int last = (int)a.points - 1;
    const double share = 1.0 / ((double)a.points * per);
    float gamma[V], beta[V];
    load_parameters<V>(a.gamma ? a.gamma + c : nullptr, 1.f, gamma);
    load_parameters<V>(a.beta ? a.beta + c : nullptr, 0.f, beta);
    for (int64_t image = at.stride; image < a.images; image += h.strides) {
        const T *x = (const T *)a.x + image * a.points * a.ldx + c;
        const double pivot = load_value(x + group * per - v * V);        // the group's first
        typename Values<T, V>::Held w[I];
#pragma unroll
        for (int i = 0; i < I; ++i) {
            // (the last point again where there is none: left out of the sums)
            const int point = min(r + i * h.high, last);
            w[i] = Values<T, V>::hold(x + (int64_t)point * a.ldx);
        }
        Moments m;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            Moments o;
            float v[V];
            Values<T, V>::values(w[i], v);
#pragma unroll
            for (int e = 0; e < V; ++e)
                o.add(v[e], pivot);
            const bool in = here && r + i * h.high <= last;
            m.sum += in ? o.sum : 0;
            m.squares += in ? o.squares : 0;
        }
        const double2 all = join_groups(double2{m.sum, m.squares}, h, each, group, here, sums, sums_of_group);
        m.sum = all.x;
        m.squares = all.y;
        const float mean = (float)(pivot + m.sum * share), rstd = reciprocal_root(m.variance(share) + a.eps);
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int point = r + i * h.high;
            if (here && point <= last) {
                if constexpr (V == 8)
                    asm volatile("" : "+v"(w[i]));         // taken apart again: as floats they took twice the registers throughout
                float v[V];
                Values<T, V>::values(w[i], v);
#pragma unroll
                for (int e = 0; e < V; ++e)
                    v[e] = activation<ACT>(__builtin_fmaf(v[e] - mean, rstd * gamma[e], beta[e]));
                Values<T, V>::store_past((T *)a.y + (image * a.points + point) * a.ldy + c, v);
            }
        }
        if (a.mean && here && r == 0 && v % each == 0) {
            a.mean[image * a.groups + at.run * h.groups + group] = mean;
            a.rstd[image * a.groups + at.run * h.groups + group] = rstd;
        }
    }
}

// part: [stride][2][channel]
template <typename T, int V, int I, int ACT>
__global__ __launch_bounds__(kHeldThreads) void held_backward_kernel(GroupNorm a, Held h, float *part) {
    extern __shared__ float2 of[];
    float2 *of_group = of + blockDim.x;
    const HeldPlace at(h);
    const int per = a.channels / a.groups, each = per / V, v = threadIdx.x % h.across, r = threadIdx.x / h.across;
    const int group = v / each, c = at.run * h.groups * per + v * V;
    const bool here = r < h.high;
    const int last = (int)a.points - 1;
    const float share = 1.f / ((float)a.points * per);
    float gamma[V], beta[V];
    Total<V> s1[V], s2[V];
    load_parameters<V>(a.gamma ? a.gamma + c : nullptr, 1.f, gamma);
    load_parameters<V>(a.beta ? a.beta + c : nullptr, 0.f, beta);
#pragma unroll
    for (int e = 0; e < V; ++e) {
        beta[e] *= kUnit<ACT>;
        s1[e] = s2[e] = 0;
    }
    for (int64_t image = at.stride; image < a.images; image += h.strides) {
        const int64_t row0 = image * a.points, unit = image * a.groups + at.run * h.groups + group;
        const float mean = a.mean[unit], rstd = a.rstd[unit];
        // x's words stay as they are until the second use, with g beside them
        typename Values<T, V>::Held x[I];
        float gg[I][V], t = 0, u = 0, b1[V], b2[V], slope[V];
#pragma unroll
        for (int i = 0; i < I; ++i) {
            // (the last point again where there is none: left out of the sums)
            const int point = min(r + i * h.high, last);
            x[i] = Values<T, V>::hold((const T *)a.x + (row0 + point) * a.ldx + c);
            Values<T, V>::load((const T *)a.dy + (row0 + point) * a.lddy + c, gg[i]);
        }
#pragma unroll
        for (int e = 0; e < V; ++e) {
            b1[e] = b2[e] = 0;
            slope[e] = rstd * gamma[e] * kUnit<ACT>;
        }
#pragma unroll
        for (int i = 0; i < I; ++i)
            if (here && r + i * h.high <= last) {
                float xs[V];
                Values<T, V>::values(x[i], xs);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float d = xs[e] - mean;
                    gg[i][e] = activation_gradient<ACT>(gg[i][e], __builtin_fmaf(d, slope[e], beta[e]));
                    b1[e] += gg[i][e];
                    b2[e] = __builtin_fmaf(gg[i][e], d, b2[e]);
                }
            }
#pragma unroll
        for (int e = 0; e < V; ++e) {
            b2[e] *= rstd;
            s1[e] += b1[e];
            s2[e] += b2[e];
            t = __builtin_fmaf(gamma[e], b1[e], t);
            u = __builtin_fmaf(gamma[e], b2[e], u);
        }
        if (!a.y)
            continue;
        // dx = g gamma rstd - (x - mean) rstd^2 m2 - rstd m1
        const float2 m = join_groups(float2{t, u}, h, each, group, here, of, of_group);
        const float m1 = -rstd * (m.x * share), m2 = -rstd * (rstd * (m.y * share));
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int point = r + i * h.high;
            if (here && point <= last) {
                float xs[V];
                Values<T, V>::values(x[i], xs);
#pragma unroll
                for (int e = 0; e < V; ++e)
                    xs[e] = __builtin_fmaf(gg[i][e], rstd * gamma[e], __builtin_fmaf(xs[e] - mean, m2, m1));
                Values<T, V>::store((T *)a.y + (row0 + point) * a.ldy + c, xs);
            }
        }
    }
    if (!a.dgamma && !a.dbeta)
        return;
    float *to = part + (int64_t)at.stride * 2 * a.channels;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        float2 t = {(float)s1[e], (float)s2[e]};
        __syncthreads();
        of[threadIdx.x] = t;
        for (int n = h.high, half; n > 1; n = half) {
            half = (n + 1) / 2;
            __syncthreads();
            if (r < n - half) {
                const float2 o = of[threadIdx.x + half * h.across];
                t.x += o.x;
                t.y += o.y;
                of[threadIdx.x] = t;
            }
        }
        if (r == 0) {
            to[c + e] = t.x;
            to[a.channels + c + e] = t.y;
        }
    }
}

struct HeldPlan {
    Held h;
    int v, each;             // channels of a vector; points of a thread
    int threads;
    uint32_t grid;
};
// Whether a group of an image fits: neighbouring groups until a point's part is
// kLine bytes, a cache line, as far as they fit; at most eight points a thread.
// With kLine 64, 128 and 256, forward and SiLU's gradients in us: 4096 images of 64
// points x 256 channels in bf16, 32 groups, 72 and 115, 52 and 104, 47 and 96; 2048
// of 196 x 96 in fp32, 24 groups, 72 and 112, 56 and 101, 70 and 128; a group at a
// time (327 and 198 us of gradients) is the slowest.
bool held_plan(int32_t dtype, int64_t images, int64_t points, int32_t channels, int32_t groups, HeldPlan *o) {
    constexpr int kLine = 128;
    const int per = channels / groups, size = dtype == HPACML_BF16 ? 2 : 4;
    o->v = size == 2 && per % 8 == 0 ? 8 : per % 4 == 0 ? 4 : 1;
    const int64_t most = (int64_t)kHeldThreads * 8;
    if (points > most || points * (per / o->v) > most)
        return false;
    int run = 1;
    for (int k = 1; k <= groups && points * k * (per / o->v) <= most && k * (per / o->v) <= kHeldThreads; ++k)
        if (groups % k == 0) {
            run = k;
            if (k * per * size >= kLine)
                break;
        }
    o->h.groups = run;
    o->h.across = run * (per / o->v);
    if (o->h.across > kHeldThreads)
        return false;
    // the fewest threads of 256, 512 with at most eight points each
    for (o->threads = 256; o->threads <= kHeldThreads; o->threads *= 2) {
        o->h.high = o->threads / o->h.across;
        if (o->h.high > 0 && (points + o->h.high - 1) / o->h.high <= 8)
            break;
    }
    if (o->threads > kHeldThreads)
        return false;
    if (o->h.high > points)
        o->h.high = (int32_t)points;
    const int64_t each = (points + o->h.high - 1) / o->h.high;
    o->each = each <= 2 ? 2 : each <= 4 ? 4 : 8;
    o->h.runs = groups / run;
    const int64_t want = 256 * 2048 / o->threads / o->h.runs + 1;
    o->h.strides = (int32_t)(images < want ? images : want);
    o->grid = (uint32_t)(o->h.strides * o->h.runs);
    return true;
}

template <typename T, int V, int I>
hipError_t launch_held(const GroupNorm &a, const HeldPlan &o, bool backward, hipStream_t stream) {
    const size_t pairs = (size_t)(o.threads + o.h.groups), lds = pairs * sizeof(float2);
    if (!backward)
        return with_activation(a.act, [&](auto act) {
            held_forward_kernel<T, V, I, decltype(act)::value><<<o.grid, o.threads, pairs * sizeof(double2), stream>>>(a, o.h);
            return hipGetLastError();
        });
    float *part = (float *)a.scratch, *room = part + (int64_t)o.h.strides * 2 * a.channels;
    const hipError_t e = with_activation(a.act, [&](auto act) {
        held_backward_kernel<T, V, I, decltype(act)::value><<<o.grid, o.threads, lds, stream>>>(a, o.h, part);
        return hipGetLastError();
    });
    return e == hipSuccess ? launch_parameters(a, part, o.h.strides, room, stream) : e;
}
template <typename T, int V>
hipError_t launch_held(const GroupNorm &a, const HeldPlan &o, bool backward, hipStream_t stream) {
    return o.each == 2 ? launch_held<T, V, 2>(a, o, backward, stream)
           : o.each == 4 ? launch_held<T, V, 4>(a, o, backward, stream) : launch_held<T, V, 8>(a, o, backward, stream);
}

}  // namespace

int64_t norm_held_scratch(int32_t dtype, int64_t images, int64_t points, int32_t channels, int32_t groups, bool backward) {
    HeldPlan o;
    if (!held_plan(dtype, images, points, channels, groups, &o))
        return -1;
    return backward ? ((int64_t)o.h.strides * 2 * channels + column_sums_room(o.h.strides, 2 * channels)) * 4 : 0;
}

hipError_t launch_norm_held(const GroupNorm &a, int32_t dtype, bool backward, hipStream_t stream) {
    HeldPlan o;
    held_plan(dtype, a.images, a.points, a.channels, a.groups, &o);
    if (dtype == HPACML_F32)
        return o.v == 4 ? launch_held<float, 4>(a, o, backward, stream) : launch_held<float, 1>(a, o, backward, stream);
    return o.v == 8   ? launch_held<uint16_t, 8>(a, o, backward, stream)
           : o.v == 4 ? launch_held<uint16_t, 4>(a, o, backward, stream)
                      : launch_held<uint16_t, 1>(a, o, backward, stream);
}

}  // namespace hpacml
