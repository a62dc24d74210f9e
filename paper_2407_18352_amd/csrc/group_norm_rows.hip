// Group norm of images of one point: in one launch, in registers.  Memory bounds
// it: 65,536 x 512 in bf16, 16 groups, takes 34 us (3.9 TB/s; 32 with sums in 32 bits,
// which were wrong far from zero), in fp32 58 (4.6 TB/s).  Results go through the
// caches: past them it took 24 us, but the next call finds nothing there, and the two
// together took 57 us instead of 52.  Its gradients with SiLU take 54-56 us, in fp32 89.
#include "group_norm_device.hpp"

namespace hpacml {

namespace {

// ---- images of one point ------------------------------------------------------------

// L lanes (a power of two) hold a group of a row, I vectors of V channels each;
// a wave has 64 / L neighbouring groups, or all groups of as many rows as it has
// room for, and goes from row to row, so that a lane's channels stay the same.
constexpr int kRowWaves = 8;
struct Rows {
    int32_t lanes, vectors, column_blocks;     // L; of a group; waves that a row takes
    int32_t rows;                              // of a wave at a time
    int32_t strides;                           // blocks of the same groups
};

template <typename T, int V, int I>
struct RowLane {
    int group, lane, sub;                      // sub: its row among the wave's
    bool here[I];
    int c[I];
    float gamma[I][V], beta[I][V];
    __device__ __forceinline__ RowLane(const GroupNorm &a, const Rows &p, int column_block) {
        const int per = a.channels / a.groups, l = threadIdx.x & 63;
        const int slot = l / p.lanes;
        sub = p.column_blocks > 1 ? 0 : slot / a.groups;
        group = p.column_blocks > 1 ? column_block * (64 / p.lanes) + slot : slot % a.groups;
        lane = l % p.lanes;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int v = lane + i * p.lanes;
            here[i] = sub < p.rows && group < a.groups && v < p.vectors;
            c[i] = here[i] ? group * per + v * V : 0;
        }
        if (a.gamma)
#pragma unroll
            for (int i = 0; i < I; ++i)
                load_parameters<V>(a.gamma + c[i], 1.f, gamma[i]);
        else
#pragma unroll
            for (int i = 0; i < I; ++i)
                load_parameters<V>(nullptr, 1.f, gamma[i]);
        if (a.beta)
#pragma unroll
            for (int i = 0; i < I; ++i)
                load_parameters<V>(a.beta + c[i], 0.f, beta[i]);
        else
#pragma unroll
            for (int i = 0; i < I; ++i)
                load_parameters<V>(nullptr, 0.f, beta[i]);
    }
    __device__ __forceinline__ void load(const T *row, float (&v)[I][V]) const {
#pragma unroll
        for (int i = 0; i < I; ++i) {
            Values<T, V>::load(row + c[i], v[i]);      // of channel 0 where there is none: left out of the sums
        }
    }
};

// (With the compiler's own choice of registers bf16 in whole vectors had two blocks a
// CU instead of three: 65,536 x 512 38 us.)
template <typename T, int V, int I, int ACT>
__global__ __launch_bounds__(64 * kRowWaves, V == 8 && I == 1 ? 6 : 1) void rows_forward_kernel(GroupNorm a, Rows p) {
    const int column_block = blockIdx.x % p.column_blocks, wave = threadIdx.x >> 6;
    const RowLane<T, V, I> k(a, p, column_block);
    const double share = 1.0 / (a.channels / a.groups);
    constexpr int kAtOnce = V * I <= 16 ? 2 : 1;     // rows whose loads go out together
    const int64_t step = (int64_t)p.strides * kRowWaves * p.rows;
    for (int64_t first = ((int64_t)(blockIdx.x / p.column_blocks) * kRowWaves + wave) * p.rows; first < a.images; first += step * kAtOnce) {
        typename Values<T, V>::Held w[kAtOnce][I];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
            for (int i = 0; i < I; ++i)        // of channel 0 where there is none: left out of the sums
                w[u][i] = Values<T, V>::hold((const T *)a.x + min(first + u * step + k.sub, a.images - 1) * a.ldx + k.c[i]);
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int64_t row = first + u * step + k.sub;
            float v[I][V];
#pragma unroll
            for (int i = 0; i < I; ++i)
                Values<T, V>::values(w[u][i], v[i]);
            const double pivot = __shfl(v[0][0], (threadIdx.x & 63) & -p.lanes);
            Moments m;
#pragma unroll
            for (int i = 0; i < I; ++i) {
                Moments o;
#pragma unroll
                for (int e = 0; e < V; ++e)
                    o.add(v[i][e], pivot);
                m.sum += k.here[i] ? o.sum : 0;
                m.squares += k.here[i] ? o.squares : 0;
            }
            m.sum = join_lanes(m.sum, p.lanes);
            m.squares = join_lanes(m.squares, p.lanes);
            const float mean = (float)(pivot + m.sum * share), rstd = reciprocal_root(m.variance(share) + a.eps);
            const bool live = row < a.images;
#pragma unroll
            for (int i = 0; i < I; ++i)
                if (live && k.here[i]) {
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        v[i][e] = activation<ACT>(__builtin_fmaf(v[i][e] - mean, rstd * k.gamma[i][e], k.beta[i][e]));
                    Values<T, V>::store((T *)a.y + row * a.ldy + k.c[i], v[i]);
                }
            if (a.mean && live && k.lane == 0 && k.here[0]) {
                a.mean[row * a.groups + k.group] = mean;
                a.rstd[row * a.groups + k.group] = rstd;
            }
        }
    }
}

// part: [block of the same groups][2][channel]
template <typename T, int V, int I, int ACT>
__global__ __launch_bounds__(64 * kRowWaves) void rows_backward_kernel(GroupNorm a, Rows p, float *part) {
    __shared__ float2 of[kRowWaves][64][V];
    const int column_block = blockIdx.x % p.column_blocks, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const RowLane<T, V, I> k(a, p, column_block);
    const float share = 1.f / (float)(a.channels / a.groups);
    Total<I * V> s1[I][V], s2[I][V];
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e)
            s1[i][e] = s2[i][e] = 0;
    for (int64_t first = ((int64_t)(blockIdx.x / p.column_blocks) * kRowWaves + wave) * p.rows; first < a.images;
         first += (int64_t)p.strides * kRowWaves * p.rows) {
        // (a lane without a row has the last one again, and leaves it out)
        const bool live = first + k.sub < a.images;
        const int64_t row = min(first + k.sub, a.images - 1);
        float v[I][V], g[I][V], t = 0, u = 0;
        k.load((const T *)a.x + row * a.ldx, v);
        k.load((const T *)a.dy + row * a.lddy, g);
        const int64_t at = row * a.groups + min(k.group, a.groups - 1);
        const float mean = a.mean[at], rstd = a.rstd[at];
#pragma unroll
        for (int i = 0; i < I; ++i) {
            float to = 0, uo = 0;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = v[i][e] - mean;
                const float o = activation_gradient<ACT>(g[i][e], __builtin_fmaf(d, rstd * k.gamma[i][e] * kUnit<ACT>, k.beta[i][e] * kUnit<ACT>));
                v[i][e] = d * rstd;
                s1[i][e] += live ? o : 0.f;
                s2[i][e] += live ? o * v[i][e] : 0.f;
                g[i][e] = o * k.gamma[i][e];
                to += g[i][e];
                uo = __builtin_fmaf(g[i][e], v[i][e], uo);
            }
            t += k.here[i] ? to : 0.f;
            u += k.here[i] ? uo : 0.f;
        }
        if (a.y) {
            const float m1 = join_lanes(t, p.lanes) * share, m2 = join_lanes(u, p.lanes) * share;
#pragma unroll
            for (int i = 0; i < I; ++i)
                if (live && k.here[i]) {
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        v[i][e] = rstd * ((g[i][e] - m1) - v[i][e] * m2);
                    Values<T, V>::store((T *)a.y + row * a.ldy + k.c[i], v[i]);
                }
        }
    }
    if (!a.dgamma && !a.dbeta)
        return;
    float *to = part + (int64_t)(blockIdx.x / p.column_blocks) * 2 * a.channels;
#pragma unroll
    for (int i = 0; i < I; ++i) {
#pragma unroll
        for (int e = 0; e < V; ++e)
            of[wave][lane][e] = {(float)s1[i][e], (float)s2[i][e]};
        __syncthreads();
        if (wave == 0 && k.here[i] && k.sub == 0)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float2 t = {0.f, 0.f};
                for (int r = 0; r < p.rows; ++r)
#pragma unroll
                    for (int w = 0; w < kRowWaves; ++w) {
                        const float2 o = of[w][lane + r * a.groups * p.lanes][e];
                        t.x += o.x;
                        t.y += o.y;
                    }
                to[k.c[i] + e] = t.x;
                to[a.channels + k.c[i] + e] = t.y;
            }
        __syncthreads();
    }
}

struct RowsPlan {
    Rows p;
    int v, each;             // channels of a vector; vectors of a lane
    uint32_t grid;
};
// Whether images of one point have that form.
bool rows_plan(int32_t dtype, int64_t images, int64_t points, int32_t channels, int32_t groups, RowsPlan *o) {
    const int per = channels / groups;
    if (points != 1)
        return false;
    o->v = dtype == HPACML_BF16 && per % 8 == 0 ? 8 : per % 4 == 0 ? 4 : 1;
    o->p.vectors = per / o->v;
    o->p.lanes = 1;
    while (o->p.lanes < 64 && o->p.lanes < o->p.vectors)
        o->p.lanes *= 2;
    o->each = 1;
    while (o->each * o->p.lanes < o->p.vectors)
        o->each *= 2;
    if (o->each > 8 || o->each * o->v > 32)         // a lane's values in registers
        return false;
    const int at_a_time = 64 / o->p.lanes;
    o->p.column_blocks = (groups + at_a_time - 1) / at_a_time;
    o->p.rows = at_a_time / groups < 1 ? 1 : at_a_time / groups;
    const int64_t at_once = (int64_t)kRowWaves * o->p.rows, most = (images + at_once - 1) / at_once, want = 1024 / o->p.column_blocks + 1;
    o->p.strides = (int32_t)(most < want ? most : want);
    o->grid = (uint32_t)(o->p.strides * o->p.column_blocks);
    return true;
}

template <typename T, int V, int I>
hipError_t launch_rows(const GroupNorm &a, const RowsPlan &o, bool backward, hipStream_t stream) {
    if (!backward)
        return with_activation(a.act, [&](auto act) {
            rows_forward_kernel<T, V, I, decltype(act)::value><<<o.grid, 64 * kRowWaves, 0, stream>>>(a, o.p);
            return hipGetLastError();
        });
    float *part = (float *)a.scratch, *room = part + (int64_t)o.p.strides * 2 * a.channels;
    const hipError_t e = with_activation(a.act, [&](auto act) {
        rows_backward_kernel<T, V, I, decltype(act)::value><<<o.grid, 64 * kRowWaves, 0, stream>>>(a, o.p, part);
        return hipGetLastError();
    });
    return e == hipSuccess ? launch_parameters(a, part, o.p.strides, room, stream) : e;
}
template <typename T, int V>
hipError_t launch_rows(const GroupNorm &a, const RowsPlan &o, bool backward, hipStream_t stream) {
    if (o.each == 1)
        return launch_rows<T, V, 1>(a, o, backward, stream);
    if (o.each == 2)
        return launch_rows<T, V, 2>(a, o, backward, stream);
    if constexpr (V < 8)
        if (o.each > 4)
            return launch_rows<T, V, 8>(a, o, backward, stream);
    return launch_rows<T, V, 4>(a, o, backward, stream);
}

}  // namespace

int64_t norm_rows_scratch(int32_t dtype, int64_t images, int64_t points, int32_t channels, int32_t groups, bool backward) {
    RowsPlan o;
    if (!rows_plan(dtype, images, points, channels, groups, &o))
        return -1;
    return backward ? ((int64_t)o.p.strides * 2 * channels + column_sums_room(o.p.strides, 2 * channels)) * 4 : 0;
}

hipError_t launch_norm_rows(const GroupNorm &a, int32_t dtype, bool backward, hipStream_t stream) {
    RowsPlan o;
    rows_plan(dtype, a.images, a.points, a.channels, a.groups, &o);
    if (dtype == HPACML_F32)
        return o.v == 4 ? launch_rows<float, 4>(a, o, backward, stream) : launch_rows<float, 1>(a, o, backward, stream);
    return o.v == 8   ? launch_rows<uint16_t, 8>(a, o, backward, stream)
           : o.v == 4 ? launch_rows<uint16_t, 4>(a, o, backward, stream)
                      : launch_rows<uint16_t, 1>(a, o, backward, stream);
}

}  // namespace hpacml
