// Group norm with an activation, channels last, and its backward pass.
//
// Three forms.  Where an image is one point (a hidden layer's activations), a few
// lanes of a wave hold a group of it in registers: one reading, one launch
// (rows_*).  Where a group of an image fits the registers of a block, the same
// with a block (held_*).  Otherwise three launches (parts_*): sums of every channel over runs
// of an image's points, which a second launch joins to the groups' statistics,
// and the results, from a second reading (of what the first left in the
// Infinity Cache, up to 256 MB).  A thread has the same few neighbouring
// channels throughout, so that their parameters are in registers, and the sums
// that the parameters' gradients are made of stay apart until the end.
//
// Statistics: the mean of a few values in registers, the squares about it, and
// pairs of (mean, squares) joined as such, so that no difference of large sums
// occurs; joins of many in 64 bits.
#include <type_traits>

#include "columns.hpp"
#include "dense8.hpp"
#include "group_norm.hpp"
#include "hpacmlt.h"

namespace hpacml {

namespace {

// By the exponential's and the reciprocal's own instructions: z log2(e) is
// rounded to 2^-24 of itself, which moves the result by |z| 2^-24 (1 - result) of
// it, less than the roundings around it, and the square of a SiLU's slope takes
// five instructions a value where expf and a division take thirty: the backward
// pass of 134 million values is bound by memory so, not by its arithmetic.
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504088896f)); }

__device__ __forceinline__ float activation(float z, int32_t act) {
    if (act == HPACML_ACT_RELU)
        return relu_keep_nan(z);
    return act == HPACMLT_ACT_SILU ? z * sigmoid(z) : z;
}
// g = dy act'(z)
__device__ __forceinline__ float activation_gradient(float dy, float z, int32_t act) {
    if (act == HPACML_ACT_RELU)
        return z <= 0.f ? 0.f : dy;
    if (act == HPACMLT_ACT_SILU) {
        const float s = sigmoid(z);
        return dy * (s * (1.f + z * (1.f - s)));
    }
    return dy;
}

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
    static __device__ __forceinline__ void store(T *p, const float (&v)[V]) {
        if constexpr (V == 1)
            store_value(p, v[0]);
        else {
            Word w;
#pragma unroll
            for (int e = 0; e < kBytes / 4; ++e) {
                if constexpr (sizeof(T) == 4)
                    w[e] = __builtin_bit_cast(uint32_t, v[e]);
                else
                    w[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
            }
            *(Any *)p = w;
        }
    }
};

// ---- parts of an image ------------------------------------------------------------

// A block takes `run` points of an image and up to 256 vectors of V channels,
// `high` (a power of two) points at a time.
struct Parts {
    int32_t vectors, across, high;       // of a row; of a block; points at a time
    uint32_t column_tiles, runs;         // of a row, of an image
    int64_t run, blocks;                 // points; of all images
};

struct Place {
    int64_t image, first, last;          // points of the record
    int c, r;                            // the thread's first channel, its point
    bool here;
};
template <int V>
__device__ __forceinline__ Place place_of(const GroupNorm &a, const Parts &p, int64_t block) {
    Place q;
    const int64_t i = block / p.column_tiles;
    const int tile = (int)(block % p.column_tiles);
    q.image = i / p.runs;
    const int64_t at = (int64_t)(i % p.runs) * p.run;
    q.first = q.image * a.points + at;
    q.last = q.image * a.points + min(at + p.run, a.points);
    q.r = threadIdx.x / p.across;
    const int v = tile * p.across + threadIdx.x % p.across;
    q.c = v * V;
    q.here = q.r < p.high && v < p.vectors;
    return q;
}

// (mean, squares about it) of n values and of m: of both
__device__ __forceinline__ void join_moments(float &mean, float &squares, float n, float mean2, float squares2, float m) {
    const float d = mean2 - mean, share = m / (n + m);
    mean += d * share;
    squares += squares2 + d * d * (n * share);
}

// [image][run][channel] (mean, squares)
template <typename T, int V>
__global__ __launch_bounds__(256) void parts_moments_kernel(GroupNorm a, Parts p, float2 *part) {
    constexpr int kBatch = 8;
    __shared__ float2 of[256][V];
    for (int64_t block = blockIdx.x; block < p.blocks; block += gridDim.x) {
        const Place q = place_of<V>(a, p, block);
        float mean[V], squares[V], n = 0;
#pragma unroll
        for (int e = 0; e < V; ++e)
            mean[e] = squares[e] = 0;
        if (q.here) {
            const T *x = (const T *)a.x + q.c;
            int64_t row = q.first + q.r;
            for (; row + (kBatch - 1) * p.high < q.last; row += kBatch * p.high) {
                float v[kBatch][V];
#pragma unroll
                for (int b = 0; b < kBatch; ++b)
                    Values<T, V>::load(x + (row + b * p.high) * a.ldx, v[b]);
                const float share = kBatch / (n + kBatch), weight = n * share;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float t = 0, s = 0;
#pragma unroll
                    for (int b = 0; b < kBatch; ++b)
                        t += v[b][e];
                    t *= 1.f / kBatch;
#pragma unroll
                    for (int b = 0; b < kBatch; ++b)
                        s = __builtin_fmaf(v[b][e] - t, v[b][e] - t, s);
                    const float d = t - mean[e];
                    mean[e] += d * share;
                    squares[e] += s + d * d * weight;
                }
                n += kBatch;
            }
            for (; row < q.last; row += p.high) {
                float v[V];
                Values<T, V>::load(x + row * a.ldx, v);
#pragma unroll
                for (int e = 0; e < V; ++e)
                    join_moments(mean[e], squares[e], n, v[e], 0.f, 1.f);
                n += 1;
            }
        }
#pragma unroll
        for (int e = 0; e < V; ++e)
            of[threadIdx.x][e] = {mean[e], squares[e]};
        // threads' points: every `high`-th from r on; joined in halves
        for (int h = p.high / 2; h > 0; h /= 2) {
            __syncthreads();
            const int rows = (int)(q.last - q.first);
            auto count = [&](int r) {         // values of the threads r, r + 2 h, ... that r has joined
                const int step = 2 * h;
                int t = 0;
                if (rows > r)
                    t = (rows - r + step - 1) / step;
                return (float)t;
            };
            if (q.here && q.r < h) {
                const float m = count(q.r + h);
                n = count(q.r);
                if (m > 0)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float2 o = of[threadIdx.x + h * p.across][e];
                        join_moments(mean[e], squares[e], n, o.x, o.y, m);
                        of[threadIdx.x][e] = {mean[e], squares[e]};
                    }
            }
        }
        if (q.here && q.r == 0) {
            float2 *to = part + (block / p.column_tiles) * (int64_t)a.channels + q.c;
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (q.c + e < a.channels)
                    to[e] = {mean[e], squares[e]};
        }
        __syncthreads();
    }
}

__device__ __forceinline__ double join_block(double t, double (&of_wave)[4]) {
#pragma unroll
    for (int s = 1; s < 64; s *= 2)
        t += __shfl_xor(t, s);
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        of_wave[threadIdx.x >> 6] = t;
    __syncthreads();
    return (of_wave[0] + of_wave[1]) + (of_wave[2] + of_wave[3]);
}

// The partial results of an image's group, `per` channels of each run: a thread
// takes every so many runs of one channel (with one index over all of them, and
// its divisions, 2049 runs of 4 channels took 23 us).
template <typename F>
__device__ __forceinline__ void over_runs(int per, uint32_t runs, F f) {
    const int across = min(per, 256), high = 256 / across, c0 = threadIdx.x % across, r0 = threadIdx.x / across;
    if (r0 < high)
        for (int c = c0; c < per; c += across)
#pragma unroll 4
            for (uint32_t r = r0; r < runs; r += high)
                f(c, r);
}

// A block per image and group: mean and rstd.
__global__ __launch_bounds__(256) void parts_join_kernel(GroupNorm a, Parts p, const float2 *part, float *mean_to, float *rstd_to) {
    __shared__ double of_wave[4];
    for (int64_t unit = blockIdx.x; unit < a.images * a.groups; unit += gridDim.x) {
        const int64_t image = unit / a.groups;
        const int per = a.channels / a.groups, c0 = (int)(unit % a.groups) * per;
        const float2 *at = part + image * p.runs * a.channels + c0;
        auto values = [&](uint32_t r) { return (double)min(p.run, a.points - r * p.run); };
        double t = 0;
        over_runs(per, p.runs, [&](int c, uint32_t r) { t += values(r) * at[(int64_t)r * a.channels + c].x; });
        const double n = (double)a.points * per, mean = join_block(t, of_wave) / n;
        t = 0;
        over_runs(per, p.runs, [&](int c, uint32_t r) {
            const float2 o = at[(int64_t)r * a.channels + c];
            t += (double)o.y + values(r) * (o.x - mean) * (o.x - mean);
        });
        t = join_block(t, of_wave);
        if (threadIdx.x == 0) {
            mean_to[unit] = (float)mean;
            rstd_to[unit] = (float)(1.0 / sqrt(t / n + (double)a.eps));
        }
    }
}

// The parameters of a thread's channels.
template <int V>
struct Channels {
    float mean[V], rstd[V], gamma[V], beta[V];
    __device__ __forceinline__ void load(const GroupNorm &a, int64_t image, int c, const float *means, const float *rstds) {
        const int per = a.channels / a.groups;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int ce = min(c + e, a.channels - 1);
            const int64_t at = image * a.groups + ce / per;
            mean[e] = means[at];
            rstd[e] = rstds[at];
            gamma[e] = a.gamma ? a.gamma[ce] : 1.f;
            beta[e] = a.beta ? a.beta[ce] : 0.f;
        }
    }
};

template <typename T, int V>
__global__ __launch_bounds__(256) void parts_apply_kernel(GroupNorm a, Parts p, const float *means, const float *rstds) {
    for (int64_t block = blockIdx.x; block < p.blocks; block += gridDim.x) {
        const Place q = place_of<V>(a, p, block);
        if (!q.here)
            continue;
        Channels<V> k;
        k.load(a, q.image, q.c, means, rstds);
#pragma unroll
        for (int e = 0; e < V; ++e)
            k.gamma[e] *= k.rstd[e];
#pragma unroll 4
        for (int64_t row = q.first + q.r; row < q.last; row += p.high) {
            float v[V];
            Values<T, V>::load((const T *)a.x + row * a.ldx + q.c, v);
#pragma unroll
            for (int e = 0; e < V; ++e)
                v[e] = activation(__builtin_fmaf(v[e] - k.mean[e], k.gamma[e], k.beta[e]), a.act);
            Values<T, V>::store((T *)a.y + row * a.ldy + q.c, v);
        }
    }
}

// sums of g and of g (x - mean) rstd: [image][run][2][channel]
template <typename T, int V>
__global__ __launch_bounds__(256) void parts_sums_kernel(GroupNorm a, Parts p, float *part) {
    __shared__ float2 of[256][V];
    for (int64_t block = blockIdx.x; block < p.blocks; block += gridDim.x) {
        const Place q = place_of<V>(a, p, block);
        float s1[V], s2[V];
#pragma unroll
        for (int e = 0; e < V; ++e)
            s1[e] = s2[e] = 0;
        Channels<V> k;
        if (q.here) {
            k.load(a, q.image, q.c, a.mean, a.rstd);
#pragma unroll 4
            for (int64_t row = q.first + q.r; row < q.last; row += p.high) {
                float v[V], g[V];
                Values<T, V>::load((const T *)a.x + row * a.ldx + q.c, v);
                Values<T, V>::load((const T *)a.dy + row * a.lddy + q.c, g);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float d = v[e] - k.mean[e];
                    const float t = activation_gradient(g[e], __builtin_fmaf(d, k.rstd[e] * k.gamma[e], k.beta[e]), a.act);
                    s1[e] += t;
                    s2[e] = __builtin_fmaf(t, d, s2[e]);
                }
            }
        }
#pragma unroll
        for (int e = 0; e < V; ++e)
            of[threadIdx.x][e] = {s1[e], s2[e]};
        for (int h = p.high / 2; h > 0; h /= 2) {
            __syncthreads();
            if (q.here && q.r < h)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float2 o = of[threadIdx.x + h * p.across][e];
                    s1[e] += o.x;
                    s2[e] += o.y;
                    of[threadIdx.x][e] = {s1[e], s2[e]};
                }
        }
        if (q.here && q.r == 0) {
            float *to = part + (block / p.column_tiles) * (int64_t)(2 * a.channels) + q.c;
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (q.c + e < a.channels) {
                    to[e] = s1[e];
                    to[a.channels + e] = s2[e] * k.rstd[e];
                }
        }
        __syncthreads();
    }
}

// A block per image and group: the means of g gamma and g gamma (x - mean) rstd.
__global__ __launch_bounds__(256) void parts_means_kernel(GroupNorm a, Parts p, const float *part, float2 *means) {
    __shared__ double of_wave[4];
    for (int64_t unit = blockIdx.x; unit < a.images * a.groups; unit += gridDim.x) {
        const int64_t image = unit / a.groups;
        const int per = a.channels / a.groups, c0 = (int)(unit % a.groups) * per;
        const float *at = part + image * p.runs * 2 * a.channels + c0;
        double t = 0, u = 0;
        over_runs(per, p.runs, [&](int c, uint32_t r) {
            const float *o = at + (int64_t)r * 2 * a.channels + c;
            const double gamma = a.gamma ? a.gamma[c0 + c] : 1.f;
            t += gamma * o[0];
            u += gamma * o[a.channels];
        });
        const double n = (double)a.points * per;
        t = join_block(t, of_wave) / n;
        u = join_block(u, of_wave) / n;
        if (threadIdx.x == 0)
            means[unit] = {(float)t, (float)u};
    }
}

template <typename T, int V>
__global__ __launch_bounds__(256) void parts_dx_kernel(GroupNorm a, Parts p, const float2 *means) {
    for (int64_t block = blockIdx.x; block < p.blocks; block += gridDim.x) {
        const Place q = place_of<V>(a, p, block);
        if (!q.here)
            continue;
        Channels<V> k;
        k.load(a, q.image, q.c, a.mean, a.rstd);
        float m1[V], m2[V];
        const int per = a.channels / a.groups;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float2 m = means[q.image * a.groups + min(q.c + e, a.channels - 1) / per];
            m1[e] = m.x;
            m2[e] = m.y;
        }
#pragma unroll 4
        for (int64_t row = q.first + q.r; row < q.last; row += p.high) {
            float v[V], g[V];
            Values<T, V>::load((const T *)a.x + row * a.ldx + q.c, v);
            Values<T, V>::load((const T *)a.dy + row * a.lddy + q.c, g);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = v[e] - k.mean[e];
                const float t = activation_gradient(g[e], __builtin_fmaf(d, k.rstd[e] * k.gamma[e], k.beta[e]), a.act) * k.gamma[e];
                v[e] = k.rstd[e] * ((t - m1[e]) - d * k.rstd[e] * m2[e]);
            }
            Values<T, V>::store((T *)a.y + row * a.ldy + q.c, v);
        }
    }
}

// dbeta and dgamma from rows of partial sums, [2][channels] each
hipError_t launch_parameters(const GroupNorm &a, const float *part, int64_t rows, float *room, hipStream_t stream) {
    if (!a.dgamma && !a.dbeta)
        return hipSuccess;
    return launch_column_sums({part, rows, 2 * a.channels, 2 * a.channels, a.dbeta, a.dgamma, a.channels, a.accumulate, room}, stream);
}

// ---- images of one point ------------------------------------------------------------

// L lanes (a power of two) hold a group of a row, I vectors of V channels each;
// a wave has 64 / L neighbouring groups and goes from row to row, so that a
// lane's channels stay the same.
constexpr int kRowWaves = 8;
struct Rows {
    int32_t lanes, vectors, column_blocks;     // L; of a group; waves that a row takes
    int32_t strides;                           // blocks of the same groups
};

template <int L_MOST>
__device__ __forceinline__ float join_lanes(float t, int lanes) {
#pragma unroll
    for (int s = 1; s < L_MOST; s *= 2)
        if (s < lanes)
            t += __shfl_xor(t, s);
    return t;
}

template <typename T, int V, int I>
struct RowLane {
    int group, lane;
    bool here[I];
    int c[I];
    float gamma[I][V], beta[I][V];
    __device__ __forceinline__ RowLane(const GroupNorm &a, const Rows &p, int column_block) {
        const int per = a.channels / a.groups, l = threadIdx.x & 63;
        group = column_block * (64 / p.lanes) + l / p.lanes;
        lane = l % p.lanes;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int v = lane + i * p.lanes;
            here[i] = group < a.groups && v < p.vectors;
            c[i] = here[i] ? group * per + v * V : 0;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                gamma[i][e] = a.gamma ? a.gamma[c[i] + e] : 1.f;
                beta[i][e] = a.beta ? a.beta[c[i] + e] : 0.f;
            }
        }
    }
    __device__ __forceinline__ void load(const T *row, float (&v)[I][V]) const {
#pragma unroll
        for (int i = 0; i < I; ++i) {
            Values<T, V>::load(row + c[i], v[i]);
            if (!here[i])
#pragma unroll
                for (int e = 0; e < V; ++e)
                    v[i][e] = 0.f;
        }
    }
};

template <typename T, int V, int I>
__global__ __launch_bounds__(64 * kRowWaves) void rows_forward_kernel(GroupNorm a, Rows p) {
    const int column_block = blockIdx.x % p.column_blocks, wave = threadIdx.x >> 6;
    const RowLane<T, V, I> k(a, p, column_block);
    const float share = 1.f / (float)(a.channels / a.groups);
    constexpr int kAtOnce = V * I <= 8 ? 4 : V * I <= 16 ? 2 : 1;     // rows whose loads go out together
    const int64_t step = (int64_t)p.strides * kRowWaves;
    for (int64_t first = (int64_t)(blockIdx.x / p.column_blocks) * kRowWaves + wave; first < a.images; first += step * kAtOnce) {
        float v[kAtOnce][I][V];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
            k.load((const T *)a.x + min(first + u * step, a.images - 1) * a.ldx, v[u]);
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int64_t row = first + u * step;
            float t = 0, s = 0;
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e)
                    t += v[u][i][e];
            const float mean = join_lanes<64>(t, p.lanes) * share;
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    v[u][i][e] -= mean;
                    s = k.here[i] ? __builtin_fmaf(v[u][i][e], v[u][i][e], s) : s;
                }
            const float rstd = 1.f / sqrtf(join_lanes<64>(s, p.lanes) * share + a.eps);
            if (row >= a.images)
                continue;
#pragma unroll
            for (int i = 0; i < I; ++i)
                if (k.here[i]) {
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        v[u][i][e] = activation(__builtin_fmaf(v[u][i][e], rstd * k.gamma[i][e], k.beta[i][e]), a.act);
                    Values<T, V>::store((T *)a.y + row * a.ldy + k.c[i], v[u][i]);
                }
            if (a.mean && k.lane == 0 && k.here[0]) {
                a.mean[row * a.groups + k.group] = mean;
                a.rstd[row * a.groups + k.group] = rstd;
            }
        }
    }
}

// part: [block of the same groups][2][channel]
template <typename T, int V, int I>
__global__ __launch_bounds__(64 * kRowWaves) void rows_backward_kernel(GroupNorm a, Rows p, float *part) {
    __shared__ float2 of[kRowWaves][64][V];
    const int column_block = blockIdx.x % p.column_blocks, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const RowLane<T, V, I> k(a, p, column_block);
    const float share = 1.f / (float)(a.channels / a.groups);
    float s1[I][V], s2[I][V];
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e)
            s1[i][e] = s2[i][e] = 0;
    for (int64_t row = (int64_t)(blockIdx.x / p.column_blocks) * kRowWaves + wave; row < a.images; row += (int64_t)p.strides * kRowWaves) {
        float v[I][V], g[I][V], t = 0, u = 0;
        k.load((const T *)a.x + row * a.ldx, v);
        k.load((const T *)a.dy + row * a.lddy, g);
        const int64_t at = row * a.groups + min(k.group, a.groups - 1);
        const float mean = a.mean[at], rstd = a.rstd[at];
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = v[i][e] - mean;
                const float o = activation_gradient(g[i][e], __builtin_fmaf(d, rstd * k.gamma[i][e], k.beta[i][e]), a.act);
                v[i][e] = d * rstd;
                s1[i][e] += k.here[i] ? o : 0.f;
                s2[i][e] += k.here[i] ? o * v[i][e] : 0.f;
                g[i][e] = o * k.gamma[i][e];
                t += k.here[i] ? g[i][e] : 0.f;
                u += k.here[i] ? g[i][e] * v[i][e] : 0.f;
            }
        if (a.y) {
            const float m1 = join_lanes<64>(t, p.lanes) * share, m2 = join_lanes<64>(u, p.lanes) * share;
#pragma unroll
            for (int i = 0; i < I; ++i)
                if (k.here[i]) {
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
            of[wave][lane][e] = {s1[i][e], s2[i][e]};
        __syncthreads();
        if (wave == 0 && k.here[i])
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float2 t = of[0][lane][e];
#pragma unroll
                for (int w = 1; w < kRowWaves; ++w) {
                    t.x += of[w][lane][e].x;
                    t.y += of[w][lane][e].y;
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
    const int64_t most = (images + kRowWaves - 1) / kRowWaves, want = 1024 / o->p.column_blocks + 1;
    o->p.strides = (int32_t)(most < want ? most : want);
    o->grid = (uint32_t)(o->p.strides * o->p.column_blocks);
    return true;
}

template <typename T, int V, int I>
hipError_t launch_rows(const GroupNorm &a, const RowsPlan &o, bool backward, hipStream_t stream) {
    if (!backward) {
        rows_forward_kernel<T, V, I><<<o.grid, 64 * kRowWaves, 0, stream>>>(a, o.p);
        return hipGetLastError();
    }
    float *part = (float *)a.scratch, *room = part + (int64_t)o.p.strides * 2 * a.channels;
    rows_backward_kernel<T, V, I><<<o.grid, 64 * kRowWaves, 0, stream>>>(a, o.p, part);
    hipError_t e = hipGetLastError();
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
hipError_t launch_rows(const GroupNorm &a, const RowsPlan &o, int32_t dtype, bool backward, hipStream_t stream) {
    if (dtype == HPACML_F32)
        return o.v == 4 ? launch_rows<float, 4>(a, o, backward, stream) : launch_rows<float, 1>(a, o, backward, stream);
    return o.v == 8 ? launch_rows<uint16_t, 8>(a, o, backward, stream)
           : o.v == 4 ? launch_rows<uint16_t, 4>(a, o, backward, stream) : launch_rows<uint16_t, 1>(a, o, backward, stream);
}

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
__device__ __forceinline__ float2 join_groups(float2 t, const Held &h, int each, int group, bool here, float2 *of, float2 *of_group) {
    __syncthreads();
    of[threadIdx.x] = t;
    __syncthreads();
    const int entries = h.high * each;
    for (int g = threadIdx.x >> 5; g < h.groups; g += blockDim.x >> 5) {
        float2 s = {0.f, 0.f};
        for (int i = threadIdx.x & 31; i < entries; i += 32) {
            const float2 o = of[i / each * h.across + g * each + i % each];
            s.x += o.x;
            s.y += o.y;
        }
#pragma unroll
        for (int x = 1; x < 32; x *= 2) {
            s.x += __shfl_xor(s.x, x);
            s.y += __shfl_xor(s.y, x);
        }
        if ((threadIdx.x & 31) == 0)
            of_group[g] = s;
    }
    __syncthreads();
    return here ? of_group[group] : float2{0.f, 0.f};
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

template <typename T, int V, int I>
__global__ __launch_bounds__(kHeldThreads) void held_forward_kernel(GroupNorm a, Held h) {
    extern __shared__ float2 of[];
    float2 *of_group = of + blockDim.x;
    const HeldPlace at(h);
    const int per = a.channels / a.groups, each = per / V, v = threadIdx.x % h.across, r = threadIdx.x / h.across;
    const int group = v / each, c = at.run * h.groups * per + v * V;
    const bool here = r < h.high;
    const float share = 1.f / ((float)a.points * per);
    float gamma[V], beta[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        gamma[e] = a.gamma ? a.gamma[c + e] : 1.f;
        beta[e] = a.beta ? a.beta[c + e] : 0.f;
    }
    for (int64_t image = at.stride; image < a.images; image += h.strides) {
        const T *x = (const T *)a.x + image * a.points * a.ldx + c;
        float w[I][V], t = 0, s = 0;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int64_t point = r + (int64_t)i * h.high;
            if (here && point < a.points)
                Values<T, V>::load(x + point * a.ldx, w[i]);
            else
#pragma unroll
                for (int e = 0; e < V; ++e)
                    w[i][e] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e)
                t += w[i][e];
        const float mean = join_groups({t, 0.f}, h, each, group, here, of, of_group).x * share;
#pragma unroll
        for (int i = 0; i < I; ++i)
            if (here && r + (int64_t)i * h.high < a.points)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    w[i][e] -= mean;
                    s = __builtin_fmaf(w[i][e], w[i][e], s);
                }
        const float rstd = 1.f / sqrtf(join_groups({s, 0.f}, h, each, group, here, of, of_group).x * share + a.eps);
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int64_t point = r + (int64_t)i * h.high;
            if (here && point < a.points) {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    w[i][e] = activation(__builtin_fmaf(w[i][e], rstd * gamma[e], beta[e]), a.act);
                Values<T, V>::store((T *)a.y + (image * a.points + point) * a.ldy + c, w[i]);
            }
        }
        if (a.mean && here && r == 0 && v % each == 0) {
            a.mean[image * a.groups + at.run * h.groups + group] = mean;
            a.rstd[image * a.groups + at.run * h.groups + group] = rstd;
        }
    }
}

// part: [stride][2][channel]
template <typename T, int V, int I>
__global__ __launch_bounds__(kHeldThreads) void held_backward_kernel(GroupNorm a, Held h, float *part) {
    extern __shared__ float2 of[];
    float2 *of_group = of + blockDim.x;
    const HeldPlace at(h);
    const int per = a.channels / a.groups, each = per / V, v = threadIdx.x % h.across, r = threadIdx.x / h.across;
    const int group = v / each, c = at.run * h.groups * per + v * V;
    const bool here = r < h.high;
    const float share = 1.f / ((float)a.points * per);
    float gamma[V], beta[V], s1[V], s2[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        gamma[e] = a.gamma ? a.gamma[c + e] : 1.f;
        beta[e] = a.beta ? a.beta[c + e] : 0.f;
        s1[e] = s2[e] = 0;
    }
    for (int64_t image = at.stride; image < a.images; image += h.strides) {
        const int64_t row0 = image * a.points, unit = image * a.groups + at.run * h.groups + group;
        const float mean = a.mean[unit], rstd = a.rstd[unit];
        // x's and dy's words stay as they are between the two uses
        typename Values<T, V>::Held x[I], dy[I];
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int64_t point = r + (int64_t)i * h.high;
            if (here && point < a.points) {
                x[i] = Values<T, V>::hold((const T *)a.x + (row0 + point) * a.ldx + c);
                dy[i] = Values<T, V>::hold((const T *)a.dy + (row0 + point) * a.lddy + c);
            }
        }
        auto value = [&](int i, int e, const float (&xs)[V], const float (&gs)[V], float &g, float &d) {
            d = xs[e] - mean;
            g = activation_gradient(gs[e], __builtin_fmaf(d, rstd * gamma[e], beta[e]), a.act);
        };
        float t = 0, u = 0;
#pragma unroll
        for (int i = 0; i < I; ++i)
            if (here && r + (int64_t)i * h.high < a.points) {
                float xs[V], gs[V];
                Values<T, V>::values(x[i], xs);
                Values<T, V>::values(dy[i], gs);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float g, d;
                    value(i, e, xs, gs, g, d);
                    d *= rstd;
                    s1[e] += g;
                    s2[e] = __builtin_fmaf(g, d, s2[e]);
                    g *= gamma[e];
                    t += g;
                    u = __builtin_fmaf(g, d, u);
                }
            }
        if (!a.y)
            continue;
        const float2 m = join_groups({t, u}, h, each, group, here, of, of_group);
        const float m1 = m.x * share, m2 = m.y * share;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int64_t point = r + (int64_t)i * h.high;
            if (here && point < a.points) {
                float xs[V], gs[V];
                Values<T, V>::values(x[i], xs);
                Values<T, V>::values(dy[i], gs);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float g, d;
                    value(i, e, xs, gs, g, d);
                    xs[e] = rstd * ((g * gamma[e] - m1) - d * rstd * m2);
                }
                Values<T, V>::store((T *)a.y + (row0 + point) * a.ldy + c, xs);
            }
        }
    }
    if (!a.dgamma && !a.dbeta)
        return;
    float *to = part + (int64_t)at.stride * 2 * a.channels;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        float2 t = {s1[e], s2[e]};
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
// kLine bytes, at most eight points a thread.
bool held_plan(int32_t dtype, int64_t images, int64_t points, int32_t channels, int32_t groups, HeldPlan *o) {
    constexpr int kLine = 64;
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
    const size_t lds = (size_t)(o.threads + o.h.groups) * sizeof(float2);
    if (!backward) {
        held_forward_kernel<T, V, I><<<o.grid, o.threads, lds, stream>>>(a, o.h);
        return hipGetLastError();
    }
    float *part = (float *)a.scratch, *room = part + (int64_t)o.h.strides * 2 * a.channels;
    held_backward_kernel<T, V, I><<<o.grid, o.threads, lds, stream>>>(a, o.h, part);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? launch_parameters(a, part, o.h.strides, room, stream) : e;
}
template <typename T, int V>
hipError_t launch_held(const GroupNorm &a, const HeldPlan &o, bool backward, hipStream_t stream) {
    return o.each == 2 ? launch_held<T, V, 2>(a, o, backward, stream)
           : o.each == 4 ? launch_held<T, V, 4>(a, o, backward, stream) : launch_held<T, V, 8>(a, o, backward, stream);
}
hipError_t launch_held(const GroupNorm &a, const HeldPlan &o, int32_t dtype, bool backward, hipStream_t stream) {
    if (dtype == HPACML_F32)
        return o.v == 4 ? launch_held<float, 4>(a, o, backward, stream) : launch_held<float, 1>(a, o, backward, stream);
    return o.v == 8 ? launch_held<uint16_t, 8>(a, o, backward, stream)
           : o.v == 4 ? launch_held<uint16_t, 4>(a, o, backward, stream) : launch_held<uint16_t, 1>(a, o, backward, stream);
}

// Vectors that all of a row's channels fill: 16 bytes, or one value.
int whole_vector(int32_t dtype, int32_t channels) {
    const int v = dtype == HPACML_F32 ? 4 : 8;
    return channels % v == 0 ? v : 1;
}

Parts parts_of(int32_t dtype, int64_t images, int64_t points, int32_t channels) {
    Parts p;
    const int v = whole_vector(dtype, channels);
    p.vectors = channels / v;
    p.across = p.vectors < 256 ? p.vectors : 256;
    p.column_tiles = (uint32_t)((p.vectors + p.across - 1) / p.across);
    p.high = 1;
    while (p.high * 2 * p.across <= 256)
        p.high *= 2;
    // about eight blocks for each of 256 CUs, runs of no less than eight values a thread
    const int64_t want = 2048 / images / p.column_tiles + 1, least = 8 * p.high;
    int64_t run = (points + want - 1) / want;
    run = (run + least - 1) / least * least;
    p.run = run;
    p.runs = (uint32_t)((points + run - 1) / run);
    p.blocks = images * p.runs * p.column_tiles;
    return p;
}

// A grid's blocks of 256 threads: a launch has fewer than 2^32 threads.
uint32_t grid_of(int64_t blocks) { return (uint32_t)(blocks < 1 << 20 ? blocks : 1 << 20); }

size_t rounded(size_t n) { return (n + 255) / 256 * 256; }

template <typename T, int V>
hipError_t forward_parts(const GroupNorm &a, const Parts &p, hipStream_t stream) {
    const uint32_t blocks = grid_of(p.blocks);
    float2 *part = (float2 *)a.scratch;
    float *moments = (float *)(a.scratch + rounded((size_t)a.images * p.runs * a.channels * 8));
    float *mean = a.mean ? a.mean : moments, *rstd = a.mean ? a.rstd : moments + a.images * a.groups;
    parts_moments_kernel<T, V><<<blocks, 256, 0, stream>>>(a, p, part);
    parts_join_kernel<<<grid_of(a.images * a.groups), 256, 0, stream>>>(a, p, part, mean, rstd);
    parts_apply_kernel<T, V><<<blocks, 256, 0, stream>>>(a, p, mean, rstd);
    return hipGetLastError();
}

template <typename T, int V>
hipError_t backward_parts(const GroupNorm &a, const Parts &p, hipStream_t stream) {
    const int64_t rows = a.images * p.runs;
    const uint32_t blocks = grid_of(p.blocks);
    float *part = (float *)a.scratch;
    float2 *means = (float2 *)(a.scratch + rounded((size_t)rows * a.channels * 8));
    float *room = (float *)((char *)means + rounded((size_t)a.images * a.groups * 8));
    parts_sums_kernel<T, V><<<blocks, 256, 0, stream>>>(a, p, part);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess)
        e = launch_parameters(a, part, rows, room, stream);
    if (a.y && e == hipSuccess) {
        parts_means_kernel<<<grid_of(a.images * a.groups), 256, 0, stream>>>(a, p, part, means);
        parts_dx_kernel<T, V><<<blocks, 256, 0, stream>>>(a, p, means);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

int64_t group_norm_scratch(int32_t dtype, int64_t images, int64_t points, int32_t channels, int32_t groups, bool backward) {
    RowsPlan o;
    if (images == 0)
        return 0;
    if (rows_plan(dtype, images, points, channels, groups, &o))
        return backward ? (o.p.strides * 2 * channels + column_sums_room(o.p.strides, 2 * channels)) * 4 : 0;
    HeldPlan d;
    if (held_plan(dtype, images, points, channels, groups, &d))
        return backward ? (d.h.strides * 2 * channels + column_sums_room(d.h.strides, 2 * channels)) * 4 : 0;
    const Parts p = parts_of(dtype, images, points, channels);
    const int64_t rows = images * p.runs;
    return (int64_t)(rounded((size_t)rows * channels * 8) + rounded((size_t)images * groups * 8) +
                     (backward ? rounded((size_t)column_sums_room(rows, 2 * channels) * 4) : 0));
}

hipError_t launch_group_norm(const GroupNorm &a, int32_t dtype, hipStream_t stream) {
    RowsPlan o;
    if (a.images == 0)
        return hipSuccess;
    if (rows_plan(dtype, a.images, a.points, a.channels, a.groups, &o))
        return launch_rows(a, o, dtype, false, stream);
    HeldPlan d;
    if (held_plan(dtype, a.images, a.points, a.channels, a.groups, &d))
        return launch_held(a, d, dtype, false, stream);
    const Parts p = parts_of(dtype, a.images, a.points, a.channels);
    const int v = whole_vector(dtype, a.channels);
    if (dtype == HPACML_F32)
        return v == 4 ? forward_parts<float, 4>(a, p, stream) : forward_parts<float, 1>(a, p, stream);
    return v == 8 ? forward_parts<uint16_t, 8>(a, p, stream) : forward_parts<uint16_t, 1>(a, p, stream);
}

hipError_t launch_group_norm_backward(const GroupNorm &a, int32_t dtype, hipStream_t stream) {
    if (a.images == 0) {
        return a.accumulate ? hipSuccess : launch_parameters(a, nullptr, 0, nullptr, stream);
    }
    RowsPlan o;
    if (rows_plan(dtype, a.images, a.points, a.channels, a.groups, &o))
        return launch_rows(a, o, dtype, true, stream);
    HeldPlan d;
    if (held_plan(dtype, a.images, a.points, a.channels, a.groups, &d))
        return launch_held(a, d, dtype, true, stream);
    const Parts p = parts_of(dtype, a.images, a.points, a.channels);
    const int v = whole_vector(dtype, a.channels);
    if (dtype == HPACML_F32)
        return v == 4 ? backward_parts<float, 4>(a, p, stream) : backward_parts<float, 1>(a, p, stream);
    return v == 8 ? backward_parts<uint16_t, 8>(a, p, stream) : backward_parts<uint16_t, 1>(a, p, stream);
}

}  // namespace hpacml
