// Group norm of large images: sums of runs of points, their join, and the results
// from a second reading.  A run's values count from its first one on (Moments): with
// pairs of mean and squares in 32 bits, joined a few values at a time, 100,000 +- 0.02
// had an rstd up to 10% off.  An image of 2048^2 points x 8 channels in fp32 takes 75 us
// (27 for the first reading, 7 for the join, 43 for the results), 89 with results
// through the caches, whose write-back the next first reading meets (its gradients 121
// and 145).
#include "group_norm_device.hpp"

namespace hpacml {

namespace {

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

// f(points, how many of them exist) for the thread's points, points_at_once<V> at a time,
// so that their loads go out together (the last again where there is none).
template <int V>
constexpr int points_at_once = V == 1 ? 8 : 4;
template <int V, typename F>
__device__ __forceinline__ void over_points(const Place &q, const Parts &p, F f) {
    constexpr int kAtOnce = points_at_once<V>;
    for (int64_t row = q.first + q.r; row < q.last; row += kAtOnce * p.high) {
        int64_t rows[kAtOnce];
        int n = 0;
#pragma unroll
        for (int b = 0; b < kAtOnce; ++b) {
            rows[b] = min(row + b * p.high, q.last - 1);
            n += row + b * p.high < q.last;
        }
        f(rows, n);
    }
}

// [image][run][channel] (mean less the channel's first value of the run, deviation).
// A deviation stays in fp32's range where the sum of squares does not.
template <typename T, int V>
__global__ __launch_bounds__(256) void parts_moments_kernel(GroupNorm a, Parts p, float2 *part) {
    constexpr int kBatch = 8;
    __shared__ double2 of[256][V];
    for (int64_t block = blockIdx.x; block < p.blocks; block += gridDim.x) {
        const Place q = place_of<V>(a, p, block);
        Moments m[V];
        if (q.here) {
            const T *x = (const T *)a.x + q.c;
            float first[V];
            Values<T, V>::load(x + q.first * a.ldx, first);
            double pivot[V];
#pragma unroll
            for (int e = 0; e < V; ++e)
                pivot[e] = first[e];
            int64_t row = q.first + q.r;
            for (; row + (kBatch - 1) * p.high < q.last; row += kBatch * p.high) {
                typename Values<T, V>::Held w[kBatch];
#pragma unroll
                for (int b = 0; b < kBatch; ++b)
                    w[b] = Values<T, V>::hold(x + (row + b * p.high) * a.ldx);
#pragma unroll
                for (int b = 0; b < kBatch; ++b) {
                    float v[V];
                    Values<T, V>::values(w[b], v);
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        m[e].add(v[e], pivot[e]);
                }
            }
            for (; row < q.last; row += p.high) {
                float v[V];
                Values<T, V>::load(x + row * a.ldx, v);
#pragma unroll
                for (int e = 0; e < V; ++e)
                    m[e].add(v[e], pivot[e]);
            }
        }
#pragma unroll
        for (int e = 0; e < V; ++e)
            of[threadIdx.x][e] = {m[e].sum, m[e].squares};
        // threads' points: every `high`-th from r on; joined in halves
        for (int h = p.high / 2; h > 0; h /= 2) {
            __syncthreads();
            if (q.here && q.r < h)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const double2 o = of[threadIdx.x + h * p.across][e];
                    m[e].sum += o.x;
                    m[e].squares += o.y;
                    of[threadIdx.x][e] = {m[e].sum, m[e].squares};
                }
        }
        if (q.here && q.r == 0) {
            float2 *to = part + (block / p.column_tiles) * (int64_t)a.channels + q.c;
            const double share = 1.0 / (double)(q.last - q.first);
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (q.c + e < a.channels)
                    to[e] = {(float)(m[e].sum * share), (float)sqrt(m[e].variance(share))};
        }
        __syncthreads();
    }
}

template <int THREADS>
__device__ __forceinline__ double join_block(double t, double (&of_wave)[THREADS / 64]) {
#pragma unroll
    for (int s = 1; s < 64; s *= 2)
        t += __shfl_xor(t, s);
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        of_wave[threadIdx.x >> 6] = t;
    __syncthreads();
    t = of_wave[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w)
        t += of_wave[w];
    return t;
}

// The partial results of an image's group, `per` channels of each run: a thread
// takes every so many runs of one channel (with one index over all of them, and
// its divisions, 2049 runs of 4 channels took 23 us).
template <int THREADS, typename F>
__device__ __forceinline__ void over_runs(int per, uint32_t runs, F f) {
    const int across = min(per, THREADS), high = THREADS / across, c0 = threadIdx.x % across, r0 = threadIdx.x / across;
    if (r0 < high)
        for (int c = c0; c < per; c += across)
#pragma unroll 8
            for (uint32_t r = r0; r < runs; r += high)
                f(c, r);
}

// A block per image and group: mean and rstd.  part NULL: runs are single values.
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void parts_join_kernel(GroupNorm a, Parts p, const float2 *part, float *mean_to, float *rstd_to) {
    __shared__ double of_wave[THREADS / 64];
    for (int64_t unit = blockIdx.x; unit < a.images * a.groups; unit += gridDim.x) {
        const int64_t image = unit / a.groups;
        const int per = a.channels / a.groups, c0 = (int)(unit % a.groups) * per;
        const float2 *at = part + image * p.runs * a.channels + c0;
        const T *x = (const T *)a.x + image * a.points * a.ldx + c0;
        auto values = [&](uint32_t r) { return (double)min(p.run, a.points - r * p.run); };
        auto part_of = [&](int c, uint32_t r) { return part ? at[(int64_t)r * a.channels + c] : float2{0.f, 0.f}; };
        auto mean_of = [&](int c, uint32_t r, float more) { return (double)load_value(x + r * p.run * a.ldx + c) + more; };
        double t = 0;
        over_runs<THREADS>(per, p.runs, [&](int c, uint32_t r) { t += values(r) * mean_of(c, r, part_of(c, r).x); });
        const double n = (double)a.points * per, mean = join_block<THREADS>(t, of_wave) / n;
        t = 0;
        over_runs<THREADS>(per, p.runs, [&](int c, uint32_t r) {
            const float2 o = part_of(c, r);
            const double d = mean_of(c, r, o.x) - mean;
            t += values(r) * ((double)o.y * o.y + d * d);
        });
        t = join_block<THREADS>(t, of_wave);
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
        // (whole vectors: channels c .. c + V - 1 exist)
        const int per = a.channels / a.groups;
        load_parameters<V>(a.gamma ? a.gamma + c : nullptr, 1.f, gamma);
        load_parameters<V>(a.beta ? a.beta + c : nullptr, 0.f, beta);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int64_t at = image * a.groups + (c + e) / per;
            mean[e] = means[at];
            rstd[e] = rstds[at];
        }
    }
};

template <typename T, int V, int ACT>
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
        over_points<V>(q, p, [&](const int64_t (&rows)[points_at_once<V>], int n) {
            typename Values<T, V>::Held w[points_at_once<V>];
#pragma unroll
            for (int b = 0; b < points_at_once<V>; ++b)
                w[b] = Values<T, V>::hold((const T *)a.x + rows[b] * a.ldx + q.c);
#pragma unroll
            for (int b = 0; b < points_at_once<V>; ++b)
                if (b < n) {
                    float v[V];
                    Values<T, V>::values(w[b], v);
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        v[e] = activation<ACT>(__builtin_fmaf(v[e] - k.mean[e], k.gamma[e], k.beta[e]));
                    Values<T, V>::store_past((T *)a.y + rows[b] * a.ldy + q.c, v);
                }
        });
    }
}

// sums of g and of g (x - mean) rstd: [image][run][2][channel]
template <typename T, int V, int ACT>
__global__ __launch_bounds__(256) void parts_sums_kernel(GroupNorm a, Parts p, float *part) {
    __shared__ float2 of[256][V];
    for (int64_t block = blockIdx.x; block < p.blocks; block += gridDim.x) {
        const Place q = place_of<V>(a, p, block);
        Total<V> s1[V], s2[V];
#pragma unroll
        for (int e = 0; e < V; ++e)
            s1[e] = s2[e] = 0;
        Channels<V> k;
        if (q.here) {
            k.load(a, q.image, q.c, a.mean, a.rstd);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                k.gamma[e] *= k.rstd[e];
                k.gamma[e] *= kUnit<ACT>;
                k.beta[e] *= kUnit<ACT>;
            }
            over_points<V>(q, p, [&](const int64_t (&rows)[points_at_once<V>], int n) {
                typename Values<T, V>::Held w[points_at_once<V>], o[points_at_once<V>];
#pragma unroll
                for (int b = 0; b < points_at_once<V>; ++b) {
                    w[b] = Values<T, V>::hold((const T *)a.x + rows[b] * a.ldx + q.c);
                    o[b] = Values<T, V>::hold((const T *)a.dy + rows[b] * a.lddy + q.c);
                }
                float t1[V], t2[V];
#pragma unroll
                for (int e = 0; e < V; ++e)
                    t1[e] = t2[e] = 0;
#pragma unroll
                for (int b = 0; b < points_at_once<V>; ++b)
                    if (b < n) {
                        float v[V], g[V];
                        Values<T, V>::values(w[b], v);
                        Values<T, V>::values(o[b], g);
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            const float d = v[e] - k.mean[e];
                            const float t = activation_gradient<ACT>(g[e], __builtin_fmaf(d, k.gamma[e], k.beta[e]));
                            t1[e] += t;
                            t2[e] = __builtin_fmaf(t, d, t2[e]);
                        }
                    }
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    s1[e] += t1[e];
                    s2[e] += t2[e];
                }
            });
        }
#pragma unroll
        for (int e = 0; e < V; ++e)
            of[threadIdx.x][e] = {(float)s1[e], (float)s2[e]};
        for (int h = p.high / 2; h > 0; h /= 2) {
            __syncthreads();
            if (q.here && q.r < h)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float2 o = of[threadIdx.x + h * p.across][e];
                    s1[e] += o.x;
                    s2[e] += o.y;
                    of[threadIdx.x][e] = {(float)s1[e], (float)s2[e]};
                }
        }
        if (q.here && q.r == 0) {
            float *to = part + (block / p.column_tiles) * (int64_t)(2 * a.channels) + q.c;
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (q.c + e < a.channels) {
                    to[e] = (float)s1[e];
                    to[a.channels + e] = (float)(s2[e] * k.rstd[e]);
                }
        }
        __syncthreads();
    }
}

// A block per image and group: the means of g gamma and g gamma (x - mean) rstd.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void parts_means_kernel(GroupNorm a, Parts p, const float *part, float2 *means) {
    __shared__ double of_wave[THREADS / 64];
    for (int64_t unit = blockIdx.x; unit < a.images * a.groups; unit += gridDim.x) {
        const int64_t image = unit / a.groups;
        const int per = a.channels / a.groups, c0 = (int)(unit % a.groups) * per;
        const float *at = part + image * p.runs * 2 * a.channels + c0;
        double t = 0, u = 0;
        over_runs<THREADS>(per, p.runs, [&](int c, uint32_t r) {
            const float *o = at + (int64_t)r * 2 * a.channels + c;
            const double gamma = a.gamma ? a.gamma[c0 + c] : 1.f;
            t += gamma * o[0];
            u += gamma * o[a.channels];
        });
        const double n = (double)a.points * per;
        t = join_block<THREADS>(t, of_wave) / n;
        u = join_block<THREADS>(u, of_wave) / n;
        if (threadIdx.x == 0)
            means[unit] = {(float)t, (float)u};
    }
}

template <typename T, int V, int ACT>
__global__ __launch_bounds__(256) void parts_dx_kernel(GroupNorm a, Parts p, const float2 *means) {
    for (int64_t block = blockIdx.x; block < p.blocks; block += gridDim.x) {
        const Place q = place_of<V>(a, p, block);
        if (!q.here)
            continue;
        Channels<V> k;
        k.load(a, q.image, q.c, a.mean, a.rstd);
        // dx = g gamma rstd - (x - mean) rstd^2 m2 - rstd m1
        float slope[V], shift[V], scale[V];
        const int per = a.channels / a.groups;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float2 m = means[q.image * a.groups + min(q.c + e, a.channels - 1) / per];
            shift[e] = -k.rstd[e] * m.x;
            slope[e] = -k.rstd[e] * (k.rstd[e] * m.y);
            scale[e] = k.gamma[e] * k.rstd[e];
            k.gamma[e] = scale[e] * kUnit<ACT>;
            k.beta[e] *= kUnit<ACT>;
        }
        over_points<V>(q, p, [&](const int64_t (&rows)[points_at_once<V>], int n) {
            typename Values<T, V>::Held w[points_at_once<V>], o[points_at_once<V>];
#pragma unroll
            for (int b = 0; b < points_at_once<V>; ++b) {
                w[b] = Values<T, V>::hold((const T *)a.x + rows[b] * a.ldx + q.c);
                o[b] = Values<T, V>::hold((const T *)a.dy + rows[b] * a.lddy + q.c);
            }
#pragma unroll
            for (int b = 0; b < points_at_once<V>; ++b)
                if (b < n) {
                    float v[V], g[V];
                    Values<T, V>::values(w[b], v);
                    Values<T, V>::values(o[b], g);
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float d = v[e] - k.mean[e];
                        const float t = activation_gradient<ACT>(g[e], __builtin_fmaf(d, k.gamma[e], k.beta[e]));
                        v[e] = __builtin_fmaf(t, scale[e], __builtin_fmaf(d, slope[e], shift[e]));
                    }
                    Values<T, V>::store_past((T *)a.y + rows[b] * a.ldy + q.c, v);
                }
        });
    }
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
    // two blocks for each of 256 CUs, runs of no less than eight values a thread
    // (2048^2 points x 8 channels: 93 us with eight blocks, 89 us with two, whose runs are fewer to join)
    const int64_t want = 512 / images / p.column_tiles + 1, least = 8 * p.high;
    int64_t run = (points + want - 1) / want;
    run = (run + least - 1) / least * least;
    p.run = run;
    p.runs = (uint32_t)((points + run - 1) / run);
    p.blocks = images * p.runs * p.column_tiles;
    return p;
}

// A grid's blocks of 256 threads: a launch has fewer than 2^32 threads.
uint32_t grid_of(int64_t blocks) { return (uint32_t)(blocks < 1 << 20 ? blocks : 1 << 20); }

// Whether larger blocks join the parts of a group: there are fewer groups than CUs.
bool few_units(const GroupNorm &a) { return a.images * a.groups < 256; }

size_t rounded(size_t n) { return (n + 255) / 256 * 256; }

// Of an image of one point (whose groups are too wide for registers) a run is one value.
size_t forward_part_bytes(int64_t images, int64_t points, int64_t runs, int32_t channels) {
    return points > 1 ? rounded((size_t)images * runs * channels * 8) : 0;
}

template <typename T, int V>
hipError_t forward_parts(const GroupNorm &a, const Parts &p, hipStream_t stream) {
    const uint32_t blocks = grid_of(p.blocks);
    float2 *part = a.points > 1 ? (float2 *)a.scratch : nullptr;
    float *moments = (float *)(a.scratch + forward_part_bytes(a.images, a.points, p.runs, a.channels));
    float *mean = a.mean ? a.mean : moments, *rstd = a.mean ? a.rstd : moments + a.images * a.groups;
    if (part)
        parts_moments_kernel<T, V><<<blocks, 256, 0, stream>>>(a, p, part);
    if (few_units(a))
        parts_join_kernel<T, 1024><<<grid_of(a.images * a.groups), 1024, 0, stream>>>(a, p, part, mean, rstd);
    else
        parts_join_kernel<T, 256><<<grid_of(a.images * a.groups), 256, 0, stream>>>(a, p, part, mean, rstd);
    return with_activation(a.act, [&](auto act) {
        parts_apply_kernel<T, V, decltype(act)::value><<<blocks, 256, 0, stream>>>(a, p, mean, rstd);
        return hipGetLastError();
    });
}

template <typename T, int V>
hipError_t backward_parts(const GroupNorm &a, const Parts &p, hipStream_t stream) {
    const int64_t rows = a.images * p.runs;
    const uint32_t blocks = grid_of(p.blocks);
    float *part = (float *)a.scratch;
    float2 *means = (float2 *)(a.scratch + rounded((size_t)rows * a.channels * 8));
    float *room = (float *)((char *)means + rounded((size_t)a.images * a.groups * 8));
    hipError_t e = with_activation(a.act, [&](auto act) {
        parts_sums_kernel<T, V, decltype(act)::value><<<blocks, 256, 0, stream>>>(a, p, part);
        return hipGetLastError();
    });
    if (e == hipSuccess)
        e = launch_parameters(a, part, rows, room, stream);
    if (a.y && e == hipSuccess) {
        if (few_units(a))
            parts_means_kernel<1024><<<grid_of(a.images * a.groups), 1024, 0, stream>>>(a, p, part, means);
        else
            parts_means_kernel<256><<<grid_of(a.images * a.groups), 256, 0, stream>>>(a, p, part, means);
        e = with_activation(a.act, [&](auto act) {
            parts_dx_kernel<T, V, decltype(act)::value><<<blocks, 256, 0, stream>>>(a, p, means);
            return hipGetLastError();
        });
    }
    return e;
}

}  // namespace

int64_t norm_parts_scratch(int32_t dtype, int64_t images, int64_t points, int32_t channels, int32_t groups, bool backward) {
    const Parts p = parts_of(dtype, images, points, channels);
    const int64_t rows = images * p.runs;
    const size_t moments = rounded((size_t)images * groups * 8);        // mean and rstd, or the means of the gradients
    if (!backward)
        return (int64_t)(forward_part_bytes(images, points, p.runs, channels) + moments);
    return (int64_t)(rounded((size_t)rows * channels * 8) + moments + rounded((size_t)column_sums_room(rows, 2 * channels) * 4));
}

hipError_t launch_norm_parts(const GroupNorm &a, int32_t dtype, bool backward, hipStream_t stream) {
    const Parts p = parts_of(dtype, a.images, a.points, a.channels);
    const int v = whole_vector(dtype, a.channels);
    if (dtype == HPACML_F32) {
        if (v == 4)
            return backward ? backward_parts<float, 4>(a, p, stream) : forward_parts<float, 4>(a, p, stream);
        return backward ? backward_parts<float, 1>(a, p, stream) : forward_parts<float, 1>(a, p, stream);
    }
    if (v == 8)
        return backward ? backward_parts<uint16_t, 8>(a, p, stream) : forward_parts<uint16_t, 8>(a, p, stream);
    return backward ? backward_parts<uint16_t, 1>(a, p, stream) : forward_parts<uint16_t, 1>(a, p, stream);
}

}  // namespace hpacml
