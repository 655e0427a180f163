// norm_kernels.cuh - group norm with an activation, channels last, forward and gradient.
// Device code; included by layers.cuh inside its unnamed namespace.
//
//   xhat = (x - mean) rstd,  z = xhat weight + bias,  y = act(z)
//   dz = dy act'(z),  dx = rstd (dz weight - (s1 + xhat s2) / N),  s1 = sum dz weight,  s2 = sum dz weight xhat  over the group
//
// Everything that is summed is summed for each channel first, then over the channels of a group: one walk over the pixels serves any
// number of channels a group, and the gradient's channel sums are dbias and dweight.  Bound: memory.
#pragma once

enum { kActNone = CSER_ACT_NONE, kActRelu = CSER_ACT_RELU, kActSilu = CSER_ACT_SILU };

struct View { long long pixel, sample, worker; };      // strides in elements

template <typename T> struct NormArgs {
    const T *x, *dy;
    T *y;                                              // result: y, or dx
    View xs, dys, ys;
    const float *weight, *bias;                        // or null
    long long weight_worker, bias_worker;
    float *stats;                                      // mean [n, samples, groups], then rstd
    float2 *group_sums;                                // s1 / N, s2 / N of each sample's groups
    float *part;                                       // two planes of [n * samples][chunks][channels]
    long long plane;
    int n, samples, channels, groups, per_group, act;
    long long pixels;
    float eps;
    int tx, col_blocks, chunks;                        // tx: column vectors of a block of 256 threads
    long long chunk_pixels;
    Draw draw;
};

// Exponential and reciprocal by the hardware's approximations, about 2^-22 each: below the rounding of fp32 results' own sums by little,
// of 16-bit ones by far.
__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.f, 1.f + __expf(-z)); }

__device__ __forceinline__ float activate(float z, int act) {
    if (act == kActSilu) return z * sigmoid(z);
    if (act == kActRelu) return z > 0.f || z != z ? z : 0.f;
    return z;
}
// dy * act'(z)
__device__ __forceinline__ float slope_times(float dy, float z, int act) {
    if (act == kActSilu) {
        const float g = sigmoid(z);
        return dy * (g * fmaf(z, 1.f - g, 1.f));
    }
    if (act == kActRelu) return z > 0.f || z != z ? dy : 0.f;
    return dy;
}

// Mean and sum of squares about it of two sets, joined.
__device__ __forceinline__ void join_moments(float &n, float &mean, float &m2, float n2, float mean2, float m22) {
    const float total = n + n2;
    if (total == 0.f) return;
    const float share = n2 / total, d = mean2 - mean;
    mean = fmaf(d, share, mean);
    m2 = m2 + m22 + d * d * (n * share);
    n = total;
}

// V elements of x as they count, dropped out or not, from element e of the worker's array on; their keep bits.
template <int V, bool DROP>
__device__ __forceinline__ uint32_t counted(float (&f)[V], const Draw &d, const Words &words, long long e) {
    if (!DROP) return ~0u;
    const Drawn<V, V % 4 == 0> drawn(words, e);
    uint32_t keep = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const bool k = drawn.w[j] >= d.threshold;
        f[j] = k ? f[j] * d.factor : 0.f;
        keep |= (uint32_t)k << j;
    }
    return keep;
}

// Where a thread of the walking kernels stands.  256 threads are tx column vectors (a power of two up to 32) x 256 / tx pixels.
struct Place {
    int w, b, chunk, c, ty, rows;                      // rows: pixels that the block takes at a time
    long long first, last;
    bool in;
};
template <typename T, int V> __device__ __forceinline__ Place place(const NormArgs<T> &a) {
    Place p;
    const int col_block = blockIdx.x % a.col_blocks;
    const int rest = blockIdx.x / a.col_blocks;
    p.chunk = rest % a.chunks;
    const int sample = rest / a.chunks;
    p.w = sample / a.samples, p.b = sample % a.samples;
    p.c = (col_block * a.tx + (threadIdx.x & (a.tx - 1))) * V;
    p.ty = threadIdx.x / a.tx, p.rows = 256 / a.tx;
    p.first = p.chunk * a.chunk_pixels;
    p.last = p.first + a.chunk_pixels < a.pixels ? p.first + a.chunk_pixels : a.pixels;
    p.in = p.c < a.channels;
    return p;
}

template <int V> struct Channels {                     // a thread's channels
    float mean[V], rstd[V], weight[V], bias[V];
};
template <typename T, int V> __device__ __forceinline__ void channels_of(Channels<V> &k, const NormArgs<T> &a, int w, int b, int c, bool with_stats) {
    const float *mean = a.stats + ((long long)w * a.samples + b) * a.groups, *rstd = mean + (long long)a.n * a.samples * a.groups;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int g = (c + j) / a.per_group;
        k.mean[j] = with_stats ? mean[g] : 0.f, k.rstd[j] = with_stats ? rstd[g] : 0.f;
        k.weight[j] = a.weight ? a.weight[w * a.weight_worker + c + j] : 1.f;
        k.bias[j] = a.bias ? a.bias[w * a.bias_worker + c + j] : 0.f;
    }
}

// Moments of each channel over a chunk of a sample's pixels: plane 0 the mean, plane 1 the sum of squares about it.
template <typename T, int V, bool DROP>
__global__ void __launch_bounds__(256) norm_moments_kernel(NormArgs<T> a) {
    after_previous();
    let_next();
    const Place p = place<T, V>(a);
    const Words words(a.draw, p.w);
    float n = 0.f, mean[V], m2[V];
#pragma unroll
    for (int j = 0; j < V; ++j) mean[j] = m2[j] = 0.f;
    if (p.in) {
        const T *x = a.x + p.w * a.xs.worker + p.b * a.xs.sample + p.c;
        const long long e0 = (long long)p.b * a.pixels * a.channels + p.c;
        constexpr int U = 4;                           // pixels whose moments are taken about their own mean, then joined
        for (long long i = p.first + p.ty; i < p.last; i += U * p.rows) {
            float f[U][V];
            Vec<T, V> v[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * p.rows < p.last) v[u] = Vec<T, V>(x + (i + u * p.rows) * a.xs.pixel);
            int got = 0;
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * p.rows < p.last) {
                    v[u].floats(f[u]);
                    counted<V, DROP>(f[u], a.draw, words, e0 + (i + u * p.rows) * a.channels);
                    ++got;
                }
            const float part = 1.f / got, share = got / (n + got);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float s = f[0][j];
#pragma unroll
                for (int u = 1; u < U; ++u) s += u < got ? f[u][j] : 0.f;
                s *= part;
                float q = 0.f;
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (u < got) q = fmaf(f[u][j] - s, f[u][j] - s, q);
                const float d = s - mean[j];
                mean[j] = fmaf(d, share, mean[j]);
                m2[j] += q + d * d * (n * share);
            }
            n += got;
        }
    }
    // Threads of the same channels: those of a warp, then the eight warps.
    __shared__ float count[8][32], means[8][32 * V], squares[8][32 * V];
    for (int o = a.tx; o < 32; o <<= 1) {
        const float n2 = __shfl_xor_sync(~0u, n, o);
        float total = n;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float mean2 = __shfl_xor_sync(~0u, mean[j], o), m22 = __shfl_xor_sync(~0u, m2[j], o);
            total = n;
            // The lower lane's set comes first in both, so that both end with the same bits.
            if (threadIdx.x & o) {
                float nn = n2, mm = mean2, qq = m22;
                join_moments(nn, mm, qq, n, mean[j], m2[j]);
                mean[j] = mm, m2[j] = qq, total = nn;
            } else {
                join_moments(total, mean[j], m2[j], n2, mean2, m22);
            }
        }
        n = n + n2;
    }
    const int warp = threadIdx.x >> 5, tx = threadIdx.x & (a.tx - 1);
    if ((threadIdx.x & 31) < a.tx) {
        count[warp][tx] = n;
#pragma unroll
        for (int j = 0; j < V; ++j) means[warp][tx * V + j] = mean[j], squares[warp][tx * V + j] = m2[j];
    }
    __syncthreads();
    const int k = threadIdx.x, c = (blockIdx.x % a.col_blocks) * a.tx * V + k;
    if (k < a.tx * V && c < a.channels) {
        float nn = count[0][k / V], mm = means[0][k], qq = squares[0][k];
#pragma unroll
        for (int i = 1; i < 8; ++i) join_moments(nn, mm, qq, count[i][k / V], means[i][k], squares[i][k]);
        const long long at = (((long long)p.w * a.samples + p.b) * a.chunks + p.chunk) * a.channels + c;
        a.part[at] = mm, a.part[a.plane + at] = qq;
    }
}

// Mean and rstd of each group from its channels' moments: a warp a group.
template <typename T> __global__ void __launch_bounds__(256) norm_join_moments_kernel(NormArgs<T> a) {
    after_previous();
    let_next();
    const long long g = (long long)blockIdx.x * 8 + (threadIdx.x >> 5), all = (long long)a.n * a.samples * a.groups;
    if (g >= all) return;
    const int lane = threadIdx.x & 31;
    const long long sample = g / a.groups;
    const float *part = a.part + sample * a.chunks * a.channels + (g % a.groups) * a.per_group;
    const int entries = a.chunks * a.per_group;
    float n = 0.f, mean = 0.f, m2 = 0.f;
    for (int i = lane; i < entries; i += 32) {
        const int chunk = i / a.per_group, c = i % a.per_group;
        const long long left = a.pixels - chunk * a.chunk_pixels;
        const float count = (float)(left < a.chunk_pixels ? left : a.chunk_pixels);
        const long long at = (long long)chunk * a.channels + c;
        join_moments(n, mean, m2, count, part[at], part[a.plane + at]);
    }
    for (int o = 1; o < 32; o <<= 1) {
        const float n2 = __shfl_down_sync(~0u, n, o), mean2 = __shfl_down_sync(~0u, mean, o), m22 = __shfl_down_sync(~0u, m2, o);
        join_moments(n, mean, m2, n2, mean2, m22);     // lane 0 joins disjoint sets: what it adds has not been added by others
    }
    if (lane == 0) a.stats[g] = mean, a.stats[all + g] = 1.f / sqrtf(m2 / n + a.eps);
}

template <typename T, int V, bool DROP>
__global__ void __launch_bounds__(256) norm_apply_kernel(NormArgs<T> a) {
    after_previous();
    let_next();
    const Place p = place<T, V>(a);
    if (!p.in) return;
    const Words words(a.draw, p.w);
    Channels<V> k;
    channels_of(k, a, p.w, p.b, p.c, true);
    const T *x = a.x + p.w * a.xs.worker + p.b * a.xs.sample + p.c;
    T *y = a.y + p.w * a.ys.worker + p.b * a.ys.sample + p.c;
    const long long e0 = (long long)p.b * a.pixels * a.channels + p.c;
#pragma unroll
    for (int j = 0; j < V; ++j) k.weight[j] *= k.rstd[j];
    for (long long i = p.first + p.ty; i < p.last; i += p.rows) {
        float f[V];
        Vec<T, V> v(x + i * a.xs.pixel);
        v.floats(f);
        counted<V, DROP>(f, a.draw, words, e0 + i * a.channels);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = activate(fmaf(f[j] - k.mean[j], k.weight[j], k.bias[j]), a.act);
        v.round(f);
        v.to(y + i * a.ys.pixel);
    }
}

// Sums of dz (plane 0) and dz * xhat (plane 1) of each channel over a chunk of a sample's pixels.
template <typename T, int V, bool DROP>
__global__ void __launch_bounds__(256) norm_grad_sums_kernel(NormArgs<T> a) {
    after_previous();
    let_next();
    const Place p = place<T, V>(a);
    const Words words(a.draw, p.w);
    float s0[V], s1[V];
#pragma unroll
    for (int j = 0; j < V; ++j) s0[j] = s1[j] = 0.f;
    if (p.in) {
        Channels<V> k;
        channels_of(k, a, p.w, p.b, p.c, true);
        const T *x = a.x + p.w * a.xs.worker + p.b * a.xs.sample + p.c, *dy = a.dy + p.w * a.dys.worker + p.b * a.dys.sample + p.c;
        const long long e0 = (long long)p.b * a.pixels * a.channels + p.c;
        for (long long i = p.first + p.ty; i < p.last; i += p.rows) {
            float f[V], d[V];
            Vec<T, V> vx(x + i * a.xs.pixel), vd(dy + i * a.dys.pixel);
            vx.floats(f), vd.floats(d);
            counted<V, DROP>(f, a.draw, words, e0 + i * a.channels);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float h = (f[j] - k.mean[j]) * k.rstd[j], dz = slope_times(d[j], fmaf(h, k.weight[j], k.bias[j]), a.act);
                s0[j] += dz, s1[j] = fmaf(dz, h, s1[j]);
            }
        }
    }
    __shared__ float sums[2][8][32 * V];
    for (int o = a.tx; o < 32; o <<= 1)
#pragma unroll
        for (int j = 0; j < V; ++j) s0[j] += __shfl_xor_sync(~0u, s0[j], o), s1[j] += __shfl_xor_sync(~0u, s1[j], o);
    const int warp = threadIdx.x >> 5, tx = threadIdx.x & (a.tx - 1);
    if ((threadIdx.x & 31) < a.tx)
#pragma unroll
        for (int j = 0; j < V; ++j) sums[0][warp][tx * V + j] = s0[j], sums[1][warp][tx * V + j] = s1[j];
    __syncthreads();
    const int k = threadIdx.x, c = (blockIdx.x % a.col_blocks) * a.tx * V + k;
    if (k < a.tx * V && c < a.channels) {
        float t0 = 0.f, t1 = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) t0 += sums[0][i][k], t1 += sums[1][i][k];
        const long long at = (((long long)p.w * a.samples + p.b) * a.chunks + p.chunk) * a.channels + c;
        a.part[at] = t0, a.part[a.plane + at] = t1;
    }
}

// s1 / N and s2 / N of each group: a warp a group.
template <typename T> __global__ void __launch_bounds__(256) norm_join_sums_kernel(NormArgs<T> a) {
    after_previous();
    let_next();
    const long long g = (long long)blockIdx.x * 8 + (threadIdx.x >> 5), all = (long long)a.n * a.samples * a.groups;
    if (g >= all) return;
    const int lane = threadIdx.x & 31;
    const long long sample = g / a.groups;
    const int c0 = (int)(g % a.groups) * a.per_group, w = (int)(sample / a.samples);
    const float *part = a.part + sample * a.chunks * a.channels + c0;
    const int entries = a.chunks * a.per_group;
    float s0 = 0.f, s1 = 0.f;
    for (int i = lane; i < entries; i += 32) {
        const int chunk = i / a.per_group, c = i % a.per_group;
        const float k = a.weight ? a.weight[w * a.weight_worker + c0 + c] : 1.f;
        const long long at = (long long)chunk * a.channels + c;
        s0 = fmaf(part[at], k, s0), s1 = fmaf(part[a.plane + at], k, s1);
    }
    for (int o = 16; o; o >>= 1) s0 += __shfl_xor_sync(~0u, s0, o), s1 += __shfl_xor_sync(~0u, s1, o);
    const float of = 1.f / ((float)a.pixels * a.per_group);
    if (lane == 0) a.group_sums[g] = make_float2(s0 * of, s1 * of);
}

template <typename T, int V, bool DROP>
__global__ void __launch_bounds__(256) norm_grad_apply_kernel(NormArgs<T> a) {
    after_previous();
    let_next();
    const Place p = place<T, V>(a);
    if (!p.in) return;
    const Words words(a.draw, p.w);
    Channels<V> k;
    channels_of(k, a, p.w, p.b, p.c, true);
    float m1[V], m2[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const float2 m = a.group_sums[((long long)p.w * a.samples + p.b) * a.groups + (p.c + j) / a.per_group];
        m1[j] = m.x, m2[j] = m.y;
    }
    const T *x = a.x + p.w * a.xs.worker + p.b * a.xs.sample + p.c, *dy = a.dy + p.w * a.dys.worker + p.b * a.dys.sample + p.c;
    T *y = a.y + p.w * a.ys.worker + p.b * a.ys.sample + p.c;
    const long long e0 = (long long)p.b * a.pixels * a.channels + p.c;
    for (long long i = p.first + p.ty; i < p.last; i += p.rows) {
        float f[V], d[V];
        Vec<T, V> vx(x + i * a.xs.pixel), vd(dy + i * a.dys.pixel);
        vx.floats(f), vd.floats(d);
        const uint32_t keep = counted<V, DROP>(f, a.draw, words, e0 + i * a.channels);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float h = (f[j] - k.mean[j]) * k.rstd[j], dz = slope_times(d[j], fmaf(h, k.weight[j], k.bias[j]), a.act);
            f[j] = k.rstd[j] * (fmaf(dz, k.weight[j], -m1[j]) - h * m2[j]);
            if (DROP) f[j] = keep >> j & 1 ? f[j] * a.draw.factor : 0.f;
        }
        vx.round(f);
        vx.to(y + i * a.ys.pixel);
    }
}
