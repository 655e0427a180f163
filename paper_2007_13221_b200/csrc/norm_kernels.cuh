// norm_kernels.cuh - group norm with an activation, channels last, forward and gradient: arithmetic, and kernels for samples that do not
// fit a cluster's shared memory (norm_resident.cuh) or rows that begin anywhere.
// Device code; included by layers.cuh inside its unnamed namespace.
//
//   xhat = (x - mean) rstd,  z = xhat weight + bias,  y = act(z)
//   dz = dy act'(z),  dx = rstd (dz weight - (s1 + xhat s2) / N),  s1 = sum dz weight,  s2 = sum dz weight xhat  over the group
//
// Everything that is summed is summed for each channel first, then over the channels of a group: one walk over the pixels serves any
// number of channels a group, and the gradient's channel sums are dbias and dweight.  Bound: memory, with the issue of instructions close
// behind (of the 176 and 264 slots that an SM's quarter has for eight bf16 elements at the copy rate, silu's forward pass takes about 130 and its
// gradient 270, with 96 and 192 cycles of the special functions' pipe): two floats an instruction, approximations by single instructions.
//
// The kernels in several walks: 512 x 512 x 128 in bf16 with silu, 53 us forward (moments 21, join 5, result 23; floor 20) and 85 backward (sums
// 35, joins 8, result 42; floor 31): latency, at 15 to 28 warps an SM with four or eight loads of each thread under way.
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
    float *sums[2];                                    // of dz and dz * xhat of each sample, or null
    long long sums_sample[2];                          // from one sample's to the next's
    int n, samples, channels, groups, per_group, act;
    long long pixels;
    float eps;
    int tx, col_blocks, chunks;                        // tx: column vectors of a block of 256 threads
    long long chunk_pixels;
    Draw draw;
};

// f(act as a constant): loops with the activation inside are compiled once for each.
template <typename F> __device__ __forceinline__ void with_act(int act, F f) {
    if (act == kActSilu)
        f(std::integral_constant<int, kActSilu>());
    else if (act == kActRelu)
        f(std::integral_constant<int, kActRelu>());
    else
        f(std::integral_constant<int, kActNone>());
}

// 1 / (1 + exp(-z)) of two numbers by the exponential and the reciprocal that are instructions, each good to about 2^-22: as good as the
// rounding of z in 32 bits lets it be, and far below that of 16-bit results.  One reciprocal of the product serves both (of a silu gradient's
// time the special functions' pipe was the largest part: 8 x 16 x 56 x 56 x 256 forward 96 -> 91 us).  The factors are made 2^63 times
// smaller, so that the product of any two that are numbers is one, and so is its reciprocal; results below 2^-126 become 0 (exponentials ended
// at 2^60 saved a multiplication, and 2 % of that gradient's time, but left 2^-60 below z = -41; a branch for those cost 4 %).  NaN counts as
// the largest exponential, which leaves the other number alone, and stays in z.  e: exp(-z), so that e times the result is 1 minus it,
// without a difference of nearly equal numbers.
__device__ __forceinline__ F2 sigmoid(F2 z, F2 &e) {
    const F2 t = z * two(-1.4426950408889634f);
    float p = t.x, q = t.y;
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(p));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(q));
    e = F2{fminf(p, 0x1p127f), fminf(q, 0x1p127f)};
    const F2 s = fma2(e, two(0x1p-63f), two(0x1p-63f));
    float r = s.x * s.y;
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(r));
    unsigned long long g;
    asm("mul.rn.ftz.f32x2 %0, %1, %2;" : "=l"(g) : "l"(bits_of(F2{s.y, s.x} * two(r))), "l"(bits_of(two(0x1p-63f))));
    return pair_of(g);
}
// NaN stays NaN.
__device__ __forceinline__ float relu(float v, float z) { return z <= 0.f ? 0.f : v; }

template <int ACT> __device__ __forceinline__ F2 activate(F2 z) {
    F2 e;
    if (ACT == kActSilu) return z * sigmoid(z, e);
    if (ACT == kActRelu) return {relu(z.x, z.x), relu(z.y, z.y)};
    return z;
}
// dy * act'(z)
template <int ACT> __device__ __forceinline__ F2 slope_times(F2 dy, F2 z) {
    if (ACT == kActSilu) {
        F2 e;
        const F2 g = sigmoid(z, e);
        return dy * (g * fma2(z, e * g, two(1.f)));
    }
    if (ACT == kActRelu) return {relu(dy.x, z.x), relu(dy.y, z.y)};
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

// Sums of a few values of each of V channels, relative to the first of them, which keeps sums of squares from cancelling: that value is one of
// the set, so what is subtracted is at most as many times what is left as there are values, wherever the mean is.
template <int V> struct Batch {
    F2 first[kPairs<V>], sum[kPairs<V>], squares[kPairs<V>];

    __device__ __forceinline__ Batch() {
#pragma unroll
        for (int j = 0; j < kPairs<V>; ++j) first[j] = sum[j] = squares[j] = two(0.f);
    }
    __device__ __forceinline__ void begin(const F2 (&f)[kPairs<V>]) {
#pragma unroll
        for (int j = 0; j < kPairs<V>; ++j) first[j] = f[j], sum[j] = squares[j] = two(0.f);
    }
    __device__ __forceinline__ void add(const F2 (&f)[kPairs<V>]) {
#pragma unroll
        for (int j = 0; j < kPairs<V>; ++j) {
            const F2 d = f[j] - first[j];
            sum[j] = sum[j] + d, squares[j] = fma2(d, d, squares[j]);
        }
    }
    // Mean and sum of squares about it of `count` values, in the places of first and squares.
    __device__ __forceinline__ void end(int count) {
        const float part = count ? 1.f / count : 0.f;
#pragma unroll
        for (int j = 0; j < kPairs<V>; ++j) {
            const F2 s = sum[j] * two(part);
            first[j] = first[j] + s, squares[j] = fma2(sum[j], s * two(-1.f), squares[j]);
        }
    }
};

// Joins sets of N means and sums of squares, n * fold values behind each, of the threads of a warp whose lanes differ in bits `span` and above.
template <int N> __device__ __forceinline__ void join_lanes(float &n, float (&mean)[N], float (&m2)[N], int fold, int span) {
    for (int o = span; o < 32; o <<= 1) {
        const float n2 = __shfl_xor_sync(~0u, n, o), total = n + n2;
        const bool upper = threadIdx.x & o;                                         // the lower lane's set comes first in both
        const float share = total == 0.f ? 0.f : __fdividef(upper ? n : n2, total), weight = fold * (upper ? n2 : n) * share;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float other = __shfl_xor_sync(~0u, mean[j], o), q = __shfl_xor_sync(~0u, m2[j], o);
            const float low = upper ? other : mean[j], d = (upper ? mean[j] : other) - low;
            mean[j] = fmaf(d, share, low), m2[j] = fmaf(d * d, weight, m2[j] + q);
        }
        n = total;
    }
}

// Drops out what a worker's array has from element e on: dropped elements become 0, others stay (times the factor later); keep bits.
template <typename T, int V> __device__ __forceinline__ uint32_t drop_out(Vec<T, V> &v, const Draw &draw, const Words &words, long long e) {
    const Drawn<V, V % 4 == 0> d(words, e);
    uint32_t keep = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const bool kept = d.w[j] >= draw.threshold;
        if (!kept) v.at[j] = from_float<T>(0.f);
        keep |= (uint32_t)kept << j;
    }
    return keep;
}
// Values as they count.
template <typename T, int V, bool DROP> __device__ __forceinline__ void counted(F2 (&f)[kPairs<V>], const Vec<T, V> &v, float factor) {
    pairs_of(v, f);
    if (DROP) {
#pragma unroll
        for (int j = 0; j < kPairs<V>; ++j) f[j] = f[j] * two(factor);
    }
}

// A thread's channels: z = x * scale + shift.  (One rounding more than (x - mean) rstd weight + bias has, of the size of that of the mean.)
template <int V> struct Channels {
    F2 scale[kPairs<V>], shift[kPairs<V>], minus_mean[kPairs<V>];
};
template <typename T, int V> __device__ __forceinline__ void channels_of(Channels<V> &k, const NormArgs<T> &a, int w, int b, int c) {
    const float *means = a.stats + ((long long)w * a.samples + b) * a.groups, *rstds = means + (long long)a.n * a.samples * a.groups;
    float v[3][2 * kPairs<V>] = {};
    int g = c / a.per_group, left = a.per_group - (c - g * a.per_group);        // channels of the group from here on
#pragma unroll
    for (int j = 0; j < V; ++j) {
        if (left == 0) ++g, left = a.per_group;
        --left;
        v[2][j] = -means[g];
        v[0][j] = rstds[g] * (a.weight ? a.weight[w * a.weight_worker + c + j] : 1.f);
        v[1][j] = fmaf(v[2][j], v[0][j], a.bias ? a.bias[w * a.bias_worker + c + j] : 0.f);
    }
#pragma unroll
    for (int j = 0; j < kPairs<V>; ++j) {
        k.scale[j] = {v[0][2 * j], v[0][2 * j + 1]}, k.shift[j] = {v[1][2 * j], v[1][2 * j + 1]};
        k.minus_mean[j] = {v[2][2 * j], v[2][2 * j + 1]};
    }
}

// Sums dz and dz * (x - mean) of a vector.
template <typename T, int V, bool DROP, int ACT>
__device__ __forceinline__ void add_grad(F2 (&s0)[kPairs<V>], F2 (&s1)[kPairs<V>], const Channels<V> &k, const Vec<T, V> &vx, const Vec<T, V> &vd,
                                         float factor) {
    F2 f[kPairs<V>], d[kPairs<V>];
    counted<T, V, DROP>(f, vx, factor);
    pairs_of(vd, d);
#pragma unroll
    for (int j = 0; j < kPairs<V>; ++j) {
        const F2 dz = slope_times<ACT>(d[j], fma2(f[j], k.scale[j], k.shift[j]));
        s0[j] = s0[j] + dz, s1[j] = fma2(dz, f[j] + k.minus_mean[j], s1[j]);
    }
}
// dx of a vector, into vx: dz * scale + x * m2 + m1, with m2 = -rstd^2 s2 / N and m1 = -rstd s1 / N - mean m2.
template <typename T, int V, bool DROP, int ACT>
__device__ __forceinline__ void make_grad(Vec<T, V> &vx, const F2 (&scale)[kPairs<V>], const F2 (&shift)[kPairs<V>], const F2 (&m1)[kPairs<V>],
                                          const F2 (&m2)[kPairs<V>], const Vec<T, V> &vd, float factor, uint32_t keep) {
    F2 f[kPairs<V>], d[kPairs<V>];
    counted<T, V, DROP>(f, vx, factor);
    pairs_of(vd, d);
#pragma unroll
    for (int j = 0; j < kPairs<V>; ++j) {
        const F2 dz = slope_times<ACT>(d[j], fma2(f[j], scale[j], shift[j]));
        f[j] = fma2(dz, scale[j], fma2(f[j], m2[j], m1[j]));
        if (DROP) f[j] = {keep >> 2 * j & 1 ? f[j].x * factor : 0.f, keep >> (2 * j + 1) & 1 ? f[j].y * factor : 0.f};
    }
    round_pairs(vx, f);
}

// ------------------------------------------------------------------ in several walks
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
// The thread's element of pixel i.
template <typename T> __device__ __forceinline__ T *at_pixel(T *p, const View &v, const Place &s, long long i) {
    return p + s.w * v.worker + s.b * v.sample + i * v.pixel + s.c;
}
// Its place in the worker's array, as the dropout counts.
template <typename T> __device__ __forceinline__ long long element(const NormArgs<T> &a, const Place &s, long long i) {
    return (s.b * a.pixels + i) * a.channels + s.c;
}
constexpr int kTogether = 4, kBatch = 32;              // pixels whose loads are under way together; and whose moments are taken together

// Moments of each channel over a chunk of a sample's pixels: plane 0 the mean, plane 1 the sum of squares about it.
template <typename T, int V, bool DROP>
__global__ void __launch_bounds__(256) norm_moments_kernel(NormArgs<T> a) {
    after_previous();
    let_next();
    const Place p = place<T, V>(a);
    const Words words(a.draw, p.w);
    constexpr int U = 2 * kTogether;
    float n = 0.f, mean[V], m2[V];
#pragma unroll
    for (int j = 0; j < V; ++j) mean[j] = m2[j] = 0.f;
    if (p.in) {
        const T *x = at_pixel(a.x, a.xs, p, p.first + p.ty);
        Batch<V> m;
        int got = 0;
        auto join = [&] {
            m.end(got);
            const float total = n + got, share = got / total;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = (j & 1 ? m.first[j / 2].y : m.first[j / 2].x) - mean[j];
                mean[j] = fmaf(d, share, mean[j]), m2[j] = fmaf(d * d, n * share, m2[j] + (j & 1 ? m.squares[j / 2].y : m.squares[j / 2].x));
            }
            n = total, got = 0;
        };
        for (long long i = p.first + p.ty; i < p.last; i += U * p.rows, x += U * p.rows * a.xs.pixel) {
            Vec<T, V> v[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * p.rows < p.last) v[u] = Vec<T, V>(x + u * p.rows * a.xs.pixel);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * p.rows < p.last) {
                    if (DROP) drop_out(v[u], a.draw, words, element(a, p, i + u * p.rows));
                    F2 f[kPairs<V>];
                    counted<T, V, DROP>(f, v[u], a.draw.factor);
                    if (got == 0) m.begin(f);
                    m.add(f);
                    ++got;
                }
            if (got == kBatch) join();
        }
        if (got) join();
    }
    // Threads of the same channels: those of a warp, then the eight warps.
    join_lanes(n, mean, m2, 1, a.tx);
    __shared__ float count[8][32], means[8][32 * V], squares[8][32 * V];
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

// Sum over a block of whole warps, for all of its threads.
__device__ __forceinline__ float block_sum(float v) {
    __shared__ float sums[32];
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    if (blockDim.x == 32) return v;
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = v;
    __syncthreads();
    v = (threadIdx.x & 31) < blockDim.x / 32 ? sums[threadIdx.x & 31] : 0.f;
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    __syncthreads();
    return v;
}
// What a group's parts are: f(where, chunk, channel of the group) for a thread's share of them.
template <typename T, typename F> __device__ __forceinline__ void group_parts(const NormArgs<T> &a, long long group, F f) {
    const long long base = group / a.groups * a.chunks * a.channels + (group % a.groups) * a.per_group;
    for (int i = threadIdx.x; i < a.chunks * a.per_group; i += blockDim.x) {
        const int chunk = i / a.per_group, c = i - chunk * a.per_group;
        f(base + (long long)chunk * a.channels + c, chunk, c);
    }
}

// Mean and rstd of each group from its channels' moments: a block a group.
template <typename T> __global__ void __launch_bounds__(1024) norm_join_moments_kernel(NormArgs<T> a) {
    after_previous();
    let_next();
    const long long g = blockIdx.x;
    auto pixels = [&](int chunk) {
        const long long left = a.pixels - chunk * a.chunk_pixels;
        return (float)(left < a.chunk_pixels ? left : a.chunk_pixels);
    };
    float sum = 0.f, squares = 0.f;
    const float of = 1.f / ((float)a.pixels * a.per_group);
    group_parts(a, g, [&](long long at, int chunk, int) { sum = fmaf(pixels(chunk), a.part[at], sum); });
    const float mean = block_sum(sum) * of;
    group_parts(a, g, [&](long long at, int chunk, int) {
        const float d = a.part[at] - mean;
        squares = fmaf(pixels(chunk) * d, d, squares + a.part[a.plane + at]);
    });
    squares = block_sum(squares) * of;
    if (threadIdx.x == 0) a.stats[g] = mean, a.stats[(long long)a.n * a.samples * a.groups + g] = 1.f / sqrtf(squares + a.eps);
}

template <typename T, int V, bool DROP>
__global__ void __launch_bounds__(256) norm_apply_kernel(NormArgs<T> a) {
    after_previous();
    let_next();
    const Place p = place<T, V>(a);
    if (!p.in) return;
    const Words words(a.draw, p.w);
    Channels<V> k;
    channels_of(k, a, p.w, p.b, p.c);
    const T *x = at_pixel(a.x, a.xs, p, p.first + p.ty);
    T *y = at_pixel(a.y, a.ys, p, p.first + p.ty);
    with_act(a.act, [&](auto act) {
        for (long long i = p.first + p.ty; i < p.last; i += kTogether * p.rows, x += kTogether * p.rows * a.xs.pixel, y += kTogether * p.rows * a.ys.pixel) {
            Vec<T, V> v[kTogether];
#pragma unroll
            for (int u = 0; u < kTogether; ++u)
                if (i + u * p.rows < p.last) v[u] = Vec<T, V>(x + u * p.rows * a.xs.pixel);
#pragma unroll
            for (int u = 0; u < kTogether; ++u)
                if (i + u * p.rows < p.last) {
                    if (DROP) drop_out(v[u], a.draw, words, element(a, p, i + u * p.rows));
                    F2 f[kPairs<V>];
                    counted<T, V, DROP>(f, v[u], a.draw.factor);
#pragma unroll
                    for (int j = 0; j < kPairs<V>; ++j) f[j] = activate<decltype(act)::value>(fma2(f[j], k.scale[j], k.shift[j]));
                    round_pairs(v[u], f);
                    v[u].to(y + u * p.rows * a.ys.pixel);
                }
        }
    });
}

// Sums of dz (plane 0) and dz * xhat (plane 1) of each channel over a chunk of a sample's pixels.
template <typename T, int V, bool DROP>
__global__ void __launch_bounds__(256) norm_grad_sums_kernel(NormArgs<T> a) {
    after_previous();
    let_next();
    const Place p = place<T, V>(a);
    const Words words(a.draw, p.w);
    F2 s0[kPairs<V>], s1[kPairs<V>];
#pragma unroll
    for (int j = 0; j < kPairs<V>; ++j) s0[j] = s1[j] = two(0.f);
    if (p.in) {
        Channels<V> k;
        channels_of(k, a, p.w, p.b, p.c);
        const T *x = at_pixel(a.x, a.xs, p, p.first + p.ty), *dy = at_pixel(a.dy, a.dys, p, p.first + p.ty);
        constexpr int U = kTogether;
        with_act(a.act, [&](auto act) {
            for (long long i = p.first + p.ty; i < p.last; i += U * p.rows, x += U * p.rows * a.xs.pixel, dy += U * p.rows * a.dys.pixel) {
                Vec<T, V> vx[U], vd[U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (i + u * p.rows < p.last) vx[u] = Vec<T, V>(x + u * p.rows * a.xs.pixel), vd[u] = Vec<T, V>(dy + u * p.rows * a.dys.pixel);
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (i + u * p.rows < p.last) {
                        if (DROP) drop_out(vx[u], a.draw, words, element(a, p, i + u * p.rows));
                        add_grad<T, V, DROP, decltype(act)::value>(s0, s1, k, vx[u], vd[u], a.draw.factor);
                    }
            }
        });
    }
    float t0[2 * kPairs<V>], t1[2 * kPairs<V>];
#pragma unroll
    for (int j = 0; j < kPairs<V>; ++j) t0[2 * j] = s0[j].x, t0[2 * j + 1] = s0[j].y, t1[2 * j] = s1[j].x, t1[2 * j + 1] = s1[j].y;
    __shared__ float sums[2][8][32 * V];
    for (int o = a.tx; o < 32; o <<= 1)
#pragma unroll
        for (int j = 0; j < V; ++j) t0[j] += __shfl_xor_sync(~0u, t0[j], o), t1[j] += __shfl_xor_sync(~0u, t1[j], o);
    const int warp = threadIdx.x >> 5, tx = threadIdx.x & (a.tx - 1);
    if ((threadIdx.x & 31) < a.tx)
#pragma unroll
        for (int j = 0; j < V; ++j) sums[0][warp][tx * V + j] = t0[j], sums[1][warp][tx * V + j] = t1[j];
    __syncthreads();
    const int k = threadIdx.x, c = (blockIdx.x % a.col_blocks) * a.tx * V + k;
    if (k < a.tx * V && c < a.channels) {
        float u0 = 0.f, u1 = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) u0 += sums[0][i][k], u1 += sums[1][i][k];
        const long long sample = (long long)p.w * a.samples + p.b, at = (sample * a.chunks + p.chunk) * a.channels + c;
        a.part[at] = u0, a.part[a.plane + at] = u1 * a.stats[((long long)a.n * a.samples + sample) * a.groups + c / a.per_group];
    }
}

// s1 / N and s2 / N of each group: a block a group.
template <typename T> __global__ void __launch_bounds__(1024) norm_join_sums_kernel(NormArgs<T> a) {
    after_previous();
    let_next();
    const long long g = blockIdx.x;
    const int w = (int)(g / a.groups / a.samples), c0 = (int)(g % a.groups) * a.per_group;
    float s0 = 0.f, s1 = 0.f;
    group_parts(a, g, [&](long long at, int, int c) {
        const float k = a.weight ? a.weight[w * a.weight_worker + c0 + c] : 1.f;
        s0 = fmaf(a.part[at], k, s0), s1 = fmaf(a.part[a.plane + at], k, s1);
    });
    s0 = block_sum(s0), s1 = block_sum(s1);
    const float of = 1.f / ((float)a.pixels * a.per_group);
    if (threadIdx.x == 0) a.group_sums[g] = make_float2(s0 * of, s1 * of);
}

template <typename T, int V, bool DROP>
__global__ void __launch_bounds__(256) norm_grad_apply_kernel(NormArgs<T> a) {
    after_previous();
    let_next();
    const Place p = place<T, V>(a);
    if (!p.in) return;
    const Words words(a.draw, p.w);
    Channels<V> k;
    channels_of(k, a, p.w, p.b, p.c);
    F2 m1[kPairs<V>], m2[kPairs<V>];
    {
        const long long group0 = ((long long)p.w * a.samples + p.b) * a.groups;
        float v[2][2 * kPairs<V>] = {};
        int g = p.c / a.per_group, left = a.per_group - (p.c - g * a.per_group);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (left == 0) ++g, left = a.per_group;
            --left;
            const float rstd = a.stats[(long long)a.n * a.samples * a.groups + group0 + g];
            const float2 sums = a.group_sums[group0 + g];
            v[1][j] = -rstd * rstd * sums.y, v[0][j] = fmaf(-a.stats[group0 + g], v[1][j], -rstd * sums.x);
        }
#pragma unroll
        for (int j = 0; j < kPairs<V>; ++j) m1[j] = {v[0][2 * j], v[0][2 * j + 1]}, m2[j] = {v[1][2 * j], v[1][2 * j + 1]};
    }
    const T *x = at_pixel(a.x, a.xs, p, p.first + p.ty), *dy = at_pixel(a.dy, a.dys, p, p.first + p.ty);
    T *y = at_pixel(a.y, a.ys, p, p.first + p.ty);
    constexpr int U = 2;
    with_act(a.act, [&](auto act) {
        for (long long i = p.first + p.ty; i < p.last;
             i += U * p.rows, x += U * p.rows * a.xs.pixel, dy += U * p.rows * a.dys.pixel, y += U * p.rows * a.ys.pixel) {
            Vec<T, V> vx[U], vd[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * p.rows < p.last) vx[u] = Vec<T, V>(x + u * p.rows * a.xs.pixel), vd[u] = Vec<T, V>(dy + u * p.rows * a.dys.pixel);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * p.rows < p.last) {
                    const uint32_t keep = DROP ? drop_out(vx[u], a.draw, words, element(a, p, i + u * p.rows)) : 0;
                    make_grad<T, V, DROP, decltype(act)::value>(vx[u], k.scale, k.shift, m1, m2, vd[u], a.draw.factor, keep);
                    vx[u].to(y + u * p.rows * a.ys.pixel);
                }
        }
    });
}
