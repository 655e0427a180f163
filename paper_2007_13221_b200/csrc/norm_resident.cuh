// norm_resident.cuh - group norm in one walk over memory: what a group needs stays in shared memory between its sums and its results.
// Device code; included by layers.cuh inside its unnamed namespace.
//
// A unit of work is a slice of channels (whole groups, 128 bytes of a pixel where that can be had) of one sample; a cluster of up to eight
// blocks shares its pixels.  Every thread copies the vectors that it will work on into slots of its own in shared memory, asynchronously, all
// at once: as many bytes are under way as the block holds, and no thread waits for another's copies.  Sums run over the slots, then across
// the block, then across the cluster through distributed shared memory (the only waits: two cluster barriers), and the results
// are made from the slots.  Each element crosses HBM once in each direction, where separate kernels for sums and results read twice.
#pragma once

struct Resident {
    int sv, log_tx, slices, cluster, slots;            // sv: vectors of a slice; slots: of a thread and array
    long long per;                                     // pixels of a block
};

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// A float of another block of the cluster, at the address that it has here.
__device__ __forceinline__ float of_rank(const float *p, int rank) {
    uint32_t at;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
    return v;
}
template <int BYTES> __device__ __forceinline__ void copy_async(void *to, const void *from) {
    const uint32_t at = (uint32_t)__cvta_generic_to_shared(to);
    if (BYTES == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(from), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// f(act as a constant): loops with the activation inside are compiled once for each.
template <typename F> __device__ __forceinline__ void with_act(int act, F f) {
    if (act == kActSilu)
        f(std::integral_constant<int, kActSilu>());
    else if (act == kActRelu)
        f(std::integral_constant<int, kActRelu>());
    else
        f(std::integral_constant<int, kActNone>());
}

// Where a thread stands, and its parts of the block's shared memory.
template <typename T, int V> struct Stand {
    typedef typename Vec<T, V>::raw raw;
    int w, b, rank, c0, tx, ty, rows, here, mine;      // c0: the slice's first channel; here: its channels; mine: pixels of this thread
    long long first, last, sample;
    bool in;
    raw *x, *dy;                                       // its slots, 256 apart
    uint8_t *keep;                                     // keep bits of its slots, 256 apart
    float *red, *chan, *group;                         // two planes each: rows of sums, channels, groups

    __device__ __forceinline__ Stand(const NormArgs<T> &a, const Resident &r, unsigned char *shared, bool two, bool bits) {
        rank = blockIdx.x % r.cluster;
        const int unit = blockIdx.x / r.cluster, slice = unit % r.slices;
        sample = unit / r.slices;
        w = (int)(sample / a.samples), b = (int)(sample % a.samples);
        c0 = slice * r.sv * V;
        here = a.channels - c0 < r.sv * V ? a.channels - c0 : r.sv * V;
        tx = threadIdx.x & ((1 << r.log_tx) - 1), ty = threadIdx.x >> r.log_tx, rows = 256 >> r.log_tx;
        in = tx * V < here;
        first = rank * r.per, last = first + r.per < a.pixels ? first + r.per : a.pixels;
        const int left = first < last ? (int)(last - first) - ty : 0;
        mine = in && left > 0 ? (left + rows - 1) >> (8 - r.log_tx) : 0;
        x = reinterpret_cast<raw *>(shared) + threadIdx.x;
        dy = x + (two ? r.slots * 256 : 0);
        unsigned char *rest = shared + (size_t)r.slots * 256 * sizeof(raw) * (two ? 2 : 1);
        keep = rest + threadIdx.x;
        if (bits) rest += r.slots * 256;
        red = reinterpret_cast<float *>(rest);
        chan = red + 2 * sum_rows() * width();
        group = chan + 2 * width();
    }
    __device__ __forceinline__ int width() const { return (256 / rows) * V; }                // channels of a row of sums
    __device__ __forceinline__ int sum_rows() const { return rows < 8 ? rows : 8; }
    // Pixels of a block of the cluster.
    __device__ __forceinline__ float pixels_of(const NormArgs<T> &a, const Resident &r, int k) const {
        const long long left = a.pixels - k * r.per;
        return left <= 0 ? 0.f : (float)(left < r.per ? left : r.per);
    }
};
// Bytes of shared memory of the above.
inline size_t resident_shared(const Resident &r, int v, int size, bool two, bool bits) {
    const int rows = 256 >> r.log_tx, width = (1 << r.log_tx) * v;
    return (size_t)r.slots * 256 * (v * size * (two ? 2 : 1) + (bits ? 1 : 0)) + (size_t)(2 * std::min(rows, 8) * width + 4 * width) * 4;
}

template <typename T, int V, bool DROP>
__global__ void __launch_bounds__(256) norm_resident_kernel(NormArgs<T> a, Resident r) {
    extern __shared__ __align__(16) unsigned char shared[];
    after_previous();
    let_next();
    const Stand<T, V> s(a, r, shared, false, false);
    const T *x = a.x + s.w * a.xs.worker + s.b * a.xs.sample + s.c0 + s.tx * V + (s.first + s.ty) * a.xs.pixel;
    for (int u = 0; u < s.mine; ++u, x += s.rows * a.xs.pixel) copy_async<V * sizeof(T)>(s.x + u * 256, x);
    const float factor = DROP ? a.draw.factor : 1.f;
    const Words words(a.draw, s.w);
    float n = (float)s.mine, mean[V], m2[V];
#pragma unroll
    for (int j = 0; j < V; ++j) mean[j] = m2[j] = 0.f;
    copies_done();
    long long e = ((long long)s.b * a.pixels + s.first + s.ty) * a.channels + s.c0 + s.tx * V;
    for (int u = 0; u < s.mine; ++u) {
        Vec<T, V> v;
        v.bits = s.x[u * 256];
        if (DROP) {                                    // dropped elements become 0 in their slot
            const Drawn<V, V % 4 == 0> d(words, e);
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (d.w[j] < a.draw.threshold) v.at[j] = from_float<T>(0.f);
            s.x[u * 256] = v.bits;
            e += (long long)s.rows * a.channels;
        }
        float f[V];
        v.floats(f);
#pragma unroll
        for (int j = 0; j < V; ++j) mean[j] += f[j] * factor;
    }
    const float part = s.mine ? 1.f / n : 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) mean[j] *= part;
    for (int u = 0; u < s.mine; ++u) {
        Vec<T, V> v;
        v.bits = s.x[u * 256];
        float f[V];
        v.floats(f);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = f[j] * factor - mean[j], m2[j] = fmaf(f[j], f[j], m2[j]);
    }
    // Threads of the same channels: those of a warp (the lower lane's set first, so that both end with the same bits) ...
    const int span = 1 << r.log_tx, width = s.width();
    for (int o = span; o < 32; o <<= 1) {
        const float n2 = __shfl_xor_sync(~0u, n, o), total = n + n2;
        const bool upper = threadIdx.x & o;
        const float share = total == 0.f ? 0.f : (upper ? n : n2) / total, weight = (upper ? n2 : n) * share;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float mean2 = __shfl_xor_sync(~0u, mean[j], o), q2 = __shfl_xor_sync(~0u, m2[j], o);
            const float d = upper ? mean[j] - mean2 : mean2 - mean[j];
            mean[j] = fmaf(d, share, upper ? mean2 : mean[j]);
            m2[j] = (m2[j] + q2) + d * d * weight;
        }
        n = total;
    }
    // ... then rows of the block, of which each warp (or part of one) has left one ...
    const int sum_rows = s.sum_rows(), row = s.rows < 8 ? s.ty : threadIdx.x >> 5;
    float *red = s.red, *chan = s.chan;
    if ((threadIdx.x & 31) < span) {
#pragma unroll
        for (int j = 0; j < V; ++j) red[row * width + s.tx * V + j] = mean[j], red[(sum_rows + row) * width + s.tx * V + j] = m2[j];
    }
    __syncthreads();
    const int block_pixels = s.first < s.last ? (int)(s.last - s.first) : 0, each = s.rows / sum_rows;
    for (int k = threadIdx.x; k < s.here; k += 256) {
        float nn = 0.f, mm = 0.f, qq = 0.f;
        for (int i = 0; i < sum_rows; ++i) {
            // Pixels of the threads i * each .. i * each + each - 1 of a column: each of them takes every rows-th.
            const int whole = block_pixels / s.rows, rest = block_pixels % s.rows - i * each;
            join_moments(nn, mm, qq, (float)(whole * each + (rest < 0 ? 0 : rest < each ? rest : each)), red[i * width + k],
                         red[(sum_rows + i) * width + k]);
        }
        chan[k] = mm, chan[width + k] = qq;
    }
    if (r.cluster > 1) cluster_arrive(), cluster_wait();
    else __syncthreads();
    // ... then the blocks of the cluster and the channels of a group: a warp a group.
    const int groups = s.here / a.per_group, lane = threadIdx.x & 31, g0 = s.c0 / a.per_group;
    for (int g = threadIdx.x >> 5; g < groups; g += 8) {
        float nn = 0.f, mm = 0.f, qq = 0.f;
        for (int i = lane; i < r.cluster * a.per_group; i += 32) {
            const int k = i / a.per_group, c = g * a.per_group + i % a.per_group;
            const float mean_k = r.cluster > 1 ? of_rank(chan + c, k) : chan[c], m2_k = r.cluster > 1 ? of_rank(chan + width + c, k) : chan[width + c];
            join_moments(nn, mm, qq, s.pixels_of(a, r, k), mean_k, m2_k);
        }
        for (int o = 1; o < 32; o <<= 1) {
            const float n2 = __shfl_down_sync(~0u, nn, o), mean2 = __shfl_down_sync(~0u, mm, o), q2 = __shfl_down_sync(~0u, qq, o);
            join_moments(nn, mm, qq, n2, mean2, q2);
        }
        if (lane == 0) {
            const float rstd = 1.f / sqrtf(qq / nn + a.eps);
            s.group[g] = mm, s.group[width + g] = rstd;
            if (s.rank == 0) {
                const long long at = s.sample * a.groups + g0 + g;
                a.stats[at] = mm, a.stats[(long long)a.n * a.samples * a.groups + at] = rstd;
            }
        }
    }
    if (r.cluster > 1) cluster_arrive();               // no block leaves while others read its channels
    __syncthreads();
    if (s.mine) {
        float weight[V], bias[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c = s.tx * V + j, g = c / a.per_group;
            mean[j] = s.group[g];
            weight[j] = s.group[width + g] * (a.weight ? a.weight[s.w * a.weight_worker + s.c0 + c] : 1.f);
            bias[j] = a.bias ? a.bias[s.w * a.bias_worker + s.c0 + c] : 0.f;
        }
        T *y = a.y + s.w * a.ys.worker + s.b * a.ys.sample + s.c0 + s.tx * V + (s.first + s.ty) * a.ys.pixel;
        with_act(a.act, [&](auto act) {
            for (int u = 0; u < s.mine; ++u, y += s.rows * a.ys.pixel) {
                Vec<T, V> v;
                v.bits = s.x[u * 256];
                float f[V];
                v.floats(f);
#pragma unroll
                for (int j = 0; j < V; ++j) f[j] = activate(fmaf(f[j] * factor - mean[j], weight[j], bias[j]), decltype(act)::value);
                v.round(f);
                v.to(y);
            }
        });
    }
    if (r.cluster > 1) cluster_wait();
}

template <typename T, int V, bool DROP>
__global__ void __launch_bounds__(256) norm_grad_resident_kernel(NormArgs<T> a, Resident r) {
    extern __shared__ __align__(16) unsigned char shared[];
    after_previous();
    let_next();
    const Stand<T, V> s(a, r, shared, true, DROP);
    const T *x = a.x + s.w * a.xs.worker + s.b * a.xs.sample + s.c0 + s.tx * V + (s.first + s.ty) * a.xs.pixel;
    const T *dy = a.dy + s.w * a.dys.worker + s.b * a.dys.sample + s.c0 + s.tx * V + (s.first + s.ty) * a.dys.pixel;
    for (int u = 0; u < s.mine; ++u, x += s.rows * a.xs.pixel, dy += s.rows * a.dys.pixel) {
        copy_async<V * sizeof(T)>(s.x + u * 256, x);
        copy_async<V * sizeof(T)>(s.dy + u * 256, dy);
    }
    const float factor = DROP ? a.draw.factor : 1.f;
    const Words words(a.draw, s.w);
    Channels<V> k;
    float s0[V], s1[V];
    if (s.in) channels_of(k, a, s.w, s.b, s.c0 + s.tx * V, true);
#pragma unroll
    for (int j = 0; j < V; ++j) s0[j] = s1[j] = 0.f;
    copies_done();
    with_act(a.act, [&](auto act) {
        long long e = ((long long)s.b * a.pixels + s.first + s.ty) * a.channels + s.c0 + s.tx * V;
        for (int u = 0; u < s.mine; ++u) {
            Vec<T, V> vx, vd;
            vx.bits = s.x[u * 256], vd.bits = s.dy[u * 256];
            if (DROP) {
                const Drawn<V, V % 4 == 0> d(words, e);
                uint32_t keep = 0;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const bool kept = d.w[j] >= a.draw.threshold;
                    if (!kept) vx.at[j] = from_float<T>(0.f);
                    keep |= (uint32_t)kept << j;
                }
                s.x[u * 256] = vx.bits, s.keep[u * 256] = (uint8_t)keep;
                e += (long long)s.rows * a.channels;
            }
            float f[V], d[V];
            vx.floats(f), vd.floats(d);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float h = (f[j] * factor - k.mean[j]) * k.rstd[j];
                const float dz = slope_times(d[j], fmaf(h, k.weight[j], k.bias[j]), decltype(act)::value);
                s0[j] += dz, s1[j] = fmaf(dz, h, s1[j]);
            }
        }
    });
    const int span = 1 << r.log_tx, width = s.width();
    for (int o = span; o < 32; o <<= 1)
#pragma unroll
        for (int j = 0; j < V; ++j) s0[j] += __shfl_xor_sync(~0u, s0[j], o), s1[j] += __shfl_xor_sync(~0u, s1[j], o);
    const int sum_rows = s.sum_rows(), row = s.rows < 8 ? s.ty : threadIdx.x >> 5;
    float *red = s.red, *chan = s.chan;
    if ((threadIdx.x & 31) < span) {
#pragma unroll
        for (int j = 0; j < V; ++j) red[row * width + s.tx * V + j] = s0[j], red[(sum_rows + row) * width + s.tx * V + j] = s1[j];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < s.here; c += 256) {
        float t0 = 0.f, t1 = 0.f;
        for (int i = 0; i < sum_rows; ++i) t0 += red[i * width + c], t1 += red[(sum_rows + i) * width + c];
        chan[c] = t0, chan[width + c] = t1;
    }
    if (r.cluster > 1) cluster_arrive(), cluster_wait();
    else __syncthreads();
    if (a.part)                                        // the sample's sums: dbias's and dweight's share; each block writes some channels
        for (int c = s.rank + r.cluster * threadIdx.x; c < s.here; c += r.cluster * 256) {
            float t0 = 0.f, t1 = 0.f;
            for (int i = 0; i < r.cluster; ++i) {
                t0 += r.cluster > 1 ? of_rank(chan + c, i) : chan[c];
                t1 += r.cluster > 1 ? of_rank(chan + width + c, i) : chan[width + c];
            }
            const long long at = s.sample * a.channels + s.c0 + c;
            a.part[at] = t0, a.part[a.plane + at] = t1;
        }
    const int groups = s.here / a.per_group, lane = threadIdx.x & 31;
    const float of = 1.f / ((float)a.pixels * a.per_group);
    for (int g = threadIdx.x >> 5; g < groups; g += 8) {
        float t0 = 0.f, t1 = 0.f;
        for (int i = lane; i < r.cluster * a.per_group; i += 32) {
            const int rank = i / a.per_group, c = g * a.per_group + i % a.per_group;
            const float wt = a.weight ? a.weight[s.w * a.weight_worker + s.c0 + c] : 1.f;
            t0 = fmaf(r.cluster > 1 ? of_rank(chan + c, rank) : chan[c], wt, t0);
            t1 = fmaf(r.cluster > 1 ? of_rank(chan + width + c, rank) : chan[width + c], wt, t1);
        }
        for (int o = 16; o; o >>= 1) t0 += __shfl_xor_sync(~0u, t0, o), t1 += __shfl_xor_sync(~0u, t1, o);
        if (lane == 0) s.group[g] = t0 * of, s.group[width + g] = t1 * of;
    }
    if (r.cluster > 1) cluster_arrive();
    __syncthreads();
    if (s.mine && a.y) {
        float m1[V], m2[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int g = (s.tx * V + j) / a.per_group;
            m1[j] = s.group[g], m2[j] = s.group[width + g];
        }
        T *y = a.y + s.w * a.ys.worker + s.b * a.ys.sample + s.c0 + s.tx * V + (s.first + s.ty) * a.ys.pixel;
        with_act(a.act, [&](auto act) {
            for (int u = 0; u < s.mine; ++u, y += s.rows * a.ys.pixel) {
                Vec<T, V> vx, vd;
                vx.bits = s.x[u * 256], vd.bits = s.dy[u * 256];
                const uint32_t keep = DROP ? s.keep[u * 256] : 0;
                float f[V], d[V];
                vx.floats(f), vd.floats(d);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float h = (f[j] * factor - k.mean[j]) * k.rstd[j];
                    const float dz = slope_times(d[j], fmaf(h, k.weight[j], k.bias[j]), decltype(act)::value);
                    f[j] = k.rstd[j] * (fmaf(dz, k.weight[j], -m1[j]) - h * m2[j]);
                    if (DROP) f[j] = keep >> j & 1 ? f[j] * factor : 0.f;
                }
                vx.round(f);
                vx.to(y);
            }
        });
    }
    if (r.cluster > 1) cluster_wait();
}
