// norm_resident.cuh - group norm in one walk over memory: what a group needs stays in shared memory between its sums and its results.
// Device code; included by layers.cuh inside its unnamed namespace.
//
// A unit of work is a slice of channels (whole groups, 128 bytes of a pixel where that can be had) of one sample; a cluster of up to eight
// blocks shares its pixels.  Every thread copies the vectors that it will work on into slots of its own in shared memory, asynchronously, all
// at once: as many bytes are under way as the block holds, and no thread waits for another's copies.  Sums run over the slots, then across
// the block, then across the cluster through distributed shared memory (the only waits: two cluster barriers), and the results
// are made from the slots.  Each element crosses HBM once in each direction, where separate kernels for sums and results read twice.
#pragma once

constexpr int kBlock = 128, kLogBlock = 7;           // threads
struct Resident {
    int sv, log_tx, log_cluster, slots;                // sv: vectors of a slice; slots: of a thread and array
    int fold, log_sub;                                 // neighbouring channels of a vector that share a group; lanes of a group's sums
    uint32_t group_magic;                              // 2^32 / channels of a group, rounded up; 0 for one
    int per;                                           // pixels of a block
};
// Grid: x: blocks of a cluster for each sample, y: slices.

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// Stores v at p's place in another block of the cluster.
__device__ __forceinline__ void to_rank(float *p, int rank, float v) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(v) : "memory");
}
template <int BYTES> __device__ __forceinline__ void copy_async(void *to, const void *from) {
    const uint32_t at = (uint32_t)__cvta_generic_to_shared(to);
    if (BYTES == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(from), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Where a thread stands, and its parts of the block's shared memory.
template <typename T, int V> struct Stand {
    typedef typename Vec<T, V>::raw raw;
    int w, b, sample, rank, c0, tx, ty, log_rows, here, mine;        // c0: the slice's first channel; here: its channels; mine: pixels of this thread
    int first, last;
    bool in;
    raw *x, *dy;                                       // its slots, kBlock apart
    uint8_t *keep;                                     // keep bits of its slots, kBlock apart
    float *coef, *red, *all;                           // six planes for channels, rows of sums of two planes, two planes of each block of the cluster

    __device__ __forceinline__ Stand(const NormArgs<T> &a, const Resident &r, unsigned char *shared, bool two, bool bits) {
        rank = blockIdx.x & ((1 << r.log_cluster) - 1), sample = blockIdx.x >> r.log_cluster;
        w = (unsigned)sample / (unsigned)a.samples, b = sample - w * a.samples;
        c0 = blockIdx.y * r.sv * V;
        here = a.channels - c0 < r.sv * V ? a.channels - c0 : r.sv * V;
        log_rows = kLogBlock - r.log_tx;
        tx = threadIdx.x & ((1 << r.log_tx) - 1), ty = threadIdx.x >> r.log_tx;
        in = tx * V < here;
        const long long begin = (long long)rank * r.per;
        first = begin < a.pixels ? (int)begin : (int)a.pixels, last = begin + r.per < a.pixels ? (int)begin + r.per : (int)a.pixels;
        const int left = last - first - ty;
        mine = in && left > 0 ? (left + (1 << log_rows) - 1) >> log_rows : 0;
        x = reinterpret_cast<raw *>(shared) + threadIdx.x;
        dy = x + (two ? r.slots * kBlock : 0);
        unsigned char *rest = shared + (size_t)r.slots * kBlock * sizeof(raw) * (two ? 2 : 1);
        keep = rest + threadIdx.x;
        if (bits) rest += r.slots * kBlock;
        coef = reinterpret_cast<float *>(rest);
        red = coef + 6 * width();
        all = red + 2 * sum_rows() * width();
    }
    __device__ __forceinline__ int width() const { return (kBlock >> log_rows) * V; }        // channels of a row of sums
    __device__ __forceinline__ int sum_rows() const { return log_rows < kLogBlock - 5 ? 1 << log_rows : kBlock / 32; }
    __device__ __forceinline__ long long step(const View &v) const { return v.pixel << log_rows; }
    template <typename U> __device__ __forceinline__ U *at(U *p, const View &v) const {
        return p + w * v.worker + b * v.sample + (first + ty) * v.pixel + c0 + tx * V;
    }
    // A thread's channels of a plane of coef.
    __device__ __forceinline__ void channels(F2 (&k)[kPairs<V>], int plane) const {
        const float *p = coef + plane * width() + tx * V;
        if (V == 1) {
            k[0] = {p[0], 0.f};
        } else {
#pragma unroll
            for (int j = 0; j < kPairs<V>; ++j) k[j] = pair_of(reinterpret_cast<const unsigned long long *>(p)[j]);
        }
    }
};
// Bytes of shared memory of the above.
inline size_t resident_shared(const Resident &r, int v, int size, bool two, bool bits) {
    const int width = (1 << r.log_tx) * v, rows = std::min(kBlock >> r.log_tx, kBlock / 32);
    return (size_t)r.slots * kBlock * (v * size * (two ? 2 : 1) + (bits ? 1 : 0)) + (size_t)(6 + 2 * rows + (2 << r.log_cluster)) * width * 4;
}

// Leaves a thread's N sums (lanes joined already) for the block: row of sums, two planes.
template <int N> __device__ __forceinline__ void leave_row(float *red, int log_tx, int log_rows, const float (&p)[N], const float (&q)[N]) {
    const int sums = N << log_tx, rows = min(kBlock >> log_tx, kBlock / 32), row = log_tx > 5 ? threadIdx.x >> log_tx : threadIdx.x >> 5;
    if (log_tx >= 5 || (threadIdx.x & 31) < 1 << log_tx) {
        float *a = red + row * sums + (threadIdx.x & ((1 << log_tx) - 1)) * N, *b = a + rows * sums;
#pragma unroll
        for (int j = 0; j < N; ++j) a[j] = p[j], b[j] = q[j];
    }
}
// Two numbers of place k for all blocks of the cluster.
__device__ __forceinline__ void tell_all(const Resident &r, float *all, int rank, int sums, int k, float p, float q) {
    float *at = all + 2 * rank * sums + k;
    if (r.log_cluster == 0) {
        at[0] = p, at[sums] = q;
    } else {
        for (int i = 0; i < 1 << r.log_cluster; ++i) to_rank(at, i, p), to_rank(at + sums, i, q);
    }
}
// The blocks of a cluster, or the threads of a block of its own.
__device__ __forceinline__ void meet(const Resident &r) {
    if (r.log_cluster)
        cluster_arrive(), cluster_wait();
    else
        __syncthreads();
}
// Sum over aligned groups of 2^log_sub lanes.
__device__ __forceinline__ float lanes_sum(float v, int log_sub) {
    for (int o = 1; o < 1 << log_sub; o <<= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}
// Slots of a thread: f(first of U slots, their vectors), U at a time, then one by one.
template <int U, int V, typename T, typename L, typename F> __device__ __forceinline__ void walk_slots(int from, int to, L load, F f) {
    int u = from;
    for (; u + U <= to; u += U) {
        Vec<T, V> v[U];
#pragma unroll
        for (int i = 0; i < U; ++i) v[i].bits = load(u + i);
#pragma unroll
        for (int i = 0; i < U; ++i) f(u + i, v[i]);
    }
    for (; u < to; ++u) {
        Vec<T, V> v;
        v.bits = load(u);
        f(u, v);
    }
}

// Forward: moments of the parts of a group that a thread's vector holds, FOLD channels each, over the lanes, the block and the cluster.
template <int FOLD, int V> __device__ __forceinline__ void fold_moments(float (&mean)[V / FOLD], float (&m2)[V / FOLD], const Moments<V> &m) {
    constexpr float kOf = 1.f / FOLD;
#pragma unroll
    for (int i = 0; i < V / FOLD; ++i) {
        float f[FOLD], sum = 0.f, squares = 0.f, off = 0.f;
#pragma unroll
        for (int j = 0; j < FOLD; ++j) {
            const int c = i * FOLD + j;
            f[j] = c & 1 ? m.mean[c / 2].y : m.mean[c / 2].x;
            sum += f[j], squares += c & 1 ? m.m2[c / 2].y : m.m2[c / 2].x;
        }
        mean[i] = sum * kOf;
#pragma unroll
        for (int j = 0; j < FOLD; ++j) off = fmaf(f[j] - mean[i], f[j] - mean[i], off);
        m2[i] = fmaf(m.n, off, squares);
    }
}
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
// f(FOLD as a constant), for the powers of two up to V.
template <int V, typename F> __device__ __forceinline__ void with_fold(int fold, F f) {
    if (V >= 8 && fold == 8)
        f(std::integral_constant<int, V >= 8 ? 8 : 1>());
    else if (V >= 4 && fold == 4)
        f(std::integral_constant<int, V >= 4 ? 4 : 1>());
    else if (V >= 2 && fold == 2)
        f(std::integral_constant<int, V >= 2 ? 2 : 1>());
    else
        f(std::integral_constant<int, 1>());
}

template <typename T, int V, bool DROP>
__global__ void __launch_bounds__(kBlock) norm_resident_kernel(NormArgs<T> a, Resident r) {
    extern __shared__ __align__(16) unsigned char shared[];
    if (r.log_cluster) cluster_arrive();
    after_previous();
    let_next();
    const Stand<T, V> s(a, r, shared, false, false);
    const int width = s.width(), lane = threadIdx.x & 31;
    {
        const T *x = s.at(a.x, a.xs);
        const long long step = s.step(a.xs);
        for (int u = 0; u < s.mine; ++u, x += step) copy_async<V * sizeof(T)>(s.x + u * kBlock, x);
    }
    for (int c = threadIdx.x; c < s.here; c += kBlock) {               // planes 2 and 3: weight and bias
        s.coef[2 * width + c] = a.weight ? a.weight[s.w * a.weight_worker + s.c0 + c] : 1.f;
        s.coef[3 * width + c] = a.bias ? a.bias[s.w * a.bias_worker + s.c0 + c] : 0.f;
    }
    const Words words(a.draw, s.w);
    Moments<V> m;
    const long long e0 = ((long long)s.b * a.pixels + s.first + s.ty) * a.channels + s.c0 + s.tx * V, e_step = (long long)a.channels << s.log_rows;
    copies_done();
    for (int u0 = 0; u0 < s.mine; u0 += kBatch) {
        const int u1 = u0 + kBatch < s.mine ? u0 + kBatch : s.mine;
        walk_slots<DROP ? 2 : 4, V, T>(u0, u1, [&](int u) { return s.x[u * kBlock]; }, [&](int u, Vec<T, V> &v) {
            if (DROP) {                                // dropped elements become 0 in their slot
                drop_out(v, a.draw, words, e0 + u * e_step);
                s.x[u * kBlock] = v.bits;
            }
            F2 f[kPairs<V>];
            counted<T, V, DROP>(f, v, a.draw.factor);
            if (u == u0) m.begin(f);
            m.add(f);
        });
        m.end(u1 - u0);
    }
    // Threads of the same channels: those of a warp, then rows of the block, of which each warp (or part of one) has left one, ...
    with_fold<V>(r.fold, [&](auto fold) {
        constexpr int kFold = decltype(fold)::value;
        float mean[V / kFold], m2[V / kFold];
        fold_moments<kFold, V>(mean, m2, m);
        join_lanes(m.n, mean, m2, kFold, 1 << r.log_tx);
        leave_row(s.red, r.log_tx, s.log_rows, mean, m2);
    });
    __syncthreads();
    const int sums = width / r.fold, sum_rows = s.sum_rows(), block_pixels = s.last - s.first, each = (1 << s.log_rows) / sum_rows;
    const int whole = (block_pixels >> s.log_rows) * each, rest = block_pixels & ((1 << s.log_rows) - 1), mine = s.here / r.fold;
    const float of_block = block_pixels ? 1.f / block_pixels : 0.f;
    if (r.log_cluster) cluster_wait();                 // all blocks are there
    for (int k = threadIdx.x; k < mine; k += kBlock) {
        // Pixels of the threads i * each .. i * each + each - 1 of a column: each of them takes every rows-th.
        auto count = [&](int i) { return (float)(whole + min(max(rest - i * each, 0), each)); };
        float sum = 0.f, squares = 0.f, off = 0.f;
        for (int i = 0; i < sum_rows; ++i) sum = fmaf(count(i), s.red[i * sums + k], sum);
        const float mean = sum * of_block;
        for (int i = 0; i < sum_rows; ++i) {
            const float d = s.red[i * sums + k] - mean;
            off = fmaf(count(i) * d, d, off), squares += s.red[(sum_rows + i) * sums + k];
        }
        tell_all(r, s.all, s.rank, sums, k, mean, fmaf((float)r.fold, off, squares));
    }
    meet(r);
    // ... then the blocks of the cluster and the parts of a group, by 2^log_sub lanes a group.
    const int parts = a.per_group / r.fold, groups = s.here / a.per_group, g0 = s.c0 / a.per_group;
    const float of_group = 1.f / ((float)a.pixels * a.per_group);
    for (int base = threadIdx.x >> 5 << (5 - r.log_sub); base < groups; base += kBlock >> r.log_sub) {
        const int g = base + (lane >> r.log_sub), sub = lane & ((1 << r.log_sub) - 1), entries = g < groups ? parts << r.log_cluster : 0;
        auto values = [&](int i, float &pixels, float &mean, float &m2) {
            const int rank = i & ((1 << r.log_cluster) - 1), k = g * parts + (i >> r.log_cluster);
            pixels = (float)(r.fold * min(max((int)a.pixels - rank * r.per, 0), r.per));
            mean = s.all[2 * rank * sums + k], m2 = s.all[(2 * rank + 1) * sums + k];
        };
        float sum = 0.f, squares = 0.f, p, q, v;
        for (int i = sub; i < entries; i += 1 << r.log_sub) values(i, p, q, v), sum = fmaf(p, q, sum);
        const float mean = lanes_sum(sum, r.log_sub) * of_group;
        for (int i = sub; i < entries; i += 1 << r.log_sub) values(i, p, q, v), squares = fmaf(p * (q - mean), q - mean, squares + v);
        const float rstd = 1.f / sqrtf(lanes_sum(squares, r.log_sub) * of_group + a.eps);
        if (g < groups) {
            for (int c = g * a.per_group + sub; c < (g + 1) * a.per_group; c += 1 << r.log_sub) {          // planes 0 and 1: factor and summand
                const float scale = rstd * s.coef[2 * width + c];
                s.coef[c] = DROP ? scale * a.draw.factor : scale, s.coef[width + c] = fmaf(-mean, scale, s.coef[3 * width + c]);
            }
            if (sub == 0 && s.rank == 0) {
                const long long at = (long long)s.sample * a.groups + g0 + g;
                a.stats[at] = mean, a.stats[(long long)a.n * a.samples * a.groups + at] = rstd;
            }
        }
    }
    __syncthreads();
    if (s.mine) {
        F2 scale[kPairs<V>], shift[kPairs<V>];
        s.channels(scale, 0), s.channels(shift, 1);
        T *y = s.at(a.y, a.ys);
        const long long step = s.step(a.ys);
        with_act(a.act, [&](auto act) {
            walk_slots<4, V, T>(0, s.mine, [&](int u) { return s.x[u * kBlock]; }, [&](int, Vec<T, V> &v) {
                F2 f[kPairs<V>];
                pairs_of(v, f);
#pragma unroll
                for (int j = 0; j < kPairs<V>; ++j) f[j] = activate<decltype(act)::value>(fma2(f[j], scale[j], shift[j]));
                round_pairs(v, f);
                v.to(y);
                y += step;
            });
        });
    }
}

template <typename T, int V, bool DROP>
__global__ void __launch_bounds__(kBlock) norm_grad_resident_kernel(NormArgs<T> a, Resident r) {
    extern __shared__ __align__(16) unsigned char shared[];
    if (r.log_cluster) cluster_arrive();
    after_previous();
    let_next();
    const Stand<T, V> s(a, r, shared, true, DROP);
    const int width = s.width(), lane = threadIdx.x & 31;
    {
        const T *x = s.at(a.x, a.xs), *dy = s.at(a.dy, a.dys);
        const long long x_step = s.step(a.xs), dy_step = s.step(a.dys);
        for (int u = 0; u < s.mine; ++u, x += x_step, dy += dy_step) {
            copy_async<V * sizeof(T)>(s.x + u * kBlock, x);
            copy_async<V * sizeof(T)>(s.dy + u * kBlock, dy);
        }
    }
    // Planes: xhat = x * [0] + [1], z = xhat * [2] + [3].  With a dropout [0] carries its factor.
    for (int c = threadIdx.x; c < s.here; c += kBlock) {
        const int g = r.group_magic ? __umulhi(s.c0 + c, r.group_magic) : s.c0 + c;
        const long long at = (long long)s.sample * a.groups + g;
        const float mean = a.stats[at], rstd = a.stats[(long long)a.n * a.samples * a.groups + at];
        s.coef[c] = DROP ? rstd * a.draw.factor : rstd, s.coef[width + c] = -mean * rstd;
        s.coef[2 * width + c] = a.weight ? a.weight[s.w * a.weight_worker + s.c0 + c] : 1.f;
        s.coef[3 * width + c] = a.bias ? a.bias[s.w * a.bias_worker + s.c0 + c] : 0.f;
    }
    const Words words(a.draw, s.w);
    Channels<V> k;
    F2 s0[kPairs<V>], s1[kPairs<V>];
#pragma unroll
    for (int j = 0; j < kPairs<V>; ++j) s0[j] = s1[j] = two(0.f);
    copies_done();
    __syncthreads();
    s.channels(k.rstd, 0), s.channels(k.offset, 1), s.channels(k.weight, 2), s.channels(k.bias, 3);
    const long long e0 = ((long long)s.b * a.pixels + s.first + s.ty) * a.channels + s.c0 + s.tx * V, e_step = (long long)a.channels << s.log_rows;
    with_act(a.act, [&](auto act) {
        walk_slots<2, V, T>(0, s.mine, [&](int u) { return s.x[u * kBlock]; }, [&](int u, Vec<T, V> &vx) {
            Vec<T, V> vd;
            vd.bits = s.dy[u * kBlock];
            if (DROP) {
                s.keep[u * kBlock] = (uint8_t)drop_out(vx, a.draw, words, e0 + u * e_step);
                s.x[u * kBlock] = vx.bits;
            }
            add_grad<T, V, false, decltype(act)::value>(s0, s1, k, vx, vd, 1.f);
        });
    });
    float t0[V], t1[V];
#pragma unroll
    for (int j = 0; j < V; ++j) t0[j] = j & 1 ? s0[j / 2].y : s0[j / 2].x, t1[j] = j & 1 ? s1[j / 2].y : s1[j / 2].x;
    for (int o = 1 << r.log_tx; o < 32; o <<= 1)
#pragma unroll
        for (int j = 0; j < V; ++j) t0[j] += __shfl_xor_sync(~0u, t0[j], o), t1[j] += __shfl_xor_sync(~0u, t1[j], o);
    leave_row(s.red, r.log_tx, s.log_rows, t0, t1);
    __syncthreads();
    const int sum_rows = s.sum_rows();
    if (r.log_cluster) cluster_wait();                 // all blocks are there
    for (int c = threadIdx.x; c < s.here; c += kBlock) {
        float p = 0.f, q = 0.f;
        for (int i = 0; i < sum_rows; ++i) p += s.red[i * width + c], q += s.red[(sum_rows + i) * width + c];
        tell_all(r, s.all, s.rank, width, c, p, q);
    }
    meet(r);
    // Sums over the cluster; of a channel they are the sample's share of dbias and dweight (each block writes some channels'), times the weight
    // of its group's s1 and s2, which planes 4 and 5 take.
    for (int c = threadIdx.x; c < s.here; c += kBlock) {
        float p = 0.f, q = 0.f;
        for (int i = 0; i < 1 << r.log_cluster; ++i) p += s.all[2 * i * width + c], q += s.all[(2 * i + 1) * width + c];
        if (a.part && (c & ((1 << r.log_cluster) - 1)) == s.rank) {
            const long long at = (long long)s.sample * a.channels + s.c0 + c;
            a.part[at] = p, a.part[a.plane + at] = q;
        }
        s.coef[4 * width + c] = p * s.coef[2 * width + c], s.coef[5 * width + c] = q * s.coef[2 * width + c];
    }
    if (!a.y) return;
    __syncthreads();
    // The first two rows of sums, which all have read, become planes for -rstd s1 / N and -rstd s2 / N, with dx's own factor of a dropout in rstd.
    const int groups = s.here / a.per_group;
    const float of = -1.f / ((float)a.pixels * a.per_group);
    for (int base = threadIdx.x >> 5 << (5 - r.log_sub); base < groups; base += kBlock >> r.log_sub) {
        const int g = base + (lane >> r.log_sub), sub = lane & ((1 << r.log_sub) - 1), end = g < groups ? (g + 1) * a.per_group : 0;
        float p = 0.f, q = 0.f;
        for (int c = g * a.per_group + sub; c < end; c += 1 << r.log_sub) p += s.coef[4 * width + c], q += s.coef[5 * width + c];
        p = lanes_sum(p, r.log_sub) * of, q = lanes_sum(q, r.log_sub) * of;
        for (int c = g * a.per_group + sub; c < end; c += 1 << r.log_sub) s.red[c] = s.coef[c] * p, s.red[width + c] = s.coef[c] * q;
    }
    __syncthreads();
    if (s.mine) {
        F2 scale[kPairs<V>], m1[kPairs<V>], m2[kPairs<V>];
        s.channels(m1, 6), s.channels(m2, 7);
#pragma unroll
        for (int j = 0; j < kPairs<V>; ++j) scale[j] = k.rstd[j] * k.weight[j];
        T *y = s.at(a.y, a.ys);
        const long long step = s.step(a.ys);
        with_act(a.act, [&](auto act) {
            walk_slots<2, V, T>(0, s.mine, [&](int u) { return s.x[u * kBlock]; }, [&](int u, Vec<T, V> &vx) {
                Vec<T, V> vd;
                vd.bits = s.dy[u * kBlock];
                make_grad<T, V, false, decltype(act)::value>(vx, k, scale, m1, m2, vd, 1.f, 0);
                if (DROP) {
                    const uint32_t keep = s.keep[u * kBlock];
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        if (!(keep >> j & 1)) vx.at[j] = from_float<T>(0.f);
                }
                vx.to(y);
                y += step;
            });
        });
    }
}
