// norm_resident.cuh - group norm in one walk over memory: what a group needs stays in shared memory between its sums and its results.
// Device code; included by layers.cuh inside its unnamed namespace.
//
// A unit of work is a slice of channels (whole groups, 64 bytes of a pixel or more) of one sample; one block, or a cluster of up to eight, shares
// its pixels.  Every thread copies the vectors that it will work on into slots of its own in shared memory, asynchronously, all at once: as
// many bytes are under way as the block holds, and no thread waits for another's copies.  Sums run over the slots, then across the
// block; each block of a cluster tells all others its sums (stores to distributed shared memory, one cluster barrier a unit) and
// the results are made from the slots.  Blocks stay: as soon as a vector has been used, the next unit's takes its slot, so that loads run under
// the stores.  Each element crosses HBM once in each direction, where separate kernels for sums and results read twice.
//
// Measured, 8 x 16 samples of 56 x 56 x 256 in bf16, without activation (4.9 TB/s forward, 4.7 backward; what bounds it is the latency of the
// steps between a unit's last load and its first store, on the 16 warps that the registers leave an SM): 3 to 5 walks by kernels of
// their own 638 us for both directions; clusters of eight with reads of each other's sums 368; stores instead, fewer divisions 256; blocks that
// stay, slices of 64 bytes by two and four blocks 214.  With silu 286: 24 exponentials and reciprocals for eight elements of the gradient.
// Tried: 512 threads at 64 registers (spills, forward 93 us for 83), slices of 128 bytes by clusters of eight (100), of 32 by one block (101).
#pragma once

constexpr int kMostThreads = 256;

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

// Where a thread stands, and its parts of the block's shared memory.  `here` and what comes before it change with the unit.
template <typename T, int V> struct Stand {
    typedef typename Vec<T, V>::raw raw;
    int w, b, sample, c0, mine, here;                  // c0: the slice's first channel; mine: pixels of this thread; here: channels of the slice
    int rank, tx, ty, log_rows, warps, first, last, pixels;          // pixels: of this thread, where its channels exist
    raw *x, *dy;                                       // its slots, as far apart as there are threads
    uint8_t *keep;                                     // keep bits of its slots, likewise
    float *coef, *red, *all;                           // six planes for channels, rows of sums of two planes, twice two planes of each block of the cluster

    __device__ __forceinline__ Stand(const NormArgs<T> &a, const Resident &r, unsigned char *shared, bool two, bool bits) {
        rank = blockIdx.x & ((1 << r.log_cluster) - 1);
        log_rows = r.log_block - r.log_tx, warps = 1 << (r.log_block - 5);
        tx = threadIdx.x & ((1 << r.log_tx) - 1), ty = threadIdx.x >> r.log_tx;
        const long long begin = (long long)rank * r.per;
        first = begin < a.pixels ? (int)begin : (int)a.pixels, last = begin + r.per < a.pixels ? (int)begin + r.per : (int)a.pixels;
        const int left = last - first - ty;
        pixels = left > 0 ? (left + (1 << log_rows) - 1) >> log_rows : 0;
        x = reinterpret_cast<raw *>(shared) + threadIdx.x;
        dy = x + (two ? r.slots << r.log_block : 0);
        unsigned char *rest = shared + ((size_t)r.slots << r.log_block) * sizeof(raw) * (two ? 2 : 1);
        keep = rest + threadIdx.x;
        if (bits) rest += r.slots << r.log_block;
        coef = reinterpret_cast<float *>(rest);
        red = coef + 6 * width();
        all = red + 2 * sum_rows() * width();
    }
    __device__ __forceinline__ void go(const NormArgs<T> &a, const Resident &r, uint32_t unit) {
        sample = unit / r.slices;
        c0 = (unit - sample * r.slices) * r.sv * V;
        w = (uint32_t)sample / (uint32_t)a.samples, b = sample - w * a.samples;
        here = min(a.channels - c0, r.sv * V);
        mine = tx * V < here ? pixels : 0;
    }
    __device__ __forceinline__ int width() const { return (warps * 32 >> log_rows) * V; }        // channels of a row of sums
    __device__ __forceinline__ int sum_rows() const { return min(1 << log_rows, warps); }
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
// Leaves a thread's N sums (lanes joined already) for the block: row of sums, two planes.
template <int N> __device__ __forceinline__ void leave_row(float *red, int log_tx, const float (&p)[N], const float (&q)[N]) {
    const int sums = N << log_tx, rows = min((int)blockDim.x >> log_tx, (int)blockDim.x / 32), row = log_tx > 5 ? threadIdx.x >> log_tx : threadIdx.x >> 5;
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

// Forward: moments of the parts of a group that a thread's vector holds, FOLD channels each of n values.
template <int FOLD, int V> __device__ __forceinline__ void fold_moments(float (&mean)[V / FOLD], float (&m2)[V / FOLD], const Batch<V> &m, float n) {
    constexpr float kOf = 1.f / FOLD;
#pragma unroll
    for (int i = 0; i < V / FOLD; ++i) {
        float f[FOLD], sum = 0.f, squares = 0.f, off = 0.f;
#pragma unroll
        for (int j = 0; j < FOLD; ++j) {
            const int c = i * FOLD + j;
            f[j] = c & 1 ? m.first[c / 2].y : m.first[c / 2].x;
            sum += f[j], squares += c & 1 ? m.squares[c / 2].y : m.squares[c / 2].x;
        }
        mean[i] = sum * kOf;
#pragma unroll
        for (int j = 0; j < FOLD; ++j) off = fmaf(f[j] - mean[i], f[j] - mean[i], off);
        m2[i] = fmaf(n, off, squares);
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
__global__ void __launch_bounds__(kMostThreads) norm_resident_kernel(NormArgs<T> a, Resident r) {
    extern __shared__ __align__(16) unsigned char shared[];
    if (r.log_cluster) cluster_arrive();
    after_previous();
    let_next();
    Stand<T, V> s(a, r, shared, false, false);
    const int width = s.width(), lane = threadIdx.x & 31;
    const uint32_t clusters = gridDim.x >> r.log_cluster;
    uint32_t unit = blockIdx.x >> r.log_cluster;
    s.go(a, r, unit);
    {
        const T *x = s.at(a.x, a.xs);
        const long long step = s.step(a.xs);
        for (int u = 0; u < s.mine; ++u, x += step) copy_async<V * sizeof(T)>(s.x + (u << r.log_block), x);
    }
    if (r.log_cluster) cluster_wait();                 // all blocks are there
    float *all = s.all;
    for (;;) {
        for (int c = threadIdx.x; c < s.here; c += s.warps * 32) {               // planes 2 and 3: weight and bias
            s.coef[2 * width + c] = a.weight ? a.weight[s.w * a.weight_worker + s.c0 + c] : 1.f;
            s.coef[3 * width + c] = a.bias ? a.bias[s.w * a.bias_worker + s.c0 + c] : 0.f;
        }
        const Words words(a.draw, s.w);
        Batch<V> m;
        const long long e0 = ((long long)s.b * a.pixels + s.first + s.ty) * a.channels + s.c0 + s.tx * V, e_step = (long long)a.channels << s.log_rows;
        copies_done();
        walk_slots<DROP ? 2 : 4, V, T>(0, s.mine, [&](int u) { return s.x[u << r.log_block]; }, [&](int u, Vec<T, V> &v) {
            if (DROP) {                                    // dropped elements become 0 in their slot
                drop_out(v, a.draw, words, e0 + u * e_step);
                s.x[u << r.log_block] = v.bits;
            }
            F2 f[kPairs<V>];
            counted<T, V, DROP>(f, v, a.draw.factor);
            if (u == 0) m.begin(f);
            m.add(f);
        });
        m.end(s.mine);
        // Threads of the same channels: those of a warp, then rows of the block, of which each warp (or part of one) has left one, ...
        with_fold<V>(r.fold, [&](auto fold) {
            constexpr int kFold = decltype(fold)::value;
            float mean[V / kFold], m2[V / kFold];
            float n = (float)s.mine;
            fold_moments<kFold, V>(mean, m2, m, n);
            join_lanes(n, mean, m2, kFold, 1 << r.log_tx);
            leave_row(s.red, r.log_tx, mean, m2);
        });
        __syncthreads();
        const int sums = width / r.fold, sum_rows = s.sum_rows(), block_pixels = s.last - s.first, each = (1 << s.log_rows) / sum_rows;
        const int whole = (block_pixels >> s.log_rows) * each, rest = block_pixels & ((1 << s.log_rows) - 1), mine = s.here / r.fold;
        const float of_block = block_pixels ? 1.f / block_pixels : 0.f;
        for (int k = threadIdx.x; k < mine; k += s.warps * 32) {
            // Pixels of the threads i * each .. i * each + each - 1 of a column: each of them takes every rows-th.
            auto count = [&](int i) { return (float)(whole + min(max(rest - i * each, 0), each)); };
            float sum = 0.f, squares = 0.f, off = 0.f;
            for (int i = 0; i < sum_rows; ++i) sum = fmaf(count(i), s.red[i * sums + k], sum);
            const float mean = sum * of_block;
            for (int i = 0; i < sum_rows; ++i) {
                const float d = s.red[i * sums + k] - mean;
                off = fmaf(count(i) * d, d, off), squares += s.red[(sum_rows + i) * sums + k];
            }
            tell_all(r, all, s.rank, sums, k, mean, fmaf((float)r.fold, off, squares));
        }
        meet(r);
        // ... then the blocks of the cluster and the parts of a group, by 2^log_sub lanes a group.
        const int parts = a.per_group / r.fold, groups = s.here / a.per_group, g0 = s.c0 / a.per_group;
        const float of_group = 1.f / ((float)a.pixels * a.per_group);
        for (int base = threadIdx.x >> 5 << (5 - r.log_sub); base < groups; base += (s.warps * 32) >> r.log_sub) {
            const int g = base + (lane >> r.log_sub), sub = lane & ((1 << r.log_sub) - 1), entries = g < groups ? parts << r.log_cluster : 0;
            auto values = [&](int i, float &pixels, float &mean, float &m2) {
                const int rank = i & ((1 << r.log_cluster) - 1), k = g * parts + (i >> r.log_cluster);
                pixels = (float)(r.fold * min(max((int)a.pixels - rank * r.per, 0), r.per));
                mean = all[2 * rank * sums + k], m2 = all[(2 * rank + 1) * sums + k];
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
        // The next unit's vectors take the places of this one's as soon as these have been used.
        Stand<T, V> next = s;
        unit += clusters;
        const bool more = unit < r.units;
        if (more) next.go(a, r, unit);
        const int coming = more ? next.mine : 0;
        const T *x = next.at(a.x, a.xs);
        const long long x_step = s.step(a.xs);
        if (s.mine) {
            F2 scale[kPairs<V>], shift[kPairs<V>];
            s.channels(scale, 0), s.channels(shift, 1);
            T *y = s.at(a.y, a.ys);
            const long long step = s.step(a.ys);
            with_act(a.act, [&](auto act) {
                walk_slots<4, V, T>(0, s.mine, [&](int u) { return s.x[u << r.log_block]; }, [&](int u, Vec<T, V> &v) {
                    F2 f[kPairs<V>];
                    pairs_of(v, f);
#pragma unroll
                    for (int j = 0; j < kPairs<V>; ++j) f[j] = activate<decltype(act)::value>(fma2(f[j], scale[j], shift[j]));
                    round_pairs(v, f);
                    v.to(y);
                    y += step;
                    if (u < coming) copy_async<V * sizeof(T)>(s.x + (u << r.log_block), x);
                    x += x_step;
                });
            });
        }
        if (!more) return;
        for (int u = s.mine; u < coming; ++u, x += x_step) copy_async<V * sizeof(T)>(s.x + (u << r.log_block), x);
        s = next;
        // The block that is behind may still read the sums of this unit, but not those of the one before: they are two.
        all = all == s.all ? s.all + (2 << r.log_cluster) * sums : s.all;
    }
}

template <typename T, int V, bool DROP>
__global__ void __launch_bounds__(kMostThreads) norm_grad_resident_kernel(NormArgs<T> a, Resident r) {
    extern __shared__ __align__(16) unsigned char shared[];
    if (r.log_cluster) cluster_arrive();
    after_previous();
    let_next();
    Stand<T, V> s(a, r, shared, true, DROP);
    const int width = s.width(), lane = threadIdx.x & 31;
    const uint32_t clusters = gridDim.x >> r.log_cluster;
    uint32_t unit = blockIdx.x >> r.log_cluster;
    s.go(a, r, unit);
    {
        const T *x = s.at(a.x, a.xs), *dy = s.at(a.dy, a.dys);
        const long long x_step = s.step(a.xs), dy_step = s.step(a.dys);
        for (int u = 0; u < s.mine; ++u, x += x_step, dy += dy_step) {
            copy_async<V * sizeof(T)>(s.x + (u << r.log_block), x);
            copy_async<V * sizeof(T)>(s.dy + (u << r.log_block), dy);
        }
    }
    if (r.log_cluster) cluster_wait();                 // all blocks are there
    float *all = s.all;
    for (;;) {
        // Planes: z = x * [0] + [1], [2] = -mean, [3] = rstd.
        for (int c = threadIdx.x; c < s.here; c += s.warps * 32) {
            const int g = r.group_magic ? __umulhi(s.c0 + c, r.group_magic) : s.c0 + c;
            const long long at = (long long)s.sample * a.groups + g;
            const float mean = a.stats[at], rstd = a.stats[(long long)a.n * a.samples * a.groups + at];
            const float scale = a.weight ? rstd * a.weight[s.w * a.weight_worker + s.c0 + c] : rstd;
            s.coef[c] = scale;
            s.coef[width + c] = fmaf(-mean, scale, a.bias ? a.bias[s.w * a.bias_worker + s.c0 + c] : 0.f);
            s.coef[2 * width + c] = -mean, s.coef[3 * width + c] = rstd;
        }
        const Words words(a.draw, s.w);
        Channels<V> k;
        F2 s0[kPairs<V>], s1[kPairs<V>];
#pragma unroll
        for (int j = 0; j < kPairs<V>; ++j) s0[j] = s1[j] = two(0.f);
        copies_done();
        __syncthreads();
        s.channels(k.scale, 0), s.channels(k.shift, 1), s.channels(k.minus_mean, 2);
        const long long e0 = ((long long)s.b * a.pixels + s.first + s.ty) * a.channels + s.c0 + s.tx * V, e_step = (long long)a.channels << s.log_rows;
        with_act(a.act, [&](auto act) {
            walk_slots<2, V, T>(0, s.mine, [&](int u) { return s.x[u << r.log_block]; }, [&](int u, Vec<T, V> &vx) {
                Vec<T, V> vd;
                vd.bits = s.dy[u << r.log_block];
                if (DROP) {
                    s.keep[u << r.log_block] = (uint8_t)drop_out(vx, a.draw, words, e0 + u * e_step);
                    s.x[u << r.log_block] = vx.bits;
                }
                add_grad<T, V, DROP, decltype(act)::value>(s0, s1, k, vx, vd, a.draw.factor);
            });
        });
        float t0[V], t1[V];
#pragma unroll
        for (int j = 0; j < V; ++j) t0[j] = j & 1 ? s0[j / 2].y : s0[j / 2].x, t1[j] = j & 1 ? s1[j / 2].y : s1[j / 2].x;
        for (int o = 1 << r.log_tx; o < 32; o <<= 1)
#pragma unroll
            for (int j = 0; j < V; ++j) t0[j] += __shfl_xor_sync(~0u, t0[j], o), t1[j] += __shfl_xor_sync(~0u, t1[j], o);
        leave_row(s.red, r.log_tx, t0, t1);
        __syncthreads();
        const int sum_rows = s.sum_rows();
        for (int c = threadIdx.x; c < s.here; c += s.warps * 32) {
            float p = 0.f, q = 0.f;
            for (int i = 0; i < sum_rows; ++i) p += s.red[i * width + c], q += s.red[(sum_rows + i) * width + c];
            tell_all(r, all, s.rank, width, c, p, q);
        }
        meet(r);
        // Sums over the cluster; of a channel they are the sample's share of dbias and dweight (each block writes some channels').  Times the
        // channel's rstd and weight, planes 4 and 5 take them for its group's s1 and s2.
        for (int c = threadIdx.x; c < s.here; c += s.warps * 32) {
            float p = 0.f, q = 0.f;
            for (int i = 0; i < 1 << r.log_cluster; ++i) p += all[2 * i * width + c], q += all[(2 * i + 1) * width + c];
            q *= s.coef[3 * width + c];
            if ((c & ((1 << r.log_cluster) - 1)) == s.rank) {
                if (a.sums[0]) a.sums[0][s.sample * a.sums_sample[0] + s.c0 + c] = p;
                if (a.sums[1]) a.sums[1][s.sample * a.sums_sample[1] + s.c0 + c] = q;
            }
            s.coef[4 * width + c] = p * s.coef[c], s.coef[5 * width + c] = q * s.coef[c];
        }
        // The next unit's vectors take the places of this one's as soon as these have been used.
        Stand<T, V> next = s;
        unit += clusters;
        const bool more = unit < r.units;
        if (more) next.go(a, r, unit);
        const int coming = more ? next.mine : 0;
        const T *x = next.at(a.x, a.xs), *dy = next.at(a.dy, a.dys);
        const long long x_step = s.step(a.xs), dy_step = s.step(a.dys);
        int used = 0;                                      // slots that are on their way
        __syncthreads();
        if (a.y) {
            // The first two rows of sums, which all have read, become planes for make_grad's m1 and m2.
            const int groups = s.here / a.per_group;
            const float of = -1.f / ((float)a.pixels * a.per_group);
            for (int base = threadIdx.x >> 5 << (5 - r.log_sub); base < groups; base += (s.warps * 32) >> r.log_sub) {
                const int g = base + (lane >> r.log_sub), sub = lane & ((1 << r.log_sub) - 1), end = g < groups ? (g + 1) * a.per_group : 0;
                float p = 0.f, q = 0.f;
                for (int c = g * a.per_group + sub; c < end; c += 1 << r.log_sub) p += s.coef[4 * width + c], q += s.coef[5 * width + c];
                p = lanes_sum(p, r.log_sub) * of, q = lanes_sum(q, r.log_sub) * of;
                for (int c = g * a.per_group + sub; c < end; c += 1 << r.log_sub) {
                    const float m2 = q * s.coef[3 * width + c];
                    s.red[c] = fmaf(s.coef[2 * width + c], m2, p), s.red[width + c] = m2;
                }
            }
            __syncthreads();
            F2 m1[kPairs<V>], m2[kPairs<V>];
            s.channels(m1, 6), s.channels(m2, 7);
            T *y = s.at(a.y, a.ys);
            const long long step = s.step(a.ys);
            with_act(a.act, [&](auto act) {
                walk_slots<2, V, T>(0, s.mine, [&](int u) { return s.x[u << r.log_block]; }, [&](int u, Vec<T, V> &vx) {
                    Vec<T, V> vd;
                    vd.bits = s.dy[u << r.log_block];
                    make_grad<T, V, DROP, decltype(act)::value>(vx, k.scale, k.shift, m1, m2, vd, a.draw.factor, DROP ? s.keep[u << r.log_block] : 0);
                    vx.to(y);
                    y += step;
                    if (u < coming) copy_async<V * sizeof(T)>(s.x + (u << r.log_block), x), copy_async<V * sizeof(T)>(s.dy + (u << r.log_block), dy);
                    x += x_step, dy += dy_step;
                });
            });
            used = s.mine;
        }
        if (!more) return;
        for (int u = used; u < coming; ++u, x += x_step, dy += dy_step) {
            copy_async<V * sizeof(T)>(s.x + (u << r.log_block), x);
            copy_async<V * sizeof(T)>(s.dy + (u << r.log_block), dy);
        }
        s = next;
        // The block that is behind may still read the sums of this unit, but not those of the one before: they are two.
        all = all == s.all ? s.all + (2 << r.log_cluster) * width : s.all;
    }
}
