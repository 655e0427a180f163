// orth_small.cuh - Newton-Schulz orthogonalisation of matrices whose short side s is at most 64 (low-rank adapters, small
// layers, vectors).  Device code, included by orth.cu inside its unnamed namespace.
//
// X_k = Q_k u with Q_k a polynomial of the s x s Gram matrix alone, so the steps are taken on s x s matrices: A = G / (|u| + eps)^2,
// G = u u^T (or u^T u), |u|^2 = tr G, and per step  P = a I + b A + c A A,  Q <- P Q,  A <- P A P.  All of these are polynomials of G:
// they commute and are symmetric, so one triangle is computed.  That is s^2 l multiply-adds for G and s^2 l for out = Q u, whatever
// the number of steps, against 3 s^2 l per step.  G squares the singular values' ratio, so all of it is in 64 bits: the
// result is as exact for a small singular value as the long way in 32 bits.  (Tensor-core tiles of 128 rows would be mostly padding: 384
// adapter matrices of 16 x 1024 took 608 us that way, one 64 x 64 matrix 103 us; the chain of 3 * steps dependent
// launches-in-one of a tiled kernel is 7 us a link.)
//
//   orth_gram_kernel   a part of the long side per CTA: momentum, G's partial sums; the matrix's last CTA adds the parts in
//                      order and takes the steps.
//   orth_apply_kernel  out = scale Q u, a part of the long side per CTA.
//   orth_resident_kernel  all of it by one CTA, for matrices that fit its shared memory (16 x 1024, 64 x 512): u is read once, nothing
//                      passes through memory.
//
// Bound: the 64-bit units (64 multiply-adds per SM and cycle) for s near 64, launch and memory latency below.  The products go
// through mma.sync m8n8k4 in 64 bits (the tcgen05 instructions have no such type): same rate as plain multiply-adds but two
// shared-memory loads for 256 of them; written as 4 x 4 tiles per thread the loads took 7 times as long as the arithmetic.
#pragma once

struct SmallMat {
    long long offset, stride;
    int s, l, sp, tall;                            // sp: s rounded up to 8
    int parts, per;                                // of the long side, columns of each
    size_t partial, q;                             // places in the 64-bit workspace: [parts][tiles][64], [sp][sp]
    float scale;
};
struct SmallArgs {
    const SmallMat *mats;
    const uint2 *part;                             // (matrix, part in it), for the Gram kernel
    const uint2 *piece;                            // (matrix, first column), for the other
    double *work;
    unsigned *ticket;
    const void *grad;
    float *m;
    float mu;
    void *out;
    int out_type, steps;
};

constexpr int kSmallSide = 64;
constexpr int kGramDoubles = 8192;                 // of a piece of u in shared memory
constexpr int kApplyCols = 128, kApplyLd = kApplyCols + 8;
// Row lengths in shared memory that keep the fragments' loads free of bank conflicts: s x s matrices (8 rows of 4), and u by
// columns (4 rows of 8).
__host__ __device__ constexpr int square_ld(int sp) { return sp + 4; }
__host__ __device__ constexpr int gram_ld(int sp) { return sp % 16 ? sp : sp + 8; }

// 8 x 8 += (8 x 4) (4 x 8).  a: row lane / 4, column lane % 4; b: row lane % 4, column lane / 4; c: row lane / 4,
// columns lane % 4 * 2 and the next.
__device__ __forceinline__ void mma_f64(double (&c)[2], double a, double b) {
    asm("mma.sync.aligned.m8n8k4.row.col.f64.f64.f64.f64 {%0, %1}, {%2}, {%3}, {%0, %1};"
        : "+d"(c[0]), "+d"(c[1])
        : "d"(a), "d"(b));
}

__device__ __forceinline__ float small_u(const SmallArgs &a, float g, long long at, bool update) {
    if (!a.m) return g;
    float m = a.m[at];
    if (update) {
        m = __fadd_rn(__fmul_rn(a.mu, m), g);
        a.m[at] = m;
    }
    return __fadd_rn(g, __fmul_rn(a.mu, m));
}
// Element (i of the short side, j of the long one).
__device__ __forceinline__ long long small_at(const SmallMat &M, int i, int j) {
    return M.offset + (M.tall ? (long long)j * M.stride + i : (long long)i * M.stride + j);
}
// Tile `k` of the lower triangle, tiles numbered row by row.
__device__ __forceinline__ void triangle(int k, int &i, int &j) {
    i = (int)((sqrtf(8.f * (float)k + 1.f) - 1.f) * 0.5f);
    while ((i + 1) * (i + 2) / 2 <= k) ++i;
    while (i * (i + 1) / 2 > k) --i;
    j = k - i * (i + 1) / 2;
}
// A warp's 8 x 8 tiles of one triangle of an s x s matrix, at most N: a run of them row by row, so that most share the fragment
// of the row with the one before.
template <int N>
struct WarpTiles {
    int i[N], j[N], n = 0;                                           // this lane's row of either operand's fragment
    bool fresh[N];                                                   // another row of tiles than the one before
    __device__ __forceinline__ explicit WarpTiles(int sp) {
        const int side = sp / 8, tiles = side * (side + 1) / 2, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
        const int each = tiles / 8, more = tiles % 8, first = warp * each + (warp < more ? warp : more);
        n = each + (warp < more);
#pragma unroll
        for (int b = 0; b < N; ++b) {
            i[b] = j[b] = 0;
            if (b < n) triangle(first + b, i[b], j[b]);
            i[b] = i[b] * 8 + lane / 4, j[b] = j[b] * 8 + lane / 4;
            fresh[b] = b == 0 || i[b] != i[b > 0 ? b - 1 : 0];
        }
    }
};
// out = x y (POLY: kA I + kB x + kC x y) for symmetric commuting x and y (rows of square_ld(sp)): one triangle, mirrored.
// out is neither.  A product waits about 190 cycles for the one before it on the same accumulator: a warp's tiles go side by
// side, each as two chains.
template <int N, bool POLY>
__device__ __forceinline__ void sym_product(double *out, const double *x, const double *y, int sp, const WarpTiles<N> &w) {
    const int ld = square_ld(sp), k = threadIdx.x % 4;
    double c[N][2][2] = {};
#pragma unroll 2
    for (int e = 0; e < sp; e += 8) {
        double u[2] = {};
#pragma unroll
        for (int b = 0; b < N; ++b)
            if (b < w.n) {
                if (w.fresh[b]) u[0] = x[w.i[b] * ld + k + e], u[1] = x[w.i[b] * ld + k + e + 4];
                const double v0 = y[w.j[b] * ld + k + e], v1 = y[w.j[b] * ld + k + e + 4];
                mma_f64(c[b][0], u[0], v0);
                mma_f64(c[b][1], u[1], v1);
            }
    }
#pragma unroll
    for (int b = 0; b < N; ++b)
        if (b < w.n)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int i = w.i[b], j = w.j[b] / 8 * 8 + k * 2 + q;
                double s = c[b][0][q] + c[b][1][q];
                if (j <= i) {
                    if (POLY) s = __fma_rn((double)kC, s, __fma_rn((double)kB, x[i * ld + j], i == j ? (double)kA : 0.0));
                    out[i * ld + j] = out[j * ld + i] = s;
                }
            }
    __syncthreads();
}

// From the Gram matrix in A: Q with out = Q u; returns where it is (one of the four).
template <int N>
__device__ __forceinline__ double *small_steps(double *A, double *P, double *Q, double *W, int sp, int steps) {
    __shared__ double inv;
    const WarpTiles<N> tiles(sp);
    const int sq = square_ld(sp), lane = threadIdx.x % 32;
    if (threadIdx.x < 32) {
        double tr = 0.0;
        for (int i = lane; i < sp; i += 32) tr += A[i * sq + i];
        for (int k = 16; k; k >>= 1) tr += __shfl_xor_sync(~0u, tr, k);
        if (lane == 0) inv = 1.0 / (sqrt(tr) + (double)kEps);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < sp * sq; e += 256) {
        A[e] = A[e] * inv * inv;
        Q[e] = e % (sq + 1) == 0 ? inv : 0.0;
    }
    __syncthreads();
    for (int step = 0; step < steps; ++step) {
        sym_product<N, true>(P, A, A, sp, tiles);
        sym_product<N, false>(W, P, Q, sp, tiles);
        double *t = Q;
        Q = W, W = t;
        if (step + 1 < steps) {
            sym_product<N, false>(W, P, A, sp, tiles);
            sym_product<N, false>(A, W, P, sp, tiles);
        }
    }
    return Q;
}

template <typename T>
__global__ void __launch_bounds__(256) orth_gram_kernel(const SmallArgs a) {
    extern __shared__ __align__(16) double sh[];
    __shared__ int last;
    let_next_start();
    const uint2 pt = a.part[blockIdx.x];
    const SmallMat M = a.mats[pt.x];
    const int sp = M.sp, side = sp / 8, tiles = side * (side + 1) / 2, ld = gram_ld(sp), cols = kGramDoubles / ld / 4 * 4;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    // Few tiles: the warps share them out by columns of u, in `groups`; many: a warp has every eighth one.
    const int groups = tiles >= 8 ? 1 : 8 / tiles, group = tiles >= 8 ? 0 : warp / tiles, tile0 = tiles >= 8 ? warp : warp % tiles;
    const T *g = static_cast<const T *>(a.grad);
    constexpr int kMost = 5;                                         // 36 tiles by 8 warps
    int at_i[kMost], at_j[kMost];
    double acc[kMost][2] = {};
#pragma unroll
    for (int b = 0; b < kMost; ++b) {
        int ti = 0, tj = 0;
        if (tile0 + 8 * b < tiles) triangle(tile0 + 8 * b, ti, tj);
        at_i[b] = ti * 8 + lane / 4, at_j[b] = tj * 8 + lane / 4;
    }
    const int j0 = (int)pt.y * M.per, j1 = j0 + M.per < M.l ? j0 + M.per : M.l;
    for (int j = j0; j < j1; j += cols) {
        const int n = j1 - j < cols ? j1 - j : cols, filled = (n + 3) / 4 * 4;   // u as [column of the long side][ld]
#pragma unroll 4
        for (int e = threadIdx.x; e < filled * sp; e += 256) {
            int i, c;
            if (M.tall) c = e / sp, i = e - c * sp;
            else i = e / filled, c = e - i * filled;
            double v = 0.0;
            if (i < M.s && c < n) {
                const long long at = small_at(M, i, j + c);
                v = (double)small_u(a, to_f<T>(g[at]), at, true);
            }
            sh[c * ld + i] = v;
        }
        __syncthreads();
        if (group < groups)
#pragma unroll 2
            for (int c = group * 4; c < filled; c += groups * 4) {
                const double *row = sh + (c + lane % 4) * ld;
#pragma unroll
                for (int b = 0; b < kMost; ++b)
                    if (tile0 + 8 * b < tiles) mma_f64(acc[b], row[at_i[b]], row[at_j[b]]);
            }
        __syncthreads();
    }
    // The groups' sums, in their order.
    double *part = a.work + M.partial + (size_t)pt.y * tiles * 64;
    if (groups == 1) {
#pragma unroll
        for (int b = 0; b < kMost; ++b)
            if (group < groups && tile0 + 8 * b < tiles) {
                double *o = part + (tile0 + 8 * b) * 64 + lane * 2;
                o[0] = acc[b][0], o[1] = acc[b][1];
            }
    } else {
        sh[warp * 64 + lane * 2] = acc[0][0], sh[warp * 64 + lane * 2 + 1] = acc[0][1];
        __syncthreads();
        for (int e = threadIdx.x; e < tiles * 64; e += 256) {
            double s = 0.0;
            for (int q = 0; q < groups; ++q) s += sh[q * tiles * 64 + e];
            part[e] = s;
        }
    }
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        last = atomicAdd(&a.ticket[pt.x], 1u) == (unsigned)M.parts - 1;
        __threadfence();
    }
    __syncthreads();
    if (!last) return;
    if (threadIdx.x == 0) a.ticket[pt.x] = 0;                        // for the next call
    const int sq = square_ld(sp), all_size = sp * sq;
    double *A = sh, *P = sh + all_size, *Q = P + all_size, *W = Q + all_size;
    const double *all = a.work + M.partial;
    constexpr int kOwn = 9;                                          // 36 tiles' elements by 256 threads
    double sum[kOwn] = {};
#pragma unroll 2
    for (int p = 0; p < M.parts; ++p)
#pragma unroll
        for (int b = 0; b < kOwn; ++b)
            if (threadIdx.x + 256 * b < tiles * 64) sum[b] += __ldcg(all + (size_t)p * tiles * 64 + threadIdx.x + 256 * b);
#pragma unroll
    for (int b = 0; b < kOwn; ++b) {
        const int e = threadIdx.x + 256 * b, k = e / 64, w = e - k * 64;
        if (k >= tiles) break;
        int bi, bj;
        triangle(k, bi, bj);
        const int i = bi * 8 + w / 8, j = bj * 8 + w % 8;
        if (j <= i) A[i * sq + j] = A[j * sq + i] = sum[b];
    }
    __syncthreads();
    Q = sp <= 32 ? small_steps<2>(A, P, Q, W, sp, a.steps) : small_steps<5>(A, P, Q, W, sp, a.steps);
    double *q = a.work + M.q;
    for (int e = threadIdx.x; e < sp * sp; e += 256) q[e] = Q[e / sp * sq + e % sp] * (double)M.scale;
}

template <typename T>
__global__ void __launch_bounds__(256) orth_apply_kernel(const SmallArgs a) {
    extern __shared__ __align__(16) double sh[];
    const uint2 pc = a.piece[blockIdx.x];
    const SmallMat M = a.mats[pc.x];
    const int sp = M.sp, sq = square_ld(sp), j0 = (int)pc.y, n = M.l - j0 < kApplyCols ? M.l - j0 : kApplyCols;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    double *q = sh, *u = sh + sp * sq;                               // [sp][sq], [sp][kApplyLd]
    const T *g = static_cast<const T *>(a.grad);
    earlier_done();
    for (int e = threadIdx.x; e < sp * sp; e += 256) q[e / sp * sq + e % sp] = __ldcg(a.work + M.q + e);
#pragma unroll 4
    for (int e = threadIdx.x; e < n * sp; e += 256) {
        int i, c;
        if (M.tall) c = e / sp, i = e - c * sp;
        else i = e / n, c = e - i * n;
        double v = 0.0;
        if (i < M.s) {
            const long long at = small_at(M, i, j0 + c);
            v = (double)small_u(a, to_f<T>(g[at]), at, false);
        }
        u[i * kApplyLd + c] = v;
    }
    __syncthreads();
    // A warp takes 16 columns; the results go back through shared memory, over u.
    constexpr int kMost = kSmallSide / 8;
    double acc[kMost][2][2] = {};
    for (int k = 0; k < sp; k += 4) {
        const double *row = u + (k + lane % 4) * kApplyLd + warp * 16 + lane / 4;
        const double b0 = row[0], b1 = row[8];
        const double *col = q + lane / 4 * sq + k + lane % 4;
#pragma unroll
        for (int t = 0; t < kMost; ++t)
            if (t * 8 < sp) {
                const double v = col[t * 8 * sq];
                mma_f64(acc[t][0], v, b0);
                mma_f64(acc[t][1], v, b1);
            }
    }
    __syncthreads();
    float *r = reinterpret_cast<float *>(u);
#pragma unroll
    for (int t = 0; t < kMost; ++t)
        if (t * 8 < sp)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int p = 0; p < 2; ++p)
                    r[(t * 8 + lane / 4) * (kApplyCols + 1) + warp * 16 + h * 8 + lane % 4 * 2 + p] = (float)acc[t][h][p];
    __syncthreads();
    for (int e = threadIdx.x; e < n * M.s; e += 256) {
        int i, col;
        if (M.tall) col = e / M.s, i = e - col * M.s;
        else i = e / n, col = e - i * n;
        const long long at = small_at(M, i, j0 + col);
        const float v = r[i * (kApplyCols + 1) + col];
        if (a.out_type == CSER_TYPE_F32) static_cast<float *>(a.out)[at] = v;
        else if (a.out_type == CSER_TYPE_BF16) static_cast<__nv_bfloat16 *>(a.out)[at] = __float2bfloat16_rn(v);
        else static_cast<__half *>(a.out)[at] = __float2half_rn(v);
    }
}

// Rows of u (one per column of the long side) in shared memory, as floats.
__host__ __device__ constexpr int resident_ld(int sp) { return sp % 32 == 16 ? sp : gram_ld(sp); }
__host__ __device__ constexpr size_t resident_bytes(int sp, long long l) {
    return (size_t)sp * square_ld(sp) * 32 + (size_t)((l + 15) / 16 * 16) * resident_ld(sp) * 4;
}
constexpr size_t kResidentMost = 224 * 1024;

// MOST: eighths of the short side at most (2, 4, 8).
template <typename T, int MOST>
__global__ void __launch_bounds__(256, MOST == 8 ? 2 : 3) orth_resident_kernel(const SmallArgs a) {
    extern __shared__ __align__(16) double sh[];
    const SmallMat M = a.mats[blockIdx.x];
    const int sp = M.sp, sq = square_ld(sp), ld = resident_ld(sp), cols = (M.l + 15) / 16 * 16, eighths = sp / 8;
    const int side = sp / 8, tiles = side * (side + 1) / 2, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    double *A = sh, *P = sh + sp * sq, *Q = P + sp * sq, *W = Q + sp * sq;
    float *u = reinterpret_cast<float *>(W + sp * sq);              // [column of the long side][ld]
    const T *g = static_cast<const T *>(a.grad);
    // Eight values at a time, along memory: of a row of a wide matrix (lanes take different rows, which keeps the
    // stores to shared memory apart), or of the short side of a tall one.
    const int chunks = M.tall ? cols * eighths : sp * (cols / 8);
#pragma unroll 4
    for (int e = threadIdx.x; e < chunks; e += 256) {
        int i, c, n;
        if (M.tall) c = e / eighths, i = (e - c * eighths) * 8, n = c < M.l ? M.s - i : 0;
        else c = e / sp, i = e - c * sp, c *= 8, n = i < M.s ? M.l - c : 0;
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = 0.f;
        if (n > 0) {
            const long long at = small_at(M, i, c);
            load8(g + at, n, v);
            if (a.m) {
                float w[8];
                load8(a.m + at, n, w);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    w[k] = __fadd_rn(__fmul_rn(a.mu, w[k]), v[k]);
                    v[k] = __fadd_rn(v[k], __fmul_rn(a.mu, w[k]));
                    if (k < n) a.m[at + k] = w[k];
                }
            }
        }
        float *o = u + c * ld + i;
#pragma unroll
        for (int k = 0; k < 8; ++k) o[M.tall ? k : k * ld] = v[k];
    }
    __syncthreads();
    if (tiles >= 8) {                                                // Gram matrix: a warp's tiles side by side, each a chain
        constexpr int kMost = MOST == 8 ? 5 : 2;
        const WarpTiles<kMost> w(sp);
        double acc[kMost][2] = {};
        const float *row = u + lane % 4 * ld;
#pragma unroll 4
        for (int c = 0; c < cols; c += 4, row += 4 * ld)
#pragma unroll
            for (int b = 0; b < kMost; ++b)
                if (b < w.n) mma_f64(acc[b], (double)row[w.i[b]], (double)row[w.j[b]]);
#pragma unroll
        for (int b = 0; b < kMost; ++b)
            if (b < w.n) {
                const int i = w.i[b], j = w.j[b] / 8 * 8 + lane % 4 * 2;
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    if (j + q <= i) A[i * sq + j + q] = A[(j + q) * sq + i] = acc[b][q];
            }
    } else {                                                         // few tiles: shared out by columns too, in `groups`, four chains
        const int room = 3 * sp * sq / (tiles * 64), groups = 8 / tiles < room ? 8 / tiles : room;
        if (warp / tiles < groups) {
            const int b = warp % tiles, group = warp / tiles;
            int ti, tj;
            triangle(b, ti, tj);
            double acc[4][2] = {};
            const float *row = u + (group * 4 + lane % 4) * ld + lane / 4;
            const int step = groups * 4 * ld;
            int c = group * 4;
            for (; c + groups * 12 < cols; c += groups * 16, row += 4 * step)
#pragma unroll
                for (int h = 0; h < 4; ++h) mma_f64(acc[h], (double)row[h * step + ti * 8], (double)row[h * step + tj * 8]);
            for (; c < cols; c += groups * 4, row += step) mma_f64(acc[0], (double)row[ti * 8], (double)row[tj * 8]);
            // over P, Q and W: the groups' sums one after the other
            double *o = P + (group * tiles + b) * 64 + lane * 2;
#pragma unroll
            for (int q = 0; q < 2; ++q) o[q] = (acc[0][q] + acc[1][q]) + (acc[2][q] + acc[3][q]);
        }
        __syncthreads();
        for (int e = threadIdx.x; e < tiles * 64; e += 256) {
            const int k = e / 64, w = e - k * 64;
            int bi, bj;
            triangle(k, bi, bj);
            double s = 0.0;
            for (int q = 0; q < groups; ++q) s += P[q * tiles * 64 + e];
            const int i = bi * 8 + w / 8, j = bj * 8 + w % 8;
            if (j <= i) A[i * sq + j] = A[j * sq + i] = s;
        }
    }
    __syncthreads();
    Q = small_steps<MOST == 8 ? 5 : MOST == 4 ? 2 : 1>(A, P, Q, W, sp, a.steps);
    // out = scale Q u: a warp takes 16 columns (32 for the shortest sides: more chains at once) and puts the results where they were.
    constexpr int kCols = MOST == 2 ? 4 : 2;
    for (int c = warp * kCols * 8; c < cols; c += kCols * 64) {
        double acc[MOST][kCols][2] = {};
#pragma unroll 2
        for (int k = 0; k < sp; k += 4) {
            const float *row = u + (c + lane / 4) * ld + k + lane % 4;
            double f[kCols];
#pragma unroll
            for (int h = 0; h < kCols; ++h) f[h] = c + h * 8 < cols ? (double)row[h * 8 * ld] : 0.0;
            const double *col = Q + lane / 4 * sq + k + lane % 4;
#pragma unroll
            for (int t = 0; t < MOST; ++t)
                if (t * 8 < sp) {
                    const double v = col[t * 8 * sq];
#pragma unroll
                    for (int h = 0; h < kCols; ++h) mma_f64(acc[t][h], v, f[h]);
                }
        }
        __syncwarp();
#pragma unroll
        for (int t = 0; t < MOST; ++t)
            if (t * 8 < sp)
#pragma unroll
                for (int h = 0; h < kCols; ++h)
#pragma unroll
                    for (int p = 0; p < 2; ++p)
                        if (c + h * 8 < cols)
                            u[(c + h * 8 + lane % 4 * 2 + p) * ld + t * 8 + lane / 4] = (float)(acc[t][h][p] * (double)M.scale);
    }
    __syncthreads();
#pragma unroll 2
    for (int e = threadIdx.x; e < chunks; e += 256) {
        int i, c, n;
        if (M.tall) c = e / eighths, i = (e - c * eighths) * 8, n = c < M.l ? M.s - i : 0;
        else c = e / sp, i = e - c * sp, c *= 8, n = i < M.s ? M.l - c : 0;
        if (n <= 0) continue;
        const float *o = u + c * ld + i;
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = o[M.tall ? k : k * ld];
        const long long at = small_at(M, i, c);
        if (a.out_type == CSER_TYPE_F32) {
            float *to = static_cast<float *>(a.out) + at;
            if (n >= 8 && (reinterpret_cast<uintptr_t>(to) & 15) == 0) {
                reinterpret_cast<float4 *>(to)[0] = make_float4(v[0], v[1], v[2], v[3]);
                reinterpret_cast<float4 *>(to)[1] = make_float4(v[4], v[5], v[6], v[7]);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k < n) to[k] = v[k];
            }
        } else {
            store_row(a.out, at, n, a.out_type == CSER_TYPE_BF16, v);
        }
    }
}
