// Orthogonalised updates (cser_orth_* of include/cser_train.h): Newton-Schulz products on the matrices inside the flat
// gradients of n workers, grouped: three kernels for as many matrices as fit a workspace of 2 GB (and up to three for those with a short
// side of at most 64, orth_small.cuh).
//
//   orth_norm_kernel     one pass over g (and m, which it updates): |u|_F per matrix
//   orth_convert_kernel  X = u / (|u|_F + 1e-7) as 16-bit panels (tensor_tiles.cuh)
//   orth_products_kernel all products of all steps, persistent
//
// With s = the shorter side, l = the longer, a step is
//     A = X X^T (or X^T X)        s x s, symmetric: tiles on and below the diagonal only          s^2 l flops
//     B = b A + c A^2             s x s, symmetric, likewise                                       s^3
//     X <- a X + B X (or X B)                                                                    2 s^2 l
// 4 s^3 multiply-adds for a square: far over the tensor cores' balance point, so products are the bound for all but
// small matrices, for which the chain of 3 * steps dependent products is.
//
// No transposes.  A tall matrix is not turned: its rows become the inner dimension instead.  The half of A and B above
// the diagonal is not stored: a stage that needs it reads the mirrored block and takes it as the other majorness.
//
// Rounding.  Operands are fp16 (X, A, B times 2^12, which keeps entries of matrices with singular values in 0 .. 1.21 inside
// fp16's range).  Rounding X, A and B alone would leave 1.5e-3 relative error for a random matrix and 2e-2 for a matrix of low
// rank with little noise.  Two things take that away without another product: X's remainder is kept (a second fp16) for the
// a X term (in fp32 where the result is 32-bit), and the diagonals of A and B, which dominate them once X is near orthogonal, are kept in fp32 and left out of
// the operands:  A A = Ao Ao + (dA_i + dA_j) Ao_ij + dA_i^2 [i = j].  That leaves 3e-4 .. 1e-3.  For a 32-bit result every
// operand is a pair of fp16 and a product is hi lo + lo hi + hi hi, small terms first.
//
// Order of work.  The list of all tiles of all phases of all steps is dealt out to the CTAs in order; a tile waits for
// the tiles of its own matrix's earlier phases by a counter, so the phases of different matrices overlap.  The launch is cooperative:
// every CTA is resident, a wait always has someone to end it.  Where A's tiles are fewer than the CTAs and the long side is long, a tile is
// several entries of the list, each a share of the inner dimension: the last one waits for the others' sums and adds them up in order.
#include <cuda.h>
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <algorithm>
#include <new>
#include <vector>

#include "cser_train.h"
#include "train_host.h"

namespace {

#include "tensor_tiles.cuh"

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f, kEps = 1e-7f;
constexpr float kScale = 4096.f, kUnscale = 1.f / 4096.f, kUnscale2 = kUnscale * kUnscale;
constexpr int kNormChunk = 16384;                  // elements per CTA of the norm kernel
// How tiles are cut: 128 x 64 or 128 x 128 by one CTA, or 256 rows by a pair of CTAs (by 256 columns; 128 for a 32-bit result, whose
// sums must fit the epilogue's registers).
enum { kNarrow = 0, kSingle = 1, kPaired = 2 };
__host__ __device__ constexpr int mode_cg(int mode) { return mode == kPaired ? 2 : 1; }
__host__ __device__ constexpr int tile_n(int mode, bool split) { return mode == kNarrow ? 64 : mode == kPaired && !split ? 256 : 128; }
// The tensor cores truncate every partial sum, about 2^-24 of it for 16 terms: 2e-5 over an inner dimension of 4096.  So a
// 32-bit result's accumulator of hi hi is taken out and added up in registers, rounded, after this many stages.  X's
// product is the one whose error the steps after it do not shrink: with a low-rank matrix 9e-6 at 4 stages.
constexpr int kChunkAB = 4, kChunkX = 1;
constexpr size_t kGroupBytes = 2ull << 30;         // workspace of one group of matrices

struct OrthMat {
    __half *xh[2], *xl[2], *ah, *al, *bh, *bl;     // panels; al, bl for 32-bit results only
    float *xf[2];                                  // X in fp32, panels of 64 columns; for 32-bit results only
    float *da, *db;                                // diagonals of A and B
    long long offset, stride;                      // of the matrix in the [n, ld] arrays, worker included
    int rows, cols, tall;
    int rp, cp, sp;                                // rows, columns, short side, padded to the tile
    int k_long, k_short;                           // inner dimensions in stages
    unsigned tiles_sym, tiles_x;                   // signals that complete a phase
    float scale;
    int chunk0, chunks;                            // of the norm kernel
    float *part;                                   // sums of A's tiles over shares of the inner dimension, see choose_shares
    unsigned *joined;                              // [its tiles of A][CTAs][epilogue warps] how often one has left such sums
    int n_joined, shares;
};
struct OrthTile {
    uint32_t q;
    uint16_t i, j;
    uint16_t share, slot;                          // of A's tiles: the last share is the one that adds them up; which of its matrix's
};
struct PanelUnit {
    uint32_t q, r0, c0;                            // 32 rows, up to 4 panels
};

struct OrthArgs {
    const OrthMat *mats;
    const OrthTile *a_tiles, *sym, *x;
    int n_a, n_sym, n_x, steps;
    unsigned *done;                                // [matrices] finished tiles
    unsigned *ticket;                              // [matrices] norm kernel
    float *partial, *inv;                          // [chunks], [matrices] 1 / (norm + eps)
    const uint2 *chunk;                            // (matrix, chunk in it)
    const PanelUnit *unit;
    const void *grad;
    float *m;
    float mu;
    void *out;
    int out_type;
    unsigned *err;
    long long wait_cycles;
    unsigned stall;                                // test hook: added to what the second phase of each matrix waits for
};

// ------------------------------------------------------------------ element access
template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f(float v) { return v; }
template <> __device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f(__half v) { return __half2float(v); }

// 8 consecutive elements, `n` of them wanted (the rest 0).
template <typename T>
__device__ __forceinline__ void load8(const T *p, int n, float (&v)[8]) {
    if (n >= 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
        if constexpr (sizeof(T) == 4) {
            const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
            v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
        } else {
            const uint4 a = *reinterpret_cast<const uint4 *>(p);
            const T *e = reinterpret_cast<const T *>(&a);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = to_f<T>(e[k]);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = k < n ? to_f<T>(p[k]) : 0.f;
    }
}

#include "orth_small.cuh"

// ------------------------------------------------------------------ |u|_F, momentum, X as panels
// 8 values as one chunk of fp16 and one of what that leaves.
__device__ __forceinline__ void split8(const float *v, uint4 &hi, uint4 &lo) {
    uint32_t h[4], l[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        h[k] = pack_half2(v[2 * k], v[2 * k + 1]);
        const float2 b = __half22float2(*reinterpret_cast<const __half2 *>(&h[k]));
        l[k] = pack_half2(__fsub_rn(v[2 * k], b.x), __fsub_rn(v[2 * k + 1], b.y));
    }
    hi = make_uint4(h[0], h[1], h[2], h[3]);
    lo = make_uint4(l[0], l[1], l[2], l[3]);
}
__device__ __forceinline__ void unpack8(const uint4 &p, float *v) {
    const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float2 b = __half22float2(*reinterpret_cast<const __half2 *>(&w[k]));
        v[2 * k] = b.x, v[2 * k + 1] = b.y;
    }
}
__device__ __forceinline__ char *panel_at(__half *base, int rows, int panel) {
    return reinterpret_cast<char *>(base) + (size_t)panel * rows * 128;
}

// X in fp32: panels of 64 columns, rows of 256 bytes, chunk c of 4 columns of row r at c ^ (r & 7).
__device__ __forceinline__ uint32_t wide_chunk(uint32_t row, uint32_t c) { return row * 256 + ((c ^ (row & 7)) << 4); }
__device__ __forceinline__ char *wide_at(float *base, int rows, int panel) {
    return reinterpret_cast<char *>(base) + (size_t)panel * rows * 256;
}

// u = g, or m <- mu m + g, u = g + mu m, for 8 values.
__device__ __forceinline__ void momentum8(float mu, float (&v)[8], float (&w)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = __fadd_rn(__fmul_rn(mu, w[k]), v[k]), v[k] = __fadd_rn(v[k], __fmul_rn(mu, w[k]));
}

// A chunk of a matrix: g read (m read and written), the sum of u's squares.  The matrix's last chunk adds the
// partial sums in their order.
template <typename T>
__device__ __forceinline__ void norm_chunk(const OrthArgs &a, uint32_t q, uint32_t chunk, float *red, int &last) {
    const OrthMat &M = a.mats[q];
    const T *g = static_cast<const T *>(a.grad) + M.offset;
    float *m = a.m ? a.m + M.offset : nullptr;
    const long long total = (long long)M.rows * M.cols, e0 = (long long)chunk * kNormChunk;
    const long long end = e0 + kNormChunk < total ? e0 + kNormChunk : total;
    float sum = 0.f;
    if (M.stride == M.cols && end - e0 == kNormChunk && (reinterpret_cast<uintptr_t>(g + e0) & 15) == 0 &&
        (!m || (reinterpret_cast<uintptr_t>(m + e0) & 15) == 0)) {
        for (long long e = e0 + threadIdx.x * 8; e < end; e += 4 * 2048) {
            float v[4][8], w[4][8];                // four loads of each under way at a time
#pragma unroll
            for (int k = 0; k < 4; ++k) load8(g + e + k * 2048, 8, v[k]);
            if (m) {
#pragma unroll
                for (int k = 0; k < 4; ++k) load8(m + e + k * 2048, 8, w[k]);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    momentum8(a.mu, v[k], w[k]);
                    float4 *o = reinterpret_cast<float4 *>(m + e + k * 2048);
                    o[0] = make_float4(w[k][0], w[k][1], w[k][2], w[k][3]), o[1] = make_float4(w[k][4], w[k][5], w[k][6], w[k][7]);
                }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int p = 0; p < 8; ++p) sum = __fmaf_rn(v[k][p], v[k][p], sum);
        }
    } else if (M.stride == M.cols) {
        for (long long e = e0 + threadIdx.x * 8; e < end; e += 2048) {
            const int n = end - e < 8 ? (int)(end - e) : 8;
            float v[8], w[8];
            load8(g + e, n, v);
            if (m) {
                load8(m + e, n, w);
                momentum8(a.mu, v, w);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k < n) m[e + k] = w[k];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < n) sum = __fmaf_rn(v[k], v[k], sum);
        }
    } else {
        for (long long e = e0 + threadIdx.x; e < end; e += 256) {
            const long long r = e / M.cols, at = r * M.stride + (e - r * M.cols);
            float v = to_f<T>(g[at]);
            if (m) {
                const float w = __fadd_rn(__fmul_rn(a.mu, m[at]), v);
                m[at] = w;
                v = __fadd_rn(v, __fmul_rn(a.mu, w));
            }
            sum = __fmaf_rn(v, v, sum);
        }
    }
    for (int k = 16; k; k >>= 1) sum += __shfl_xor_sync(~0u, sum, k);
    if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        float s = 0.f;
        for (int k = 0; k < 8; ++k) s += red[k];
        a.partial[M.chunk0 + chunk] = s;
        __threadfence();
        last = atomicAdd(&a.ticket[q], 1u) == (unsigned)M.chunks - 1;
        __threadfence();
    }
    __syncthreads();
    if (!last) return;
    float s = 0.f;
#pragma unroll 8
    for (int k = threadIdx.x; k < M.chunks; k += 256) s += __ldcg(&a.partial[M.chunk0 + k]);
    for (int k = 16; k; k >>= 1) s += __shfl_xor_sync(~0u, s, k);
    __syncthreads();
    if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.f;
        for (int k = 0; k < 8; ++k) s += red[k];
        a.inv[q] = __fdiv_rn(1.f, __fadd_rn(__fsqrt_rn(s), kEps));
        a.ticket[q] = 0;                           // for the next call
        a.done[q] = 0;
    }
    for (int k = threadIdx.x; k < M.n_joined; k += 256) M.joined[k] = 0;
}

// 32 rows of up to 4 panels: a thread makes one chunk of 8 columns per panel; the padding becomes 0.
template <typename T>
__device__ __forceinline__ void make_panels(const OrthArgs &a, uint32_t q, int r0, int c0) {
    const OrthMat &M = a.mats[q];
    const int row = r0 + threadIdx.x / 8, c = threadIdx.x % 8;
    const float f = __fmul_rn(__ldcg(a.inv + q), kScale);
    float v[4][8];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int col = c0 + p * 64 + c * 8;
        const int n = row < M.rows ? M.cols - col : 0;
        const long long at = M.offset + (long long)row * M.stride + col;
        if (n > 0) {
            load8(static_cast<const T *>(a.grad) + at, n, v[p]);
            if (a.m) {
                float w[8];
                load8(a.m + at, n, w);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[p][k] = __fadd_rn(v[p][k], __fmul_rn(a.mu, w[k]));
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[p][k] = 0.f;
        }
    }
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int col = c0 + p * 64;
        if (col >= M.cp) break;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[p][k] = __fmul_rn(v[p][k], f);
        uint4 hi, lo;
        split8(v[p], hi, lo);
        const uint32_t at = panel_chunk(row, c);
        *reinterpret_cast<uint4 *>(panel_at(M.xh[0], M.rp, col / 64) + at) = hi;
        *reinterpret_cast<uint4 *>(panel_at(M.xl[0], M.rp, col / 64) + at) = lo;
        if (M.xf[0]) {
            char *w = wide_at(M.xf[0], M.rp, col / 64);
            *reinterpret_cast<float4 *>(w + wide_chunk(row, 2 * c)) = make_float4(v[p][0], v[p][1], v[p][2], v[p][3]);
            *reinterpret_cast<float4 *>(w + wide_chunk(row, 2 * c + 1)) = make_float4(v[p][4], v[p][5], v[p][6], v[p][7]);
        }
    }
}

// Both bound by memory: making X needs the whole matrix's norm, so g (and m) are read twice.  (One kernel that makes a batch's panels
// while its g and m are still in L2 read less and was slower, 387 against 375 us for 8 x 12.6 M elements with momentum: its units'
// chain of dependent loads outweighed it.)
template <typename T>
__global__ void __launch_bounds__(256) orth_norm_kernel(const OrthArgs a) {
    __shared__ float red[8];
    __shared__ int last;
    let_next_start();
    const uint2 c = a.chunk[blockIdx.x];
    norm_chunk<T>(a, c.x, c.y, red, last);
}
template <typename T>
__global__ void __launch_bounds__(256) orth_convert_kernel(const OrthArgs a) {
    const PanelUnit u = a.unit[blockIdx.x];
    earlier_done();
    make_panels<T>(a, u.q, (int)u.r0, (int)u.c0);
}

// ------------------------------------------------------------------ products
enum { kPhaseA = 0, kPhaseB = 1, kPhaseX = 2 };

template <int MODE, bool SPLIT>
using OrthPipe = Pipe<mode_cg(MODE), tile_n(MODE, SPLIT), SPLIT ? 65536 : 98304, SPLIT>;

// SHARES: some of A's tiles are summed in shares (a kernel of its own: with that code in it, 32 matrices of 1024 x 1024 with 32-bit
// results, which have none, took 3160 us instead of 2710).
template <int MODE, bool SPLIT, bool SHARES>
struct OrthJob {
    using P = OrthPipe<MODE, SPLIT>;
    static constexpr int CG = mode_cg(MODE), TN = tile_n(MODE, SPLIT), kSums = SPLIT ? TN / 64 : 1, kPartFloats = 128 * TN;
    const OrthArgs &a;
    int first, every;
    static constexpr bool kCopier = true, kRemainders = false, kWaits = true;

    struct Tile {
        int n, stages, a_lim, b_lim;
        int phase, tall, last, row0, panel0, rp;                     // row0: of this CTA; rp: rows of a panel of what is written
        int row_a, row_b;                                            // first rows of the operands
        unsigned need, *done;
        const char *a_hi, *a_lo, *b_hi, *b_lo;                       // operands, their panels' bytes
        size_t a_panel, b_panel;
        char *dst_hi, *dst_lo, *dst_wide;
        const char *src_hi, *src_lo, *src_wide;                      // A or X, for the epilogue
        float *da, *db;
        long long offset, stride;
        int rows, cols;
        float scale;
        int share, shares;
        float *part;                                                 // of this CTA's tile, shares 0, 1, ... one after the other
        unsigned *joined;
        unsigned joins;                                              // what it has counted when all of this step's are there
    };

    __device__ __forceinline__ void tile(Tile &t, int k, int rank) const {
        t.n = 0;
        const long long at = first + (long long)k * every;
        const int per_step = a.n_a + a.n_sym + a.n_x;
        if (at >= (long long)per_step * a.steps) return;
        const int in = (int)at, step = in / per_step;
        int r = in - step * per_step, phase = kPhaseA;
        const OrthTile *list = a.a_tiles;
        if (r >= a.n_a) r -= a.n_a, phase = kPhaseB, list = a.sym;
        if (phase == kPhaseB && r >= a.n_sym) r -= a.n_sym, phase = kPhaseX, list = a.x;
        const OrthTile e = list[r];
        const OrthMat &M = a.mats[e.q];
        const int width = phase == kPhaseX ? M.cp : M.sp, from = step & 1, to = from ^ 1;
        t.n = width - e.j * TN < TN ? width - e.j * TN : TN;
        t.share = e.share, t.shares = phase == kPhaseA ? M.shares : 1;
        const int k0 = SHARES && phase == kPhaseA ? M.k_long * e.share / t.shares : 0;
        t.stages = phase != kPhaseA ? M.k_short : SHARES ? M.k_long * (e.share + 1) / t.shares - k0 : M.k_long;
        // Of a symmetric matrix the stages of the panels up to the row's own 256 are stored, the others as their mirror image.
        const int tri_a = (e.i * 128 * CG / 256 + 1) * 4, tri_b = (e.j * TN / 256 + 1) * 4;
        const bool sym_a = phase == kPhaseB || (phase == kPhaseX && !M.tall), sym_b = phase == kPhaseB || (phase == kPhaseX && M.tall);
        t.a_lim = phase == kPhaseA ? (M.tall ? 0 : t.stages) : sym_a ? tri_a : t.stages;
        t.b_lim = phase == kPhaseA ? (M.tall ? 0 : t.stages) : sym_b ? tri_b : 0;
        t.phase = phase, t.tall = M.tall, t.last = phase == kPhaseX && step == a.steps - 1;
        t.row0 = t.row_a = e.i * 128 * CG + rank * 128, t.row_b = e.j * TN + rank * (t.n / CG), t.panel0 = e.j * (TN / 64);
        t.need = (unsigned)step * (2 * M.tiles_sym + M.tiles_x) + (unsigned)phase * M.tiles_sym, t.done = a.done + e.q;
        if (phase == kPhaseB) t.need += a.stall;
        __half *sym_hi = phase == kPhaseB ? M.ah : M.bh, *sym_lo = phase == kPhaseB ? M.al : M.bl;
        t.a_hi = (const char *)(sym_a ? sym_hi : M.xh[from]), t.a_lo = (const char *)(sym_a ? sym_lo : M.xl[from]);
        t.b_hi = (const char *)(sym_b ? sym_hi : M.xh[from]), t.b_lo = (const char *)(sym_b ? sym_lo : M.xl[from]);
        if (SHARES) {
            const size_t on = (size_t)k0 * (M.tall ? 8192 : (size_t)M.rp * 128);   // to the share's first stage
            t.a_hi += on, t.a_lo += on, t.b_hi += on, t.b_lo += on;
            const size_t tile_at = (size_t)e.slot * CG + rank;
            t.part = M.part + tile_at * (t.shares - 1) * kPartFloats, t.joined = M.joined + tile_at * kEpiWarps;
            t.joins = (unsigned)(step + 1) * (t.shares - 1);
        }
        t.a_panel = (size_t)(sym_a ? M.sp : M.rp) * 128, t.b_panel = (size_t)(sym_b ? M.sp : M.rp) * 128;
        t.rp = phase == kPhaseX ? M.rp : M.sp;
        t.dst_hi = (char *)(phase == kPhaseA ? M.ah : phase == kPhaseB ? M.bh : M.xh[to]);
        t.dst_lo = (char *)(phase == kPhaseA ? M.al : phase == kPhaseB ? M.bl : M.xl[to]), t.dst_wide = (char *)M.xf[to];
        t.src_hi = (const char *)(phase == kPhaseB ? M.ah : M.xh[from]), t.src_lo = (const char *)(phase == kPhaseB ? M.al : M.xl[from]);
        t.src_wide = (const char *)M.xf[from], t.da = M.da, t.db = M.db;
        t.offset = M.offset, t.stride = M.stride, t.rows = M.rows, t.cols = M.cols, t.scale = M.scale;
    }
    __device__ __forceinline__ bool ready(P &p, const Tile &t) const { return !t.need || p.wait_counter(t.done, t.need); }
    __device__ __forceinline__ bool chunk_ends(const Tile &t, int k) const {
        return k + 1 == t.stages || (SPLIT && ((k + 1) & ((t.phase == kPhaseX ? kChunkX : kChunkAB) - 1)) == 0);
    }
    __device__ __forceinline__ int bf16() const { return 0; }
    // `count` rows from `row` on of a matrix of `rp` rows, stage by stage: its panel k, or, from stage `lim` on, as the columns of
    // its rows 64 k .. 64 k + 63.
    struct Operand {
        const char *k_major, *mn_major;
        size_t panel;
        long long lo;                                                // from hi to lo
        int lim;
        __device__ __forceinline__ Operand(const char *hi, const char *low, int row, size_t panel_bytes, int limit)
            : k_major(hi + (size_t)row * 128), mn_major(hi + (size_t)(row / 64) * panel_bytes), panel(panel_bytes), lo(low - hi), lim(limit) {}
        template <int COUNT>
        __device__ __forceinline__ void load(int k, int count, uint32_t dst, uint64_t *bar) const {
            if (k < lim) {
                const char *p = k_major + (size_t)k * panel;
                bulk_copy_in(dst, p, (uint32_t)count * 128, bar);
                if (SPLIT) bulk_copy_in(dst + P::kLoOffset, p + lo, (uint32_t)count * 128, bar);
            } else {
                const char *p = mn_major + (size_t)k * 8192;
#pragma unroll
                for (int e = 0; e < COUNT / 64; ++e)
                    if (e * 64 < count) {
                        bulk_copy_in(dst + e * 8192, p + (size_t)e * panel, 8192, bar);
                        if (SPLIT) bulk_copy_in(dst + P::kLoOffset + e * 8192, p + (size_t)e * panel + lo, 8192, bar);
                    }
            }
        }
    };
    struct Loader {
        int nb;
        Operand x, y;
        __device__ __forceinline__ Loader(const OrthJob &, const Tile &t)
            : nb(t.n / CG), x(t.a_hi, t.a_lo, t.row_a, t.a_panel, t.a_lim), y(t.b_hi, t.b_lo, t.row_b, t.b_panel, t.b_lim) {}
        __device__ __forceinline__ uint32_t bytes() const { return (128 * 128 + (uint32_t)nb * 128) * (SPLIT ? 2 : 1); }
        __device__ __forceinline__ void load(int k, uint32_t sa, uint32_t sb, uint64_t *bar) const {
            x.template load<128>(k, 128, sa, bar);
            y.template load<TN / CG>(k, nb, sb, bar);
        }
    };

    // The epilogue goes panel by panel (64 columns): a thread has 16 columns of a row.  What it needs of A or X, and what
    // it makes, passes through shared memory, brought and taken away by bulk copies that a thread of its own issues: written
    // from the registers, 16 bytes to a row, the same epilogue took twice the time of a tile's products at an inner dimension
    // of 1024.  fp16 results have three buffers of 32 KB (operand, remainder), so that most of a tile's panels are
    // there when its products end; 32-bit ones one of 64 KB.
    static constexpr int kBufs = SPLIT ? 1 : 3;
    static constexpr uint32_t kLo = 16384, kWide = 32768, kBufBytes = SPLIT ? 65536 : 32768;
    // Next buffer, and the parity of each one's barriers: every role keeps its own.
    struct Ring {
        uint32_t buf = 0, ph = 0;
        __device__ __forceinline__ uint32_t parity() const { return ph >> buf & 1; }
        __device__ __forceinline__ void step() {
            ph ^= 1u << buf;
            if (++buf == kBufs) buf = 0;
        }
    };
    Ring ring, ring_in;

    __device__ __forceinline__ void load_panel(P &p, const Tile &t, int b) {
        const uint32_t at = p.extra + ring_in.buf * kBufBytes;
        uint64_t *bar = &p.sh->extra_full[ring_in.buf];
        const size_t from = ((size_t)(t.panel0 + b) * t.rp + t.row0) * 128;
        if (t.phase == kPhaseA) {
            mbar_arrive(bar);
        } else if (SPLIT && t.phase == kPhaseX) {
            mbar_arrive_expect(bar, 32768);
            bulk_copy_in(at + kWide, t.src_wide + 2 * from, 32768, bar);
        } else {
            const bool lo = SPLIT || t.phase == kPhaseX;
            mbar_arrive_expect(bar, lo ? 32768 : 16384);
            bulk_copy_in(at, t.src_hi + from, 16384, bar);
            if (lo) bulk_copy_in(at + kLo, t.src_lo + from, 16384, bar);
        }
        ring_in.step();
    }
    __device__ __forceinline__ void store_panel(P &p, const Tile &t, int b) const {
        const uint32_t at = p.extra + ring.buf * kBufBytes;
        const size_t to = ((size_t)(t.panel0 + b) * t.rp + t.row0) * 128;
        bulk_copy_out(t.dst_hi + to, at, 16384);
        if (SPLIT || t.phase == kPhaseX) bulk_copy_out(t.dst_lo + to, at + kLo, 16384);
        if (SPLIT && t.phase == kPhaseX) bulk_copy_out(t.dst_wide + 2 * to, at + kWide, 32768);
        bulk_out_commit();
    }
    // The finished panel in the buffer, in the result's type, to the caller's rows: consecutive threads take consecutive chunks.
    __device__ __forceinline__ void store_result(P &p, const Tile &t, int panel, int tid) const {
        const uint32_t at = p.extra + ring.buf * kBufBytes;
        constexpr int kChunk = SPLIT ? 4 : 8, kSize = SPLIT ? 4 : 2;  // columns of a chunk, bytes of an element
#pragma unroll 4
        for (int k = tid; k < 128 * 64 / kChunk; k += kEpiWarps * 32) {
            const int r = k / (64 / kChunk), c = k % (64 / kChunk), col = panel * 64 + c * kChunk, n = t.cols - col;
            if (t.row0 + r >= t.rows || n <= 0) continue;
            const uint4 v = shared_load16(at + (SPLIT ? kWide + wide_chunk(r, c) : panel_chunk(r, c)));
            char *o = static_cast<char *>(a.out) + (t.offset + (long long)(t.row0 + r) * t.stride + col) * kSize;
            if (n >= kChunk && (reinterpret_cast<uintptr_t>(o) & 15) == 0) {
                *reinterpret_cast<uint4 *>(o) = v;
            } else {
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < kChunk; ++e) {
                    if (e >= n) break;
                    if (SPLIT) reinterpret_cast<uint32_t *>(o)[e] = w[e];
                    else reinterpret_cast<uint16_t *>(o)[e] = (uint16_t)(e & 1 ? w[e / 2] >> 16 : w[e / 2] & 0xffff);
                }
            }
        }
    }

    // The copying thread: loads panels in order as buffers come free, tile after tile, takes each finished panel away, and
    // tells the matrix's counter when a whole tile is in memory.  It never blocks on a later tile (what that waits for may be this
    // CTA's own) while there is a panel to take away.
    __device__ __forceinline__ bool copier(P &p) {
        typename P::Walk ahead, behind;                              // tile of the next load, of the next panel to take away
        int b_in = 0, b_out = 0, used = 0;                           // panels of these, buffers in use
        bool end = false, known = false, signal = false;
        long long t0 = clock64();
        for (;;) {
            bool moved = false;
            if (signal) {                                            // before anything else: the next phase waits for it
                const Tile &t = *p.template tile_at<Tile>(behind);
                bulk_out_done();                                     // written; the next phase's readers fence their own copies
                asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(t.done) : "memory");
                signal = false, moved = true;
                p.tile_done(behind);
            }
            while (!end && used < kBufs) {
                if (!known) {
                    if (!mbar_test(&p.sh->tile_full[ahead.slot], ahead.ph)) break;
                    known = true;
                    if (p.template tile_at<Tile>(ahead)->n == 0) {
                        end = true;
                        break;
                    }
                    fence_async_global();                            // what the tile's phase reads, for the copy engine
                }
                const Tile &t = *p.template tile_at<Tile>(ahead);
                bulk_out_read<0>();
                load_panel(p, t, b_in);
                ++used, moved = true;
                if (++b_in == t.n / 64) b_in = 0, known = false, ahead.step();
            }
            if (used > 0) {
                const Tile &t = *p.template tile_at<Tile>(behind);
                if (mbar_test(t.last ? &p.sh->extra_free[ring.buf] : &p.sh->extra_done[ring.buf], ring.parity())) {
                    const bool leaves = SHARES && t.share + 1 < t.shares;   // only sums, which are not a panel's
                    if (!t.last && !leaves) store_panel(p, t, b_out);
                    ring.step();
                    --used, moved = true;
                    if (++b_out == t.n / 64) {
                        b_out = 0;
                        if (t.last || leaves) p.tile_done(behind);
                        else signal = true;
                    }
                }
            } else if (end && !signal) {
                return true;
            }
            if (moved) {
                t0 = clock64();
            } else {
                if (p.sh->dead) return false;
                if (clock64() - t0 > p.limit) {
                    p.fail();
                    return false;
                }
            }
        }
    }

    __device__ __forceinline__ bool epilogue(P &p, const Tile &t, typename P::Turn &turn, int warp, int lane) {
        const int tid = warp * 32 + lane, side = warp / 4, r = warp % 4 * 32 + lane, row = t.row0 + r, panels = t.n / 64;
        const bool last = t.last, tall = t.tall;
        const int phase = t.phase;
        float *da = t.da, *db = t.db;
        // What of the diagonals a column needs: of A for B, of B for the X of a tall matrix.
        const float *d_cols = phase == kPhaseB ? da : phase == kPhaseX && tall ? db : nullptr;
        const float d_row = phase == kPhaseB ? __ldcg(da + row) : phase == kPhaseX && !tall ? __ldcg(db + row) : 0.f;
        uint32_t tmem;
        float sum[kSums][16];                                        // of a 32-bit result's chunks
        if (SPLIT) {
            const int each = phase == kPhaseX ? kChunkX : kChunkAB, chunks = (t.stages + each - 1) / each;
            for (int c = 0; c <= chunks; ++c) {                      // hi hi, then the small products
                if (c < chunks ? !p.take(turn, tmem) : !p.take_small(turn, tmem)) return false;
#pragma unroll
                for (int b = 0; b < kSums; ++b) {
                    float v[16];
                    tmem_load(tmem + b * 64 + side * 16, v);
#pragma unroll
                    for (int k = 0; k < 16; ++k) sum[b][k] = __fadd_rn(c ? sum[b][k] : 0.f, v[k]);
                }
                if (c < chunks) p.release(turn, lane);
                else p.release_small(turn, lane);
            }
        } else if (!p.take(turn, tmem)) {
            return false;
        }
        const bool leaves = SHARES && t.share + 1 < t.shares;
        if (SHARES && t.shares > 1 && !leaves) {                               // the other shares' sums are there
            bool there = true;
            if (lane == 0) there = p.wait_counter(t.joined + warp, t.joins);
            if (!__shfl_sync(~0u, (int)there, 0)) return false;
        }
#pragma unroll kSums
        for (int b = 0; b < (SPLIT ? kSums : panels); ++b) {
            const int panel = t.panel0 + b, col = panel * 64 + side * 16;
            float4 d_col[4];                                         // asked for before the waits
#pragma unroll
            for (int k = 0; k < 4; ++k)
                d_col[k] = d_cols ? __ldcg(reinterpret_cast<const float4 *>(d_cols + col) + k) : make_float4(0.f, 0.f, 0.f, 0.f);
            if (!p.warp_wait(&p.sh->extra_full[ring.buf], ring.parity())) return false;
            const uint32_t at = p.extra + ring.buf * kBufBytes;
            float v[16];
            if (SPLIT) {
#pragma unroll
                for (int k = 0; k < 16; ++k) v[k] = sum[b][k];
            } else {
                tmem_load(tmem + b * 64 + side * 16, v);
                if (b + 1 == panels) p.release(turn, lane);
            }
            if (SHARES && t.shares > 1) {
                float4 *part = reinterpret_cast<float4 *>(t.part) + (size_t)b * 4 * (kEpiWarps * 32) + tid;
                if (leaves) {
                    part += (size_t)t.share * (kPartFloats / 4);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        part[k * kEpiWarps * 32] = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
                    if (lane == 0) mbar_arrive(&p.sh->extra_done[ring.buf]), mbar_arrive(&p.sh->extra_free[ring.buf]);
                    ring.step();
                    continue;
                }
#pragma unroll 1
                for (int e = 0; e + 1 < t.shares; ++e, part += kPartFloats / 4) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float4 q = __ldcg(part + k * kEpiWarps * 32);
                        v[4 * k] += q.x, v[4 * k + 1] += q.y, v[4 * k + 2] += q.z, v[4 * k + 3] += q.w;
                    }
                }
            }
            const unsigned on = (unsigned)(row - col);               // the diagonal is at column `on` of the 16, if below 16
            if (phase == kPhaseA) {
                if (on < 16u) {
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        if (on == (unsigned)k) da[row] = v[k] * kUnscale2, v[k] = 0.f;
                    __threadfence();
                }
#pragma unroll
                for (int k = 0; k < 16; ++k) v[k] *= kUnscale;
            } else {
                float x[16];
                if (SPLIT && phase == kPhaseX) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint4 f = shared_load16(at + kWide + wide_chunk(r, side * 4 + k));
                        x[4 * k] = __uint_as_float(f.x), x[4 * k + 1] = __uint_as_float(f.y);
                        x[4 * k + 2] = __uint_as_float(f.z), x[4 * k + 3] = __uint_as_float(f.w);
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        unpack8(shared_load16(at + panel_chunk(r, side * 2 + k)), x + 8 * k);
                        if (SPLIT || phase == kPhaseX) {
                            float l[8];
                            unpack8(shared_load16(at + kLo + panel_chunk(r, side * 2 + k)), l);
#pragma unroll
                            for (int e = 0; e < 8; ++e) x[8 * k + e] += l[e];
                        }
                    }
                }
                if (phase == kPhaseB) {
                    // x is A without its diagonal, times 2^12
                    if (on < 16u) {
#pragma unroll
                        for (int k = 0; k < 16; ++k)
                            if (on == (unsigned)k)
                                db[row] = __fmaf_rn(kC, __fmaf_rn(d_row, d_row, v[k] * kUnscale2), kB * d_row), v[k] = 0.f;
                        __threadfence();
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float4 dc = d_col[k];
                        const float d[4] = {dc.x, dc.y, dc.z, dc.w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int i = 4 * k + e;
                            const float sq = __fmaf_rn(d_row + d[e], x[i], v[i] * kUnscale);
                            v[i] = on == (unsigned)i ? 0.f : __fmaf_rn(kC, sq, kB * x[i]);
                        }
                    }
                } else if (tall) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float4 dc = d_col[k];
                        const float d[4] = {dc.x, dc.y, dc.z, dc.w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[4 * k + e] = __fmaf_rn(kA + d[e], x[4 * k + e], v[4 * k + e] * kUnscale);
                    }
                } else {
                    const float f = kA + d_row;
#pragma unroll
                    for (int k = 0; k < 16; ++k) v[k] = __fmaf_rn(f, x[k], v[k] * kUnscale);
                }
            }
            if (last) {
                const float f = kUnscale * t.scale;
#pragma unroll
                for (int k = 0; k < 16; ++k) v[k] *= f;
            }
            if (!(SPLIT && last)) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float *e = v + 8 * k;
                    uint4 hi, lo;
                    split8(e, hi, lo);
                    if (last && a.out_type == CSER_TYPE_BF16)
                        hi = make_uint4(pack_bf162(e[0], e[1]), pack_bf162(e[2], e[3]), pack_bf162(e[4], e[5]), pack_bf162(e[6], e[7]));
                    shared_store16(at + panel_chunk(r, side * 2 + k), hi);
                    if (SPLIT || phase == kPhaseX) shared_store16(at + kLo + panel_chunk(r, side * 2 + k), lo);
                }
            }
            if (SPLIT && phase == kPhaseX) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    shared_store16(at + kWide + wide_chunk(r, side * 4 + k),
                                   make_uint4(__float_as_uint(v[4 * k]), __float_as_uint(v[4 * k + 1]), __float_as_uint(v[4 * k + 2]),
                                              __float_as_uint(v[4 * k + 3])));
            }
            fence_async_shared();
            __syncwarp();
            if (lane == 0) mbar_arrive(&p.sh->extra_done[ring.buf]);
            if (last) {
                if (!p.warp_wait(&p.sh->extra_done[ring.buf], ring.parity())) return false;
                store_result(p, t, panel, tid);
                fence_async_shared();                                // read before the copy engine writes here again
                __syncwarp();
            }
            if (lane == 0) mbar_arrive(&p.sh->extra_free[ring.buf]);
            ring.step();
        }
        if (leaves) {
            __syncwarp();
            if (lane == 0) {
                __threadfence();
                asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(t.joined + warp) : "memory");
            }
        }
        return true;
    }
};

template <int MODE, bool SPLIT, bool SHARES>
__global__ void __launch_bounds__(kThreads, 1) orth_products_kernel(const __grid_constant__ OrthArgs a) {
    extern __shared__ unsigned char raw[];
    constexpr int CG = mode_cg(MODE);
    OrthPipe<MODE, SPLIT> p;
    p.template setup<OrthJob<MODE, SPLIT, SHARES>>(raw, a.err, a.wait_cycles);
    OrthJob<MODE, SPLIT, SHARES> job{a, (int)blockIdx.x / CG, (int)gridDim.x / CG};
    p.run(job);
    p.teardown();
}

}  // namespace

// ------------------------------------------------------------------ host
struct cser_orth {
    struct Group {
        int mode = kSingle, grid = 0, n_chunk = 0, n_unit = 0;
        bool shares = false;
        OrthArgs args{};
        void *tables = nullptr;                    // one allocation for the lists and matrices
    };
    int device = 0, in_type = 0, out_type = 0;
    long long first = 0, last = 0;                 // elements of the [n, ld] arrays that the matrices begin and end at
    bool split = false;
    std::vector<Group> groups;
    struct Small {                                 // matrices with a short side of at most kSmallSide
        SmallArgs args{};
        int n_part = 0, n_piece = 0, n_resident = 0, side = 0;
        size_t gram_shared = 0, apply_shared = 0, resident_shared = 0;
        void *tables = nullptr;
    } small, resident;                             // resident: those of them that fit a CTA's shared memory
    // Small matrices run beside the large ones, on a stream of the plan's own.
    cudaStream_t side = nullptr;
    cudaEvent_t fork = nullptr, join = nullptr;
    void *work = nullptr;                          // shared by the groups, which run one after the other
    unsigned *err_host = nullptr;
    unsigned stall_mcycles = 0;                    // cser_orth_debug_stall_next
    long long launches = 0;
};

namespace {

struct HostMat {
    long long offset, rows, cols, stride;
    float scale;
};

int type_size(int t) { return t == CSER_TYPE_F32 ? 4 : 2; }

template <int MODE, bool SPLIT>
cudaError_t products_launch(const OrthArgs &a, bool shares, int grid, cudaStream_t st) {
    constexpr int CG = mode_cg(MODE);
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = OrthPipe<MODE, SPLIT>::kSharedBytes;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeCooperative;
    at[0].val.cooperative = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = CG, at[1].val.clusterDim.y = 1, at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = CG == 1 ? 1 : 2;
    return cudaLaunchKernelEx(&cfg, shares ? orth_products_kernel<MODE, SPLIT, true> : orth_products_kernel<MODE, SPLIT, false>, a);
}
template <int MODE, bool SPLIT>
cudaError_t products_setup(int &pairs) {
    constexpr int CG = mode_cg(MODE);
    cudaError_t e = cudaFuncSetAttribute(orth_products_kernel<MODE, SPLIT, false>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         (int)OrthPipe<MODE, SPLIT>::kSharedBytes);
    if (e == cudaSuccess)
        e = cudaFuncSetAttribute(orth_products_kernel<MODE, SPLIT, true>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 (int)OrthPipe<MODE, SPLIT>::kSharedBytes);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(CG);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = OrthPipe<MODE, SPLIT>::kSharedBytes;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = CG, at[0].val.clusterDim.y = 1, at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    int with_shares = 0;
    e = cudaOccupancyMaxActiveClusters(&pairs, orth_products_kernel<MODE, SPLIT, false>, &cfg);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveClusters(&with_shares, orth_products_kernel<MODE, SPLIT, true>, &cfg);
    if (with_shares < pairs) pairs = with_shares;
    return e;
}

// Whether two matrices of one worker's vector share an element.  Those whose spans meet (columns of one array) row by row.
bool any_overlap(std::vector<HostMat> ms) {
    auto span_end = [](const HostMat &m) { return m.offset + (m.rows - 1) * m.stride + m.cols; };
    std::sort(ms.begin(), ms.end(), [](const HostMat &x, const HostMat &y) { return x.offset < y.offset; });
    std::vector<std::pair<long long, long long>> run;
    for (size_t k = 0; k < ms.size();) {
        long long end = span_end(ms[k]);
        size_t to = k + 1;
        for (; to < ms.size() && ms[to].offset < end; ++to) end = std::max(end, span_end(ms[to]));
        if (to > k + 1) {
            run.clear();
            for (; k < to; ++k) {
                const bool dense = ms[k].stride == ms[k].cols;
                for (long long r = 0; r < (dense ? 1 : ms[k].rows); ++r) {
                    const long long at = ms[k].offset + r * ms[k].stride;
                    run.emplace_back(at, dense ? span_end(ms[k]) : at + ms[k].cols);
                }
            }
            std::sort(run.begin(), run.end());
            for (size_t e = 1; e < run.size(); ++e)
                if (run[e].first < run[e - 1].second) return true;
        }
        k = to;
    }
    return false;
}

int orth_fail(cser_orth *h, int code, const char *what) {
    cser_internal_fail(code, "cser_orth_create: %s", what);
    cser_orth_destroy(h);
    return code;
}

// Padded dimensions and workspace of one matrix.
void shape_of(const HostMat &m, int cg, OrthMat &M) {
    M = OrthMat{};
    M.rows = (int)m.rows, M.cols = (int)m.cols, M.tall = m.rows > m.cols;
    M.rp = (int)up(m.rows, 128 * cg), M.cp = (int)up(m.cols, 128 * cg), M.sp = M.tall ? M.cp : M.rp;
    M.k_long = (int)(up(M.tall ? m.rows : m.cols, 64) / 64), M.k_short = (int)(up(M.tall ? m.cols : m.rows, 64) / 64);
    M.offset = m.offset, M.stride = m.stride, M.scale = m.scale;
}
size_t work_of(const OrthMat &M, bool split) {
    return (size_t)M.rp * M.cp * 2 * (split ? 8 : 4) + (size_t)M.sp * M.sp * 2 * (split ? 4 : 2) + (size_t)M.sp * 8;
}

// How a plan's tiles are cut, by the padded elements of all its matrices.  Pairs bring half the bytes per product: two of 2048 x
// 4096 548 us, single CTAs 744, narrow tiles 1317 (16-bit results; 32-bit 1726, 1817, 2684).  They need tiles for all SMs
// (1024 x 4096: 314, 303, 327) and matrices that 256 rows do not pad much.  Where there are few tiles the chain of phases is the
// bound and narrow ones shorten its links (512 x 512: 193, 141, 125; 8 workers' 256 x 256 and 256 x 1024: 205, 157, 143; 8 of 768 x
// 768, 288 tiles of 128 x 128: 235, 204, 220).
int choose_mode(const std::vector<HostMat> &all, bool split, int pairs, int sms) {
    double area[3] = {0, 0, 0};
    for (const HostMat &m : all)
        for (int cg = 1; cg <= 2; ++cg) {
            OrthMat M;
            shape_of(m, cg, M);
            area[cg] += (double)M.rp * M.cp;
        }
    if (area[2] <= 1.15 * area[1] && area[2] >= 256.0 * tile_n(kPaired, split) * pairs) return kPaired;
    return area[1] < 1.5 * 16384.0 * sms ? kNarrow : kSingle;
}

// In how many shares a matrix's tiles of A sum their inner dimension, where there are idle CTAs for them: so that the stages of
// one, and what joining costs in their time, are fewest.  Joining: 8 stages' time, and 2.5 for each share's sums (22 and 4
// where they are of 128 x 256 for each of a pair).  One of 100 x 60000 1560 us -> 300 (16-bit; 32-bit 3450 -> 590), two of
// 256 x 16384 580 -> 285 (1150 -> 555), 1024 x 4096 276 -> 239; with a share for every 8 stages 8 of 512 x 2048 went from 223 to 241.
int choose_shares(int tiles, int ctas, int k_long, bool wide) {
    int best = 1;
    double least = k_long;
    for (int s = 2; s <= ctas / tiles && s <= k_long; ++s) {
        const double cost = (double)k_long / s + (wide ? 22 + 4 * s : 8 + 2.5 * s);
        if (cost < least) best = s, least = cost;
    }
    return best;
}

int build_group(cser_orth *h, cser_orth::Group &G, const std::vector<HostMat> &ms, int mode, int steps, int ctas) {
    const int cg = mode_cg(mode);
    std::vector<OrthMat> mats(ms.size());
    std::vector<OrthTile> as, sym, xs;
    std::vector<uint2> chunk;
    std::vector<PanelUnit> unit;
    size_t at = 0;
    char *base = static_cast<char *>(h->work);
    int chunk0 = 0;
    for (size_t q = 0; q < ms.size(); ++q) {
        OrthMat &M = mats[q];
        shape_of(ms[q], cg, M);
        const size_t xb = (size_t)M.rp * M.cp * 2, ab = (size_t)M.sp * M.sp * 2;
        auto take = [&](size_t b) { char *p = base + at; at += b; return reinterpret_cast<__half *>(p); };
        M.xh[0] = take(xb), M.xl[0] = take(xb), M.xh[1] = take(xb), M.xl[1] = take(xb), M.ah = take(ab), M.bh = take(ab);
        if (h->split) {
            M.al = take(ab), M.bl = take(ab);
            for (float *&x : M.xf) x = reinterpret_cast<float *>(take(2 * xb));
        }
        M.da = reinterpret_cast<float *>(take((size_t)M.sp * 4)), M.db = reinterpret_cast<float *>(take((size_t)M.sp * 4));
        M.chunk0 = chunk0, M.chunks = (int)(up((long long)M.rows * M.cols, kNormChunk) / kNormChunk);
        chunk0 += M.chunks;
        for (int c = 0; c < M.chunks; ++c) chunk.push_back(make_uint2((unsigned)q, (unsigned)c));
        for (int r = 0; r < M.rp; r += 32)
            for (int c = 0; c < M.cp; c += 256) unit.push_back({(uint32_t)q, (uint32_t)r, (uint32_t)c});
        const int tm = 128 * cg, tn = tile_n(mode, h->split);
        for (int j = 0; j * tn < M.sp; ++j)
            for (int i = 0; i * tm < M.sp; ++i)
                if (i * tm / 256 >= j * tn / 256) sym.push_back({(uint32_t)q, (uint16_t)i, (uint16_t)j, 0, 0}), M.tiles_sym += cg;
        if (M.tall) {
            for (int i = 0; i * tm < M.rp; ++i)
                for (int j = 0; j * tn < M.cp; ++j) xs.push_back({(uint32_t)q, (uint16_t)i, (uint16_t)j, 0, 0}), M.tiles_x += cg;
        } else {
            for (int j = 0; j * tn < M.cp; ++j)
                for (int i = 0; i * tm < M.rp; ++i) xs.push_back({(uint32_t)q, (uint16_t)i, (uint16_t)j, 0, 0}), M.tiles_x += cg;
        }
    }
    // Kernels of small matrices beside this one need SMs of their own: it starts when all of its CTAs fit.
    const int beside = h->small.n_part + h->resident.n_resident, spare = beside * 4 < ctas ? beside : ctas / 4;
    const int most = ctas - (spare + cg - 1) / cg;
    size_t part_floats = 0, joins = 0;             // of the matrices' `part` and `joined`, at first as offsets
    std::vector<size_t> part_at(ms.size()), join_at(ms.size());
    for (size_t k = 0; k < sym.size();) {
        const uint32_t q = sym[k].q;
        OrthMat &M = mats[q];
        M.shares = choose_shares((int)sym.size(), most, M.k_long, tile_n(mode, h->split) == 256);
        part_at[q] = part_floats, join_at[q] = joins;
        const size_t k1 = k;
        for (; k < sym.size() && sym[k].q == q; ++k)
            for (int e = 0; e < M.shares; ++e) as.push_back({q, sym[k].i, sym[k].j, (uint16_t)e, (uint16_t)(k - k1)});
        G.shares |= M.shares > 1;
        M.n_joined = M.shares > 1 ? (int)(k - k1) * cg * kEpiWarps : 0;
        part_floats += (k - k1) * cg * (M.shares - 1) * 128 * tile_n(mode, h->split), joins += M.n_joined;
    }
    const size_t n = ms.size();
    size_t bytes = 0;
    auto place = [&](size_t b) { const size_t p = bytes; bytes += (b + 255) / 256 * 256; return p; };
    const size_t o_mat = place(n * sizeof(OrthMat)), o_as = place(as.size() * sizeof(OrthTile)), o_sym = place(sym.size() * sizeof(OrthTile)),
                 o_pt = place(part_floats * 4), o_join = place(joins * 4), o_x = place(xs.size() * sizeof(OrthTile)), o_ck = place(chunk.size() * sizeof(uint2)),
                 o_un = place(unit.size() * sizeof(PanelUnit)),
                 o_done = place(n * 4), o_tick = place(n * 4),
                 o_inv = place(n * 4), o_part = place((size_t)chunk0 * 4);
    TRY(cudaMalloc(&G.tables, bytes));
    char *t = static_cast<char *>(G.tables);
    TRY(cudaMemset(t + o_done, 0, bytes - o_done));
    for (size_t q = 0; q < n; ++q) {
        mats[q].part = reinterpret_cast<float *>(t + o_pt) + part_at[q];
        mats[q].joined = reinterpret_cast<unsigned *>(t + o_join) + join_at[q];
    }
    TRY(cudaMemcpy(t + o_mat, mats.data(), n * sizeof(OrthMat), cudaMemcpyHostToDevice));
    TRY(cudaMemcpy(t + o_as, as.data(), as.size() * sizeof(OrthTile), cudaMemcpyHostToDevice));
    TRY(cudaMemcpy(t + o_sym, sym.data(), sym.size() * sizeof(OrthTile), cudaMemcpyHostToDevice));
    TRY(cudaMemcpy(t + o_x, xs.data(), xs.size() * sizeof(OrthTile), cudaMemcpyHostToDevice));
    TRY(cudaMemcpy(t + o_un, unit.data(), unit.size() * sizeof(PanelUnit), cudaMemcpyHostToDevice));
    TRY(cudaMemcpy(t + o_ck, chunk.data(), chunk.size() * sizeof(uint2), cudaMemcpyHostToDevice));
    OrthArgs &A = G.args;
    A.n_a = (int)as.size(), A.n_sym = (int)sym.size(), A.n_x = (int)xs.size(), A.steps = steps;
    A.mats = reinterpret_cast<OrthMat *>(t + o_mat);
    A.a_tiles = reinterpret_cast<OrthTile *>(t + o_as);
    A.sym = reinterpret_cast<OrthTile *>(t + o_sym);
    A.x = reinterpret_cast<OrthTile *>(t + o_x);
    A.chunk = reinterpret_cast<uint2 *>(t + o_ck), A.unit = reinterpret_cast<PanelUnit *>(t + o_un);
    A.done = reinterpret_cast<unsigned *>(t + o_done), A.ticket = reinterpret_cast<unsigned *>(t + o_tick);
    A.inv = reinterpret_cast<float *>(t + o_inv), A.partial = reinterpret_cast<float *>(t + o_part);
    A.out_type = h->out_type;
    G.n_chunk = (int)chunk.size(), G.n_unit = (int)unit.size(), G.mode = mode;
    const int widest = A.n_a > A.n_x ? A.n_a : A.n_x;               // there are at least as many tiles of A as of B
    G.grid = (widest < most ? widest : most) * cg;
    return CSER_OK;
}

// `ctas`: SMs for these alone.
int build_small(cser_orth *h, const std::vector<HostMat> &ms, int steps, int ctas) {
    std::vector<SmallMat> mats(ms.size());
    std::vector<uint2> part, piece;
    size_t work = 0;
    int most = 0;
    for (size_t q = 0; q < ms.size(); ++q) {
        SmallMat &M = mats[q];
        M.tall = ms[q].rows > ms[q].cols;
        M.s = (int)(M.tall ? ms[q].cols : ms[q].rows), M.l = (int)(M.tall ? ms[q].rows : ms[q].cols), M.sp = (int)up(M.s, 8);
        M.offset = ms[q].offset, M.stride = ms[q].stride, M.scale = ms[q].scale;
        // Parts of at least one piece of u in shared memory, and 16 at most, since the last CTA adds them up alone, or as many as there
        // are SMs that would be idle (one of 64 x 60000: 640 us by 16, 215 by 148).
        const long long cols = kGramDoubles / gram_ld(M.sp) / 4 * 4, fit = up(M.l, cols) / cols;
        const int idle = ctas / (int)ms.size(), top = idle < 16 ? 16 : idle;
        M.parts = fit < top ? (int)fit : top;
        M.per = (int)(up(up(M.l, M.parts) / M.parts, cols));
        M.parts = (int)(up(M.l, M.per) / M.per);
        const int side = M.sp / 8;
        M.partial = work, work += (size_t)M.parts * side * (side + 1) / 2 * 64;
        M.q = work, work += (size_t)M.sp * M.sp;
        for (int k = 0; k < M.parts; ++k) part.push_back(make_uint2((unsigned)q, (unsigned)k));
        for (int j = 0; j < M.l; j += kApplyCols) piece.push_back(make_uint2((unsigned)q, (unsigned)j));
        if (M.sp > most) most = M.sp;
    }
    size_t bytes = 0;
    auto place = [&](size_t b) { const size_t p = bytes; bytes += (b + 255) / 256 * 256; return p; };
    const size_t o_mat = place(mats.size() * sizeof(SmallMat)), o_part = place(part.size() * sizeof(uint2)),
                 o_piece = place(piece.size() * sizeof(uint2)), o_tick = place(mats.size() * 4), o_work = place(work * 8);
    cser_orth::Small &S = h->small;
    TRY(cudaMalloc(&S.tables, bytes));
    char *t = static_cast<char *>(S.tables);
    TRY(cudaMemset(t + o_tick, 0, mats.size() * 4));
    TRY(cudaMemcpy(t + o_mat, mats.data(), mats.size() * sizeof(SmallMat), cudaMemcpyHostToDevice));
    TRY(cudaMemcpy(t + o_part, part.data(), part.size() * sizeof(uint2), cudaMemcpyHostToDevice));
    TRY(cudaMemcpy(t + o_piece, piece.data(), piece.size() * sizeof(uint2), cudaMemcpyHostToDevice));
    S.args.mats = reinterpret_cast<SmallMat *>(t + o_mat), S.args.part = reinterpret_cast<uint2 *>(t + o_part);
    S.args.piece = reinterpret_cast<uint2 *>(t + o_piece), S.args.ticket = reinterpret_cast<unsigned *>(t + o_tick);
    S.args.work = reinterpret_cast<double *>(t + o_work), S.args.out_type = h->out_type, S.args.steps = steps;
    S.n_part = (int)part.size(), S.n_piece = (int)piece.size();
    const size_t four = (size_t)most * square_ld(most) * 4;
    S.gram_shared = (four > kGramDoubles ? four : kGramDoubles) * 8;
    S.apply_shared = ((size_t)most * square_ld(most) + (size_t)most * kApplyLd) * 8;
    return CSER_OK;
}
int build_resident(cser_orth *h, const std::vector<HostMat> &ms, int steps) {
    std::vector<SmallMat> mats(ms.size());
    cser_orth::Small &S = h->resident;
    for (size_t q = 0; q < ms.size(); ++q) {
        SmallMat &M = mats[q];
        M.tall = ms[q].rows > ms[q].cols;
        M.s = (int)(M.tall ? ms[q].cols : ms[q].rows), M.l = (int)(M.tall ? ms[q].rows : ms[q].cols), M.sp = (int)up(M.s, 8);
        M.offset = ms[q].offset, M.stride = ms[q].stride, M.scale = ms[q].scale;
        const size_t b = resident_bytes(M.sp, M.l);
        if (b > S.resident_shared) S.resident_shared = b;
        if (M.sp > S.side) S.side = M.sp;
    }
    TRY(cudaMalloc(&S.tables, mats.size() * sizeof(SmallMat)));
    TRY(cudaMemcpy(S.tables, mats.data(), mats.size() * sizeof(SmallMat), cudaMemcpyHostToDevice));
    S.args.mats = static_cast<SmallMat *>(S.tables), S.args.out_type = h->out_type, S.args.steps = steps;
    S.n_resident = (int)mats.size();
    return CSER_OK;
}
template <typename T>
cudaError_t small_setup(const cser_orth::Small &S) {
    cudaError_t e = cudaFuncSetAttribute(orth_gram_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S.gram_shared);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(orth_apply_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S.apply_shared);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(orth_resident_kernel<T, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S.resident_shared);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(orth_resident_kernel<T, 4>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S.resident_shared);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(orth_resident_kernel<T, 8>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S.resident_shared);
    return e;
}
template <typename T>
cudaError_t small_launch(const cser_orth::Small &S, const SmallArgs &a, cudaStream_t st) {
    if (S.n_resident) {
        return launch_kernel(S.side <= 16 ? orth_resident_kernel<T, 2> : S.side <= 32 ? orth_resident_kernel<T, 4> : orth_resident_kernel<T, 8>, (unsigned)S.n_resident, 256, S.resident_shared,
                             1, false, st, a);
    }
    cudaError_t e = launch_kernel(orth_gram_kernel<T>, (unsigned)S.n_part, 256, S.gram_shared, 1, false, st, a);
    return e == cudaSuccess ? launch_kernel(orth_apply_kernel<T>, (unsigned)S.n_piece, 256, S.apply_shared, 1, true, st, a) : e;
}

template <typename T>
cudaError_t prologue_launch(const cser_orth::Group &G, const OrthArgs &a, cudaStream_t st) {
    // The norm kernel follows the group before it (or another call), whose products read what it writes: no overlap there.
    cudaError_t e = launch_kernel(orth_norm_kernel<T>, (unsigned)G.n_chunk, 256, 0, 1, false, st, a);
    return e == cudaSuccess ? launch_kernel(orth_convert_kernel<T>, (unsigned)G.n_unit, 256, 0, 1, true, st, a) : e;
}

}  // namespace

extern "C" {

cser_orth_handle cser_orth_create(int32_t n_workers, int64_t ld, int32_t n_matrices, const int64_t *offset,
                                  const int64_t *rows, const int64_t *cols, const int64_t *row_stride,
                                  const float *scale, int32_t steps, int32_t in_type, int32_t out_type) {
    auto bad = [](const char *what) { cser_internal_fail(CSER_ERR_INVALID, "cser_orth_create: %s", what); return nullptr; };
    if (n_workers < 1 || ld < 1 || n_matrices < 1) return bad("n_workers, ld and n_matrices must be positive");
    if (!offset || !rows || !cols) return bad("offset, rows and cols must not be NULL");
    if (steps < 1 || steps > 16) return bad("steps must be in 1..16");
    if (in_type < 0 || in_type > 2 || out_type < 0 || out_type > 2) return bad("unknown element type");
    if ((long long)n_workers * n_matrices > (1 << 20)) return bad("more than 2^20 matrices");
    if (ld > (1ll << 46) / n_workers) return bad("n_workers * ld must be at most 2^46");   // and no sum below overflows
    std::vector<HostMat> one, all, small;          // of one worker; of all of them
    cser_orth *h = nullptr;
    try {
        for (int k = 0; k < n_matrices; ++k) {
            const long long st = row_stride ? row_stride[k] : cols[k];
            if (rows[k] < 1 || cols[k] < 1 || rows[k] > 65536 || cols[k] > 65536) return bad("rows and cols must be in 1..65536");
            if (st < cols[k] || st > ld) return bad("row_stride must be at least cols and at most ld");
            if (offset[k] < 0 || offset[k] > ld || offset[k] + (rows[k] - 1) * st + cols[k] > ld)
                return bad("a matrix reaches outside the vector");
            if (scale && !isfinite(scale[k])) return bad("scale must be finite");
            one.push_back({offset[k], rows[k], cols[k], st, scale ? scale[k] : 1.f});
        }
        if (any_overlap(one)) return bad("two matrices overlap");
        for (int w = 0; w < n_workers; ++w)
            for (HostMat m : one) {
                m.offset += (long long)w * ld;
                (m.rows <= kSmallSide || m.cols <= kSmallSide ? small : all).push_back(m);
            }
        h = new cser_orth;
        h->in_type = in_type, h->out_type = out_type, h->split = out_type == CSER_TYPE_F32;
        h->first = ld;
        for (const HostMat &m : one) {
            h->first = std::min(h->first, m.offset);
            h->last = std::max(h->last, (n_workers - 1) * (long long)ld + m.offset + (m.rows - 1) * m.stride + m.cols);
        }
        if (cudaGetDevice(&h->device) != cudaSuccess) {
            orth_fail(h, CSER_ERR_CUDA, "no CUDA device");
            return nullptr;
        }
        int fit_ctas[3] = {0, 0, 0};               // CTAs (pairs) of each mode that are resident together
        cudaError_t er = h->split ? products_setup<kNarrow, true>(fit_ctas[kNarrow]) : products_setup<kNarrow, false>(fit_ctas[kNarrow]);
        if (er == cudaSuccess)
            er = h->split ? products_setup<kSingle, true>(fit_ctas[kSingle]) : products_setup<kSingle, false>(fit_ctas[kSingle]);
        if (er == cudaSuccess)
            er = h->split ? products_setup<kPaired, true>(fit_ctas[kPaired]) : products_setup<kPaired, false>(fit_ctas[kPaired]);
        if (er != cudaSuccess || fit_ctas[kNarrow] < 1 || fit_ctas[kSingle] < 1 || fit_ctas[kPaired] < 1) {
            orth_fail(h, CSER_ERR_CUDA, er != cudaSuccess ? cudaGetErrorString(er) : "the kernel does not fit this GPU");
            return nullptr;
        }
        const int mode = choose_mode(all, h->split, fit_ctas[kPaired], fit_ctas[kSingle]), cg = mode_cg(mode);
        // Groups that fit the workspace, one after the other.
        std::vector<std::vector<HostMat>> parts;
        size_t most = 0, now = 0;
        for (const HostMat &m : all) {
            OrthMat M;
            shape_of(m, cg, M);
            const size_t need = work_of(M, h->split);
            if (parts.empty() || now + need > kGroupBytes) parts.emplace_back(), now = 0;
            parts.back().push_back(m);
            now += need;
            if (now > most) most = now;
        }
        if (most) er = cudaMalloc(&h->work, most);
        std::vector<HostMat> fit, rest;
        for (const HostMat &m : small) {
            const long long side = m.rows < m.cols ? m.rows : m.cols, longer = m.rows < m.cols ? m.cols : m.rows;
            // One CTA for a whole matrix pays where there are matrices for most SMs, or little to do: 33 x 1000 took 100 us alone,
            // against 54 by two kernels that spread it; 384 of 16 x 1024 took 48 against 120.
            const bool pays = (int)small.size() >= fit_ctas[kPaired] || side * side * longer <= 1 << 19;
            (pays && resident_bytes((int)up(side, 8), longer) <= kResidentMost ? fit : rest).push_back(m);
        }
        if (er == cudaSuccess && !small.empty()) {
            if ((!rest.empty() && build_small(h, rest, steps, all.empty() ? fit_ctas[kSingle] : 0) != CSER_OK) || (!fit.empty() && build_resident(h, fit, steps) != CSER_OK)) {
                cser_orth_destroy(h);
                return nullptr;
            }
            // shared memory is a property of the kernel, not of the plan: what any plan can need
            cser_orth::Small any;
            any.gram_shared = (size_t)kSmallSide * square_ld(kSmallSide) * 4 * 8;
            any.apply_shared = (size_t)kSmallSide * (square_ld(kSmallSide) + kApplyLd) * 8;
            any.resident_shared = kResidentMost;
            er = small_setup<float>(any);
            if (er == cudaSuccess) er = small_setup<__nv_bfloat16>(any);
            if (er == cudaSuccess) er = small_setup<__half>(any);
        }
        if (!all.empty() && !small.empty()) {
            if (er == cudaSuccess) er = cudaStreamCreateWithFlags(&h->side, cudaStreamNonBlocking);
            if (er == cudaSuccess) er = cudaEventCreateWithFlags(&h->fork, cudaEventDisableTiming);
            if (er == cudaSuccess) er = cudaEventCreateWithFlags(&h->join, cudaEventDisableTiming);
        }
        unsigned *err_dev = nullptr;
        if (er == cudaSuccess) er = cser_internal_take_word(&h->err_host, &err_dev);
        if (er != cudaSuccess) {
            orth_fail(h, er == cudaErrorMemoryAllocation ? CSER_ERR_NOMEM : CSER_ERR_CUDA, cudaGetErrorString(er));
            return nullptr;
        }
        h->groups.resize(parts.size());
        for (size_t g = 0; g < parts.size(); ++g) {
            cser_orth::Group &G = h->groups[g];
            if (build_group(h, G, parts[g], mode, steps, fit_ctas[mode]) != CSER_OK) {
                cser_orth_destroy(h);
                return nullptr;
            }
            G.args.err = err_dev;
        }
        return h;
    } catch (const std::bad_alloc &) {
        if (h) cser_orth_destroy(h);
        cser_internal_fail(CSER_ERR_NOMEM, "cser_orth_create: host allocation failed");
        return nullptr;
    }
}

int cser_orth_apply(cser_orth_handle h, const void *grad, float *m, float mu, void *out, void *stream) {
    if (!h) return cser_internal_fail(CSER_ERR_INVALID, "cser_orth_apply: NULL handle");
    int dev = -1;
    TRY(cudaGetDevice(&dev));
    if (dev != h->device)
        return cser_internal_fail(CSER_ERR_INVALID, "handle belongs to device %d, current device is %d", h->device, dev);
    if (*reinterpret_cast<volatile unsigned *>(h->err_host))
        return cser_internal_fail(CSER_ERR_CUDA, "a device-side wait ran out in an earlier cser_orth_apply: its results are incomplete, "
                                                 "make a new plan");
    if (int rc = cser_internal_check_ptr(grad, "cser_orth_apply: grad")) return rc;
    if (int rc = cser_internal_check_ptr(out, "cser_orth_apply: out")) return rc;
    if (m)
        if (int rc = cser_internal_check_ptr(m, "cser_orth_apply: m")) return rc;
    if (m && !(mu >= 0.f && mu < 1.f)) return cser_internal_fail(CSER_ERR_INVALID, "cser_orth_apply: mu must be in [0, 1)");
    if ((uintptr_t)grad % type_size(h->in_type) || (uintptr_t)out % type_size(h->out_type) || (uintptr_t)m % 4)
        return cser_internal_fail(CSER_ERR_INVALID, "cser_orth_apply: a pointer is not aligned to its element type");
    if (grad == out && h->in_type != h->out_type)
        return cser_internal_fail(CSER_ERR_INVALID, "cser_orth_apply: out may be grad only where the types are the same");
    // From the first matrix's beginning to the last one's end.
    auto apart = [&](const void *x, int size_x, const void *y, int size_y) {
        const uintptr_t p = (uintptr_t)x, q = (uintptr_t)y;
        return p + h->last * size_x <= q + h->first * size_y || q + h->last * size_y <= p + h->first * size_x;
    };
    const int size_in = type_size(h->in_type), size_out = type_size(h->out_type);
    if (grad != out && !apart(grad, size_in, out, size_out))
        return cser_internal_fail(CSER_ERR_INVALID, "cser_orth_apply: out must be grad itself or apart from it");
    if (m && (!apart(m, 4, grad, size_in) || !apart(m, 4, out, size_out)))
        return cser_internal_fail(CSER_ERR_INVALID, "cser_orth_apply: m must be an array of its own");
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool both = !h->groups.empty() && (h->resident.tables || h->small.tables);
    cudaStream_t small_st = both ? h->side : st;
    for (cser_orth::Group &G : h->groups) {
        OrthArgs a = G.args;
        a.grad = grad, a.m = m, a.mu = mu, a.out = out;
        a.wait_cycles = h->stall_mcycles ? h->stall_mcycles * 1000000ll : kWaitCycles;
        a.stall = h->stall_mcycles ? 1u << 30 : 0;
        cudaError_t e = h->in_type == CSER_TYPE_F32    ? prologue_launch<float>(G, a, st)
                        : h->in_type == CSER_TYPE_BF16 ? prologue_launch<__nv_bfloat16>(G, a, st)
                                                       : prologue_launch<__half>(G, a, st);
        TRY(e);
        // The small matrices' kernels follow the last group's products in time, onto the SMs that those leave: the other way round the
        // products, whose CTAs start together or not at all, waited for them.
        const bool fork = both && &G == &h->groups.back();
        if (fork) TRY(cudaEventRecord(h->fork, st));
        if (G.mode == kNarrow) e = h->split ? products_launch<kNarrow, true>(a, G.shares, G.grid, st) : products_launch<kNarrow, false>(a, G.shares, G.grid, st);
        else if (G.mode == kSingle) e = h->split ? products_launch<kSingle, true>(a, G.shares, G.grid, st) : products_launch<kSingle, false>(a, G.shares, G.grid, st);
        else e = h->split ? products_launch<kPaired, true>(a, G.shares, G.grid, st) : products_launch<kPaired, false>(a, G.shares, G.grid, st);
        TRY(e);
        h->launches += 3;
    }
    if (both) TRY(cudaStreamWaitEvent(small_st, h->fork, 0));
    for (const cser_orth::Small *S : {&h->resident, &h->small}) {
        if (!S->tables) continue;
        SmallArgs a = S->args;
        a.grad = grad, a.m = m, a.mu = mu, a.out = out;
        const cudaError_t e = h->in_type == CSER_TYPE_F32    ? small_launch<float>(*S, a, small_st)
                              : h->in_type == CSER_TYPE_BF16 ? small_launch<__nv_bfloat16>(*S, a, small_st)
                                                             : small_launch<__half>(*S, a, small_st);
        TRY(e);
        h->launches += S->n_resident ? 1 : 2;
    }
    h->stall_mcycles = 0;
    if (both) {
        TRY(cudaEventRecord(h->join, small_st));
        TRY(cudaStreamWaitEvent(st, h->join, 0));
    }
    return CSER_OK;
}

void cser_orth_destroy(cser_orth_handle h) {
    if (!h) return;
    if (h->side) cudaStreamSynchronize(h->side), cudaStreamDestroy(h->side);
    if (h->fork) cudaEventDestroy(h->fork);
    if (h->join) cudaEventDestroy(h->join);
    for (cser_orth::Group &G : h->groups)
        if (G.tables) cudaFree(G.tables);
    if (h->small.tables) cudaFree(h->small.tables);
    if (h->resident.tables) cudaFree(h->resident.tables);
    if (h->work) cudaFree(h->work);
    if (h->err_host) cser_internal_give_word(h->err_host);
    delete h;
}

int cser_orth_debug_stall_next(cser_orth_handle h, unsigned wait_mcycles) {
    if (!h) return cser_internal_fail(CSER_ERR_INVALID, "cser_orth_debug_stall_next: NULL handle");
    if (wait_mcycles < 1 || wait_mcycles > 2000)
        return cser_internal_fail(CSER_ERR_INVALID, "cser_orth_debug_stall_next: wait_mcycles must be in 1..2000");
    if (h->groups.empty()) return cser_internal_fail(CSER_ERR_INVALID, "cser_orth_debug_stall_next: the plan has no kernel that waits");
    h->stall_mcycles = wait_mcycles;
    return CSER_OK;
}

int64_t cser_orth_launch_count(cser_orth_handle h) { return h ? h->launches : 0; }

}  // extern "C"
