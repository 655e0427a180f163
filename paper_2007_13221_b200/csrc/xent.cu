// Softmax cross entropy of a linear head over a large vocabulary and its gradient (cser_xent_* of include/cser_train.h).
//
//   z = h W^T,  lse = log sum exp z,  loss = lse - z[target];    dz = (exp(z - lse) - [target]) dloss,  dh = dz W,  dW = dz^T h
//
// The logits are never kept.  cser_xent_loss: one kernel of 128 x 256 tiles of z whose epilogue reduces its tile to a
// maximum and a sum of exponentials per row and quarter tile, and one that joins them.  cser_xent_grad: for each piece of
// the vocabulary a kernel computes the tiles of z again and leaves dz in 16 bits, as panels (tensor_tiles.cuh), and
// one kernel makes from them the piece's rows of dW (inner dimension: tokens) and the piece's share of dh (inner dimension: the piece).
// The products that need dz, h or W the other way round take the same tiles with the other majorness.  Operands are read where they lie, but for
// rows that no tensor copy can start at (not 16 bytes apart, or at another address), which each call packs first.
//
// Bound.  6 T V D multiply-adds' flops (8 with z computed again) against 2 V D elements of W and dW moved: the tensor cores for
// T above about 500, the read of W (and the write of dW) below.
//
// Rounding.  dz is rounded to the operands' type, 8 (bf16) or 11 (fp16) bits, as any product on these inputs has to.
// It is held relative to the worker's largest |dloss| (times 2^12 for fp16, whose smallest normal number is above 1 / V for a
// large vocabulary) and the factor is put back in fp32 at the end: for a mean over tokens dz is p - [target] itself, not p / T rounded.
// fp16's range ends 2^-37 below the largest |dloss| that way, and a token of little weight would have its row of dh made from what is left of
// it: p = 1e-5 under a weight of 2^-20 is nothing.  So where a worker's weights are more than 2^6 apart, dz is left a second time for dh, each row
// relative to its own |dloss| (dW's rows add tokens up, and there 2^-37 of the largest is little).
// That rounding and the result's are all there is: 1.9e-3 of a bf16 gradient in the 2-norm, where products of unrounded dz leave the result's
// own, 1.7e-3 (fp16 2.6e-4 and 2.1e-4).  Up to 32 tokens what it left is kept too, in rows that are padding otherwise: no more bytes, no more
// stages, and 1.7e-3.  Above, the same would take both gradients' products twice, half as much time again.
#include <cuda.h>
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <float.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <new>

#include "cser_train.h"
#include "train_host.h"

namespace {

#include "tensor_tiles.cuh"

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -FLT_MAX;                // a maximum of nothing: no finite logit is lower, and differences from it are not NaN
constexpr size_t kPieceBytes = 256ull << 20;
// The tensor cores truncate every partial sum: 1.2e-6 of a logit over an inner dimension of 1024 (2.5e-6 of a small loss), 3e-6
// over 4096.  So the loss's accumulators are taken out and added up, rounded, after this many stages: an inner dimension of 256
// for few tokens, where memory is the bound, of 512 for many (of 256 the epilogue cannot keep up: tensor cores 73 % busy
// instead of 85 % at 2048 tokens x 16384 x 4096).  The gradient's logits are summed in
// the same chunks, so that p is of the logits that lse is of: 1 - p = 8e-4 of a nearly certain token came out 3 % off without
// (4096 x 32768 x 4096, gradient 2.55 ms without, 2.62 with).
__host__ __device__ constexpr int loss_chunk(int cg) { return cg == 1 ? 4 : 8; }
constexpr int kOwnRatio = 256;                     // tokens of a worker up to which every warp finds the largest |dloss| itself
constexpr int kJoinRows = 20;                     // rows that the last CTA joins itself, a warp or more for each

// 2^x, flushing: the instruction.
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

struct WorkerScale {
    float unscale;
    int flags;
};
// dh is made from dz_rows; dW is made from h_clean.
enum { kByRow = 1, kCleaned = 2 };

struct XentArgs {
    CUtensorMap h, w;                              // (dim, row, worker), boxes of 64 x 64
    int n, tokens, vocab, dim;
    int h_workers, w_workers;                      // 1: one array for all workers
    int bf16;
    int token_tiles, piece0, piece_n;              // vocabulary entries of this launch
    int tp;                                        // rows of a dz panel
    // loss
    float2 *part;                                  // [parts][n * tokens] maximum and sum
    int parts;
    float *z_target;                               // [n * tokens]
    const int64_t *target;
    int64_t ignore;
    float *loss, *lse_out;
    unsigned *ticket;                              // of the CTAs of a loss whose last one joins the parts
    // gradient
    const float *lse, *dloss;
    float *ratio;                                  // [n * tokens] dloss relative to the largest, times the type's scale
    WorkerScale *scale;                            // [n] what takes that back
    float *row_unscale;                            // [n * tokens] the same for a row of dh
    char *dz;                                      // [n][piece / 64 panels][tp rows][128 bytes]
    char *dz_rows;                                 // the same with a factor for each row; fp16 only
    const uint16_t *h_at;                          // what the map `h` is of
    long long h_row, h_worker;
    uint16_t *h_clean;                             // [n][clean_rows][dim, rounded up to 8] see clean_rows()
    int clean_rows;
    const CUtensorMap *h_clean_map;                // in the workspace: arguments of a launch take time on the host
    size_t dz_worker;
    float *acc;                                    // [n][splits][acc_rows][acc_cols] dh of the pieces so far
    int acc_rows, acc_cols, first_piece, last_piece;
    int splits, shares;                            // of dh's inner dimension: kept in acc; of this piece, 1 .. splits, each of a stage at least
    void *dh, *dw;
    long long dw_stride;
    CUtensorMap dh_map, dw_map;                    // of the results, boxes of 64 x 32, where
    int dh_boxes, dw_boxes;                        // these say that their address and rows allow it
    unsigned *err;
};

// ------------------------------------------------------------------ dloss, relative to the largest
// How far apart the weights of a worker's tokens are beyond which dh's rows have factors of their own: up to there every p above 1e-6
// keeps all of fp16's bits.  Gradients with and without, fp16: 8 x 512 x 30522 x 1024 750 to 860 us and 680, 8 x 16 394 and 371, 4096 x 32768 x
// 4096 2.8 ms and 2.6.
constexpr float kApart = 64.f;
__device__ __forceinline__ float type_scale(const XentArgs &a) { return a.bf16 ? 1.f : 4096.f; }
// The largest and the smallest finite |dloss| but 0 of a worker's tokens that count.  (One that is not finite spoils its own row
// of dh, not all.)  And whether a token that does not count, or whose dloss is 0, has a hidden state that is not finite: no logit, and so no
// lse, is finite then.
struct Weights {
    float top, low;
    int dirty;
    // By `n` threads of which this is `k`; not yet joined between warps.
    __device__ __forceinline__ Weights(const XentArgs &a, int worker, int k, int n) : top(0.f), low(INFINITY), dirty(0) {
        const size_t base = (size_t)worker * a.tokens;
        for (int t = k; t < a.tokens; t += n) {
            const float d = fabsf(a.dloss[base + t]), lse = a.lse[base + t];
            const bool counts = a.target[base + t] != a.ignore && d != 0.f;
            if (counts && isfinite(d)) top = fmaxf(top, d), low = fminf(low, d);
            dirty |= !counts && !isfinite(lse);
        }
        join();
    }
    __device__ __forceinline__ void join() {
#pragma unroll
        for (int m = 16; m; m >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, m)), low = fminf(low, __shfl_xor_sync(~0u, low, m));
        dirty = __any_sync(~0u, dirty);
    }
    __device__ __forceinline__ WorkerScale scale(const XentArgs &a) const {
        return {top / type_scale(a), (!a.bf16 && low * kApart < top ? kByRow : 0) | (dirty ? kCleaned : 0)};
    }
};
// 32 rows of hidden states by a warp, as dW takes them where a worker has such tokens: theirs as zeros (dz is 0 there, but 0 x NaN is
// not), and zeros up to the products' 64.
__device__ __forceinline__ void clean_rows(const XentArgs &a, int worker, int row0, int lane) {
    const size_t at = (size_t)worker * a.tokens + row0 + lane;
    const bool zero = row0 + lane >= a.tokens || ((a.target[at] == a.ignore || a.dloss[at] == 0.f) && !isfinite(a.lse[at]));
    const unsigned zeros = __ballot_sync(~0u, zero);
    const int padded = (a.dim + 7) / 8 * 8;
#pragma unroll 1
    for (int r = 0; r < 32; ++r) {
        const uint16_t *from = a.h_at + worker * a.h_worker + (row0 + r) * a.h_row;
        uint16_t *to = a.h_clean + ((size_t)worker * a.clean_rows + row0 + r) * padded;
#pragma unroll 1
        for (int c = lane; c < padded; c += 32) to[c] = zeros >> r & 1 || c >= a.dim ? (uint16_t)0 : from[c];
    }
}
// A row's factor of dz relative to the largest dloss, and what takes its factor of dh back.
__device__ __forceinline__ float row_ratio(const XentArgs &a, size_t at, float top, const WorkerScale &of, float &unscale) {
    const int64_t y = a.target[at];
    unscale = of.unscale;
    if (y == a.ignore) return 0.f;
    if (y < 0 || y >= a.vocab) return NAN;
    const float d = a.dloss[at];
    if (d == 0.f) return 0.f;
    if (!isfinite(d)) return NAN;
    if (of.flags & kByRow) unscale = fabsf(d) / type_scale(a);
    return d / top * type_scale(a);
}
// One CTA per worker.
__global__ void __launch_bounds__(1024) xent_ratio_kernel(const __grid_constant__ XentArgs a) {
    __shared__ float red[2][32];
    let_next_start();
    earlier_done();
    Weights w(a, blockIdx.x, threadIdx.x, 1024);
    if (threadIdx.x % 32 == 0) red[0][threadIdx.x / 32] = w.top, red[1][threadIdx.x / 32] = w.low;
    __syncthreads();
    w.top = red[0][threadIdx.x % 32], w.low = red[1][threadIdx.x % 32];
    w.join();
    w.dirty = __syncthreads_or(w.dirty);
    const WorkerScale of = w.scale(a);
    if (threadIdx.x == 0) a.scale[blockIdx.x] = of;
    const size_t base = (size_t)blockIdx.x * a.tokens;
    for (int t = threadIdx.x; t < a.tokens; t += 1024) {
        float unscale;
        a.ratio[base + t] = row_ratio(a, base + t, w.top, of, unscale), a.row_unscale[base + t] = unscale;
    }
}

// Boxes of 64 rows that a CTA's 128 tokens take, `left` of which there are: what the second one's place holds instead reaches
// only rows of results that nobody reads (loss and gradients of 8 workers x 16 tokens x 30522 x 1024: 472 us with
// both, 445 with one; loss of one token 26.2, 23.9).
__device__ __forceinline__ int row_boxes(int left) { return left > 64 ? 2 : 1; }
constexpr int kLowRows = 32;                       // tokens of a worker up to which dz keeps what its rounding left
// What 8 values have beyond their 16-bit forms `o`, in 16 bits.
__device__ __forceinline__ uint4 remainder8(const float *v, const uint4 &o, int bf16) {
    const uint32_t w[4] = {o.x, o.y, o.z, o.w};
    uint32_t r[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (bf16) {
            const float2 b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&w[k]));
            r[k] = pack_bf162(v[2 * k] - b.x, v[2 * k + 1] - b.y);
        } else {
            const float2 b = __half22float2(*reinterpret_cast<const __half2 *>(&w[k]));
            r[k] = pack_half2(v[2 * k] - b.x, v[2 * k + 1] - b.y);
        }
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

// ------------------------------------------------------------------ logits, tile by tile
// What the tiles of z are for: a loss, or dz; over a long inner dimension in chunks, the same ones for both: a loss near 0 is
// the difference of lse and z, and so is p - 1.
enum { kLoss = 0, kLongLoss = 1, kGrad = 2, kLongGrad = 3 };
template <int CG, int WHAT>
struct LogitsJob {
    static constexpr bool GRAD = WHAT >= kGrad, LONG = WHAT == kLongLoss || WHAT == kLongGrad;
    const XentArgs &a;
    int first, every, vocab_tiles;
    static constexpr bool kCopier = false, kRemainders = false, kWaits = false;

    struct Tile {
        int w, i, j, n, stages, a_lim, b_lim;
    };
    __device__ __forceinline__ void tile(Tile &t, int k, int) const {
        const int at = first + k * every, per = a.token_tiles * vocab_tiles;
        t.w = at / per, t.n = 0;
        if (t.w >= a.n) return;
        const int r = at - t.w * per;
        t.j = r / a.token_tiles, t.i = r - t.j * a.token_tiles;
        t.n = 256, t.stages = (a.dim + 63) / 64, t.a_lim = t.b_lim = t.stages;
    }
    __device__ __forceinline__ bool ready(Pipe<CG> &, const Tile &) const { return true; }
    __device__ __forceinline__ bool chunk_ends(const Tile &t, int k) const {
        return k + 1 == t.stages || (LONG && (k + 1) % loss_chunk(CG) == 0);
    }
    __device__ __forceinline__ int bf16() const { return a.bf16; }
    struct Loader {
        const CUtensorMap *h, *w;
        int row_a, row_b, wa, wb, boxes;
        __device__ __forceinline__ Loader(const LogitsJob &job, const Tile &t, int rank = CG == 1 ? 0 : (int)cluster_rank())
            : h(&job.a.h), w(&job.a.w), row_a(t.i * 128 * CG + rank * 128), row_b(job.a.piece0 + t.j * 256 + rank * 128),
              wa(job.a.h_workers == 1 ? 0 : t.w), wb(job.a.w_workers == 1 ? 0 : t.w), boxes(row_boxes(job.a.tokens - row_a)) {}
        __device__ __forceinline__ void settle(const LogitsJob &, const Tile &) const {}
        __device__ __forceinline__ uint32_t bytes() const { return Pipe<CG>::kStageBytes - 16384 + (uint32_t)boxes * 8192; }
        __device__ __forceinline__ void load(int k, uint32_t sa, uint32_t sb, uint64_t *bar) const {
#pragma unroll
            for (int p = 0; p < 2; ++p)
                if (p < boxes) tensor_copy_in(sa + p * 8192, h, k * 64, row_a + p * 64, wa, bar);
#pragma unroll
            for (int p = 0; p < 4 / CG; ++p) tensor_copy_in(sb + p * 8192, w, k * 64, row_b + p * 64, wb, bar);
        }
    };
    // The accumulator's turn, or all chunks added up, rounded: the warp's 64 columns.
    template <int N>
    __device__ __forceinline__ bool sums(Pipe<CG> &p, typename Pipe<CG>::Turn &turn, int chunks, int c0, int lane, float (&v)[N][32]) const {
        uint32_t tmem;
        for (int c = 0; c < chunks; ++c) {
            if (!p.take(turn, tmem)) return false;
            if (!LONG) break;
            if (c == 0) {
#pragma unroll
                for (int b = 0; b < N; ++b) tmem_load(tmem + c0 + b * 32, v[b]);
            } else
#pragma unroll
            for (int b = 0; b < 2 * N; ++b) {
                float x[16];
                tmem_load(tmem + c0 + b * 16, x);
#pragma unroll
                for (int k = 0; k < 16; ++k) v[b / 2][b % 2 * 16 + k] = __fadd_rn(v[b / 2][b % 2 * 16 + k], x[k]);
            }
            p.release(turn, lane);
        }
        return true;
    }
    // 32 columns of a row, of which `left` are not 0, times `factor` into the panels at `base`; `in`: the first one's place in the piece.
    __device__ __forceinline__ void leave(float (&x)[32], float factor, int left, char *base, int worker, int in, int row, bool lows) const {
#pragma unroll
        for (int k = 0; k < 32; ++k) x[k] *= factor;
        if (left < 32) {
#pragma unroll
            for (int k = 0; k < 32; ++k)
                if (k >= left) x[k] = 0.f;
        }
        char *dz = base + (size_t)worker * a.dz_worker + (size_t)(in / 64) * a.tp * 128;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float *e = x + 8 * k;
            uint4 o;
            if (a.bf16)
                o = make_uint4(pack_bf162(e[0], e[1]), pack_bf162(e[2], e[3]), pack_bf162(e[4], e[5]), pack_bf162(e[6], e[7]));
            else
                o = make_uint4(pack_half2(e[0], e[1]), pack_half2(e[2], e[3]), pack_half2(e[4], e[5]), pack_half2(e[6], e[7]));
            char *to = dz + panel_chunk(row, in % 64 / 8 + k);
            *reinterpret_cast<uint4 *>(to) = o;
            if (lows) *reinterpret_cast<uint4 *>(to + 32 * 128) = remainder8(e, o, a.bf16);
        }
    }
    __device__ __forceinline__ bool epilogue(Pipe<CG> &p, const Tile &t, typename Pipe<CG>::Turn &turn, int warp, int lane) const {
        const int row = t.i * 128 * CG + (int)p.rank * 128 + warp % 4 * 32 + lane;
        const int c0 = warp / 4 * 64;
        const bool live = row < a.tokens, lows = CG == 1 && a.tokens <= kLowRows;
        // Rows of zeros up to a multiple of 64 are the inner dimension's padding in dW; warps whose rows are none of these have
        // nothing to do.
        const int chunks = LONG ? (t.stages + loss_chunk(CG) - 1) / loss_chunk(CG) : 1;
        if (row - lane >= (!GRAD ? a.tokens : lows ? 32 : (a.tokens + 63) / 64 * 64)) {
            uint32_t unused;
            for (int c = 0; c < chunks; ++c) {
                if (!p.take(turn, unused)) return false;
                p.release(turn, lane);
            }
            return true;
        }
        const size_t at = (size_t)t.w * a.tokens + row;
        int target = -1;
        if (live) {
            const int64_t y = a.target[at];
            if (y >= 0 && y < a.vocab && y != a.ignore) target = (int)y;
        }
        float v[LONG ? 2 : 1][32];                                   // all 64 columns, or 32 at a time
        if constexpr (!GRAD) {
            if (!sums(p, turn, chunks, c0, lane, v)) return false;
            float m = kLowest, s = 0.f;
#pragma unroll(LONG ? 2 : 1)
            for (int b = 0; b < 64; b += 32) {
                const int col = t.j * 256 + c0 + b;
                float(&z)[32] = v[LONG ? b / 32 : 0];
                if (!LONG) {
                    tmem_load(p.acc_at(turn) + c0 + b, z);
                    if (b == 32) p.release(turn, lane);
                }
                if (col + 32 > a.vocab) {
#pragma unroll
                    for (int k = 0; k < 32; ++k)
                        if (col + k >= a.vocab) z[k] = -INFINITY;
                }
                float top = m;
#pragma unroll
                for (int k = 0; k < 32; ++k) top = fmaxf(top, z[k]);
                float e[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < 32; ++k) e[k % 4] += exp2_fast((z[k] - top) * kLog2e);
                s = __fmaf_rn(s, exp2_fast((m - top) * kLog2e), (e[0] + e[1]) + (e[2] + e[3]));
                m = top;
                const unsigned off = (unsigned)(target - col);
                if (off < 32u) {
#pragma unroll
                    for (int k = 0; k < 32; ++k)
                        if (off == (unsigned)k) a.z_target[at] = z[k];
                }
            }
            if (live) a.part[(size_t)(t.j * 4 + warp / 4) * a.n * a.tokens + at] = make_float2(m, s);
        } else {
            float ratio = 0.f, lse = 0.f;
            int flags;
            if (a.tokens <= kOwnRatio) {                             // no kernel came before that worked the ratios out
                const Weights weights(a, t.w, lane, 32);
                const WorkerScale of = weights.scale(a);
                float unscale = 0.f;
                if (live) ratio = row_ratio(a, at, weights.top, of, unscale);
                if (t.j == 0 && warp < 4 && live) a.row_unscale[at] = unscale;
                if (warp == 0 && lane == 0) a.scale[t.w] = of;
                flags = of.flags;
            } else {
                if (live) ratio = a.ratio[at];
                flags = a.scale[t.w].flags;
            }
            if (flags & kCleaned && t.j == 0 && a.first_piece && warp < 4) clean_rows(a, t.w, row - lane, lane);
            if (live) lse = a.lse[at];
            if (!sums(p, turn, chunks, c0, lane, v)) return false;
#pragma unroll(LONG ? 2 : 1)
            for (int b = 0; b < 64; b += 32) {
                const int in = t.j * 256 + c0 + b, col = a.piece0 + in;
                float(&x)[32] = v[LONG ? b / 32 : 0];
                if (!LONG) {
                    tmem_load(p.acc_at(turn) + c0 + b, x);
                    if (b == 32) p.release(turn, lane);
                }
#pragma unroll
                for (int k = 0; k < 32; ++k) x[k] = exp2_fast((x[k] - lse) * kLog2e);   // the difference first: it is exact where p is near 1
                const unsigned off = (unsigned)(target - col);
                if (off < 32u) {
#pragma unroll
                    for (int k = 0; k < 32; ++k)
                        if (off == (unsigned)k) x[k] -= 1.f;
                }
                const int left = ratio == 0.f ? 0 : a.vocab - col;   // padding, and tokens that do not count, are 0 whatever x is
                leave(x, ratio, left, a.dz, t.w, in, row, lows);
                if (flags & kByRow) leave(x, ratio == 0.f ? 0.f : type_scale(a) / fabsf(ratio), left, a.dz_rows, t.w, in, row, lows);
            }
        }
        return true;
    }
};

// z[target] of a row, or what makes its loss 0 or NaN; asked for before its parts are joined.
struct RowTarget {
    int64_t y;
    float z;
    __device__ __forceinline__ RowTarget(const XentArgs &a, size_t at, bool live) : y(live ? a.target[at] : 0), z(live ? __ldcg(a.z_target + at) : 0.f) {}
    // From the largest logit and the sum of exponentials relative to it; the logits' difference first: it is exact where the loss is small.
    __device__ __forceinline__ void loss(const XentArgs &a, size_t at, float m, float s) const {
        const float l = logf(s);
        a.lse_out[at] = m + l;
        if (a.loss) a.loss[at] = y == a.ignore ? 0.f : y >= 0 && y < a.vocab ? (m - z) + l : NAN;
    }
};

// The parts of 32 rows joined by 32 warps: a lane takes a row, a warp every 32nd part, four of them at a time.
__global__ void __launch_bounds__(1024) xent_join_kernel(const __grid_constant__ XentArgs a) {
    __shared__ float2 red[32][32];
    let_next_start();
    earlier_done();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const size_t rows = (size_t)a.n * a.tokens, at = (size_t)blockIdx.x * 32 + lane;
    const RowTarget of(a, at, warp == 0 && at < rows);
    float m = kLowest, s = 0.f;
    if (at < rows)
        for (int k = warp; k < a.parts; k += 128) {
            float2 q[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) q[e] = k + 32 * e < a.parts ? a.part[(k + 32 * e) * rows + at] : make_float2(kLowest, 0.f);
            const float top = fmaxf(fmaxf(m, fmaxf(q[0].x, q[1].x)), fmaxf(q[2].x, q[3].x));
            s *= exp2_fast((m - top) * kLog2e);
#pragma unroll
            for (int e = 0; e < 4; ++e) s += q[e].y * exp2_fast((q[e].x - top) * kLog2e);
            m = top;
        }
    red[warp][lane] = make_float2(m, s);
    __syncthreads();
    if (warp == 0 && at < rows) {
        for (int k = 1; k < 32; ++k) {
            const float2 q = red[k][lane];
            const float top = fmaxf(m, q.x);
            s = s * exp2_fast((m - top) * kLog2e) + q.y * exp2_fast((q.x - top) * kLog2e);
            m = top;
        }
        of.loss(a, at, m, s);
    }
}

template <int CG, int WHAT>
__global__ void __launch_bounds__(kThreads, 1) xent_logits_kernel(const __grid_constant__ XentArgs a) {
    extern __shared__ unsigned char raw[];
    let_next_start();
    if (threadIdx.x == 0) prefetch_tensor_map(&a.h), prefetch_tensor_map(&a.w);
    Pipe<CG> p;
    p.template setup<LogitsJob<CG, WHAT>>(raw, a.err);
    LogitsJob<CG, WHAT> job{a, (int)blockIdx.x / CG, (int)gridDim.x / CG, (a.piece_n + 255) / 256};
    p.run(job);
    p.teardown();
    if constexpr (WHAT < kGrad) {
        // Few rows: the last CTA to finish joins their parts (a kernel of its own: 5 us after 14).
        if (a.n * a.tokens > kJoinRows) return;
        __shared__ bool last;
        if (threadIdx.x == 0) {                                      // after the CTA's barrier in teardown()
            unsigned before;
            asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(before) : "l"(a.ticket) : "memory");
            last = before == gridDim.x - 1;
            if (last) *a.ticket = 0;                                 // for the next call
        }
        __syncthreads();
        if (!last) return;
        // A warp for each 256 parts of a row: what more of them would save, their joining costs.
        const int rows = a.n * a.tokens, most = kThreads / 32 / rows, share = min(most, (a.parts + 255) / 256);
        const int warp = threadIdx.x / 32, row = warp / share, lane = threadIdx.x % 32;
        const RowTarget of(a, threadIdx.x, threadIdx.x < rows);
        __shared__ float2 red[kThreads / 32];
        float m = kLowest, s = 0.f;
        if (row < rows)
            for (int k = warp % share * 32 + lane; k < a.parts; k += 32 * share * 8) {   // 8 on their way at a time
                float2 q[8];
                float top = m;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int at = k + 32 * share * e;
                    q[e] = at < a.parts ? __ldcg(a.part + (size_t)at * rows + row) : make_float2(kLowest, 0.f);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) top = fmaxf(top, q[e].x);
                s *= exp2_fast((m - top) * kLog2e);
#pragma unroll
                for (int e = 0; e < 8; ++e) s += q[e].y * exp2_fast((q[e].x - top) * kLog2e);
                m = top;
            }
        for (int k = 16; k; k >>= 1) {
            const float qm = __shfl_xor_sync(~0u, m, k), qs = __shfl_xor_sync(~0u, s, k);
            const float top = fmaxf(m, qm);
            s = s * exp2_fast((m - top) * kLog2e) + qs * exp2_fast((qm - top) * kLog2e);
            m = top;
        }
        if (lane == 0) red[warp] = make_float2(m, s);
        __syncthreads();
        if (threadIdx.x < rows) {
            m = kLowest, s = 0.f;
            for (int k = 0; k < share; ++k) {
                const float2 q = red[threadIdx.x * share + k];
                const float top = fmaxf(m, q.x);
                s = s * exp2_fast((m - top) * kLog2e) + q.y * exp2_fast((q.x - top) * kLog2e);
                m = top;
            }
            of.loss(a, threadIdx.x, m, s);
        }
    }
}

// ------------------------------------------------------------------ dh and dW of a piece
// Results leave through 4 KB of shared memory per epilogue warp, 32 rows of up to 64 columns, so that a store instruction
// covers whole lines of four rows (or one row, where rows are not 16 bytes apart) and not 16 bytes of 32 rows.
template <int CG>
using GradPipe = Pipe<CG, 256, kEpiWarps * 4096>;

template <int CG>
struct GradJob {
    using P = GradPipe<CG>;
    const XentArgs &a;
    int first, every, n_dh, n_dw, dim_tiles, vocab_tiles, early;
    int known = -1, flags = 0;                     // of the worker of the copying thread's last tile
    static constexpr bool kCopier = false, kRemainders = CG == 1, kWaits = false;
    __device__ __forceinline__ bool remainders() const { return a.tokens <= kLowRows; }

    struct Tile {
        int w, i, j, n, stages, a_lim, b_lim, k0, split, dw;
    };
    // dh's tiles are long (the piece), dW's short (the tokens).  All of dh's come first, dealt out in turn; the CTAs that got one
    // less than the others take `early` tiles of dW in its place, the rest of dW is dealt out in turn again.
    __device__ __forceinline__ void tile(Tile &t, int k, int) const {
        const int extra = n_dh % every, mine = n_dh / every + (first < extra);
        int at;
        t.n = 0, t.dw = k >= mine;
        if (!t.dw) {
            at = k * every + first;
        } else {
            int rest = k - mine, begin = 0;
            if (extra) {
                begin = early * (every - extra);
                if (first >= extra) {
                    if (rest < early) begin = -1;
                    else rest -= early;
                }
            }
            at = begin < 0 ? rest * (every - extra) + first - extra : begin + rest * every + first;
            if (at >= n_dw) return;
        }
        t.j = at % dim_tiles, at /= dim_tiles;
        const int width = (a.dim + 64 * CG - 1) / (64 * CG) * (64 * CG);
        t.n = width - t.j * 256 < 256 ? width - t.j * 256 : 256;
        if (t.dw) {
            t.i = at % vocab_tiles, t.w = at / vocab_tiles;
            t.k0 = 0, t.stages = (a.tokens + 63) / 64, t.split = 0, t.a_lim = 0;
        } else {
            t.split = at % a.shares, at /= a.shares;
            t.i = at % a.token_tiles, t.w = at / a.token_tiles;
            const int all = (a.piece_n + 63) / 64;
            t.k0 = (int)((long long)all * t.split / a.shares);
            t.stages = (int)((long long)all * (t.split + 1) / a.shares) - t.k0, t.a_lim = t.stages;
        }
        t.b_lim = 0;
    }
    __device__ __forceinline__ bool ready(P &, const Tile &) const { return true; }
    __device__ __forceinline__ bool chunk_ends(const Tile &t, int k) const { return k + 1 == t.stages; }
    __device__ __forceinline__ int bf16() const { return a.bf16; }
    struct Loader {
        const CUtensorMap *b;
        const char *dz;
        size_t panel;
        int dw, col, row0, worker, boxes, rows;
        __device__ __forceinline__ Loader(const GradJob &job, const Tile &t) {
            const int rank = CG == 1 ? 0 : (int)cluster_rank();
            const XentArgs &a = job.a;
            const int row = t.i * 128 * CG + rank * 128;
            dw = t.dw, panel = (size_t)a.tp * 128, b = dw ? &a.h : &a.w, boxes = t.n / CG / 64;
            dz = a.dz + (size_t)t.w * a.dz_worker + (dw ? (size_t)(row / 64) * panel : (size_t)t.k0 * panel + (size_t)row * 128);
            col = t.j * 256 + rank * (t.n / CG), row0 = dw ? 0 : a.piece0 + t.k0 * 64;
            worker = (dw ? a.h_workers : a.w_workers) == 1 ? 0 : t.w, rows = dw ? 2 : row_boxes(a.tokens - row);
        }
        __device__ __forceinline__ void settle(GradJob &job, const Tile &t) {
            if (job.known != t.w) job.known = t.w, job.flags = __ldcg(&job.a.scale[t.w].flags);
            if (!dw && job.flags & kByRow) dz += job.a.dz_rows - job.a.dz;
            if (dw && job.flags & kCleaned) b = job.a.h_clean_map, worker = t.w;
        }
        __device__ __forceinline__ uint32_t bytes() const { return (uint32_t)(rows + boxes) * 8192; }
        __device__ __forceinline__ void load(int k, uint32_t sa, uint32_t sb, uint64_t *bar) const {
            if (dw) {
                bulk_copy_in(sa, dz + (size_t)k * 8192, 8192, bar);
                bulk_copy_in(sa + 8192, dz + panel + (size_t)k * 8192, 8192, bar);
            } else {
                bulk_copy_in(sa, dz + (size_t)k * panel, (uint32_t)rows * 8192, bar);
            }
#pragma unroll
            for (int p = 0; p < 4 / CG; ++p)
                if (p < boxes) tensor_copy_in(sb + p * 8192, b, col + p * 64, row0 + k * 64, worker, bar);
        }
    };
    // N columns of a row: dh's share of a piece is added to the earlier ones', what is complete goes, in 16 bits, into the warp's
    // 4 KB of shared memory, a panel of 32 rows.
    template <int N>
    __device__ __forceinline__ void columns(const Tile &t, float (&v)[N], int row, int col, bool live, bool leaves, float f, uint32_t at,
                                            int lane, int chunk) const {
        if (!t.dw && (!a.first_piece || !leaves)) {
            float4 *acc = reinterpret_cast<float4 *>(a.acc + (((size_t)t.w * a.splits + t.split) * a.acc_rows + row) * a.acc_cols + col);
            if (!a.first_piece && live) {
#pragma unroll
                for (int k = 0; k < N / 4; ++k) {
                    const float4 q = acc[k];
                    v[4 * k] += q.x, v[4 * k + 1] += q.y, v[4 * k + 2] += q.z, v[4 * k + 3] += q.w;
                }
            }
            if (!leaves) {
#pragma unroll
                for (int k = 0; k < N / 4; ++k)
                    if (live) acc[k] = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
                return;
            }
        }
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] *= f;
#pragma unroll
        for (int k = 0; k < N / 8; ++k) {
            const float *e = v + 8 * k;
            shared_store16(at + panel_chunk(lane, chunk + k),
                           a.bf16 ? make_uint4(pack_bf162(e[0], e[1]), pack_bf162(e[2], e[3]), pack_bf162(e[4], e[5]), pack_bf162(e[6], e[7]))
                                  : make_uint4(pack_half2(e[0], e[1]), pack_half2(e[2], e[3]), pack_half2(e[4], e[5]), pack_half2(e[6], e[7])));
        }
    }
    __device__ __forceinline__ bool epilogue(P &p, const Tile &t, typename P::Turn &turn, int warp, int lane) const {
        uint32_t tmem;
        const int row0 = t.i * 128 * CG + (int)p.rank * 128 + warp % 4 * 32, row = row0 + lane;
        const int quarter = t.n / 4, c0 = warp / 4 * quarter, col0 = t.j * 256 + c0;
        const bool leaves = t.dw || (a.last_piece && a.splits == 1);
        const uint32_t at = p.extra + (uint32_t)warp * 4096;
        const int rows = (t.dw ? a.piece_n : a.tokens) - row0;
        const float f = t.dw ? a.scale[t.w].unscale : lane < rows ? a.row_unscale[(size_t)t.w * a.tokens + row] : 0.f;
        if (!p.take(turn, tmem)) return false;
        if (rows <= 0) {
            p.release(turn, lane);
            return true;
        }
        if (CG == 1) {
            if (lane == 0) bulk_out_read<0>();                       // the last tile's rows have left the buffer
            __syncwarp();
        }
        if (CG == 1 && quarter == 64) {
#pragma unroll 1
            for (int b = 0; b < 64; b += 32) {
                float v[32];
                tmem_load(tmem + c0 + b, v);
                if (b == 32) p.release(turn, lane);
                columns(t, v, row, col0 + b, lane < rows, leaves, f, at, lane, b / 8);
            }
        } else {
#pragma unroll 1
            for (int b = 0; b < quarter; b += 16) {
                float v[16];
                tmem_load(tmem + c0 + b, v);
                if (b + 16 >= quarter) p.release(turn, lane);
                columns(t, v, row, col0 + b, lane < rows, leaves, f, at, lane, b / 8);
            }
        }
        if (!leaves) return true;
        // Tiles of dW by single CTAs are one or two stages long, and this is their bound: rows sent off by the copy engine, and 32 columns
        // at a time, 8 x 16 tokens x 30522 x 1024, gradients 327 -> 293 us.  By pairs, where a tile's products take
        // longer, it made no difference (8 x 512 tokens 735 us either way), and what follows needs no maps.
        if (CG == 1 && quarter == 64 && (t.dw ? a.dw_boxes : a.dh_boxes)) {
            fence_async_shared();
            __syncwarp();
            if (lane == 0) {
                tensor_copy_out(t.dw ? &a.dw_map : &a.dh_map, at, col0, t.dw ? a.piece0 + row0 : row0, t.w);
                bulk_out_commit();
            }
            return true;
        }
        __syncwarp();
        const int cols = a.dim - col0 < quarter ? a.dim - col0 : quarter;
        uint16_t *o = t.dw ? static_cast<uint16_t *>(a.dw) + t.w * a.dw_stride + (long long)(a.piece0 + row0) * a.dim + col0
                           : static_cast<uint16_t *>(a.dh) + ((long long)t.w * a.tokens + row0) * a.dim + col0;
        if (cols > 0 && (a.dim & 7) == 0 && (reinterpret_cast<uintptr_t>(o) & 15) == 0) {
            const int chunks = cols / 8;                             // whole ones: dim and quarter are multiples of 8
            for (int e = lane; e < 32 * chunks; e += 32) {
                const int r = e / chunks, c = e - r * chunks;
                if (r < rows) *reinterpret_cast<uint4 *>(o + (long long)r * a.dim + c * 8) = shared_load16(at + panel_chunk(r, c));
            }
        } else {
            for (int c = lane; c < cols; c += 32) {
#pragma unroll 8
                for (int r = 0; r < 32; ++r) {
                    uint16_t v;
                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at + panel_chunk(r, c / 8) + c % 8 * 2));
                    if (r < rows) o[(long long)r * a.dim + c] = v;
                }
            }
        }
        __syncwarp();
        return true;
    }
};

template <int CG>
__global__ void __launch_bounds__(kThreads, 1) xent_grad_kernel(const __grid_constant__ XentArgs a, int n_dh, int n_dw) {
    extern __shared__ unsigned char raw[];
    let_next_start();
    if (threadIdx.x == 0) prefetch_tensor_map(&a.h), prefetch_tensor_map(&a.w);
    GradPipe<CG> p;
    p.template setup<GradJob<CG>>(raw, a.err);
    const int width = (a.dim + 64 * CG - 1) / (64 * CG) * (64 * CG);
    GradJob<CG> job{a, (int)blockIdx.x / CG, (int)gridDim.x / CG, n_dh, n_dw, (width + 255) / 256,
                    (a.piece_n + 128 * CG - 1) / (128 * CG), 0};
    if (n_dh && n_dw) {
        // A tile of dh in tiles of dW, whose epilogue takes as long as 12 stages, and of which there may not be that many.
        const int stages = ((a.piece_n + 63) / 64 + a.shares - 1) / a.shares, less = job.every - n_dh % job.every;
        const int each = (a.tokens + 63) / 64, fits = n_dw / less;
        job.early = stages / (each < 12 ? 12 : each);
        if (job.early > fits) job.early = fits;
    }
    p.run(job);
    if (CG == 1) bulk_out_done();                  // of the threads that sent results off
    p.teardown();
}

// Where the inner dimension was split: the shares of dh added up, four columns a thread, by eight threads that take an eighth of the
// shares each (by one, the 148 shares of 1 token x 102595 x 40 took as long as the rest).
constexpr int kJoinWays = 8;
__global__ void __launch_bounds__(256) xent_join_dh_kernel(const __grid_constant__ XentArgs a) {
    __shared__ float4 red[kJoinWays][32];
    let_next_start();
    earlier_done();
    const int groups = (a.dim + 3) / 4, way = threadIdx.x / 32, lane = threadIdx.x % 32;
    const long long e = (long long)blockIdx.x * 32 + lane, row_at = e / groups;
    const int col = (int)(e - row_at * groups) * 4;
    const bool live = row_at < (long long)a.n * a.tokens;
    const int w = (int)(row_at / a.tokens), row = (int)(row_at - (long long)w * a.tokens);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (live) {
        const float4 *from = reinterpret_cast<const float4 *>(a.acc + ((size_t)w * a.splits * a.acc_rows + row) * a.acc_cols + col);
        const size_t next = (size_t)a.acc_rows * a.acc_cols / 4;
        const int end = a.splits * (way + 1) / kJoinWays;
#pragma unroll 4
        for (int s = a.splits * way / kJoinWays; s < end; ++s) {
            const float4 q = from[s * next];
            v.x += q.x, v.y += q.y, v.z += q.z, v.w += q.w;
        }
    }
    red[way][lane] = v;
    __syncthreads();
    if (way || !live) return;
    for (int k = 1; k < kJoinWays; ++k) {
        const float4 q = red[k][lane];
        v.x += q.x, v.y += q.y, v.z += q.z, v.w += q.w;
    }
    const float f = a.row_unscale[row_at];
    uint16_t *o = static_cast<uint16_t *>(a.dh) + row_at * a.dim + col;
    const uint32_t lo = a.bf16 ? pack_bf162(v.x * f, v.y * f) : pack_half2(v.x * f, v.y * f);
    const uint32_t hi = a.bf16 ? pack_bf162(v.z * f, v.w * f) : pack_half2(v.z * f, v.w * f);
    if (col + 4 <= a.dim && (reinterpret_cast<uintptr_t>(o) & 7) == 0) {
        *reinterpret_cast<uint2 *>(o) = make_uint2(lo, hi);
    } else {
        for (int k = 0; k < 4 && col + k < a.dim; ++k) o[k] = (uint16_t)((k < 2 ? lo : hi) >> (k % 2 * 16));
    }
}

// Rows that no tensor copy can start at, as rows padded to a multiple of 8; of up to two arrays.  8 columns a thread, `per` threads a
// row (a CTA per row took 200 us for 246016 rows of 37).
struct PackSource {
    const uint16_t *src;
    long long row_stride, worker_stride;
    int rows, all;                                 // of a worker, of all
    uint16_t *dst;
};
__global__ void __launch_bounds__(256) xent_pack_kernel(const PackSource x, const PackSource y, int dim, int padded, int per) {
    let_next_start();
    earlier_done();
    const unsigned slot = threadIdx.x / per;
    const int at = (int)(blockIdx.x * (256u / per) + slot), k = threadIdx.x - slot * per;
    if (slot >= 256u / per || at >= x.all + y.all) return;
    const bool second = at >= x.all;
    const PackSource &p = second ? y : x;
    const int row = at - (second ? x.all : 0), worker = row / p.rows;
    const uint16_t *s = p.src + worker * p.worker_stride + (row - worker * p.rows) * p.row_stride;
    uint16_t *d = p.dst + (long long)row * padded;
    for (int c = k * 8; c < padded; c += per * 8) {
        uint32_t v[4];
        if (c + 8 > dim) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = (c + 2 * e < dim ? (uint32_t)s[c + 2 * e] : 0u) | (c + 2 * e + 1 < dim ? (uint32_t)s[c + 2 * e + 1] << 16 : 0u);
        } else if ((reinterpret_cast<uintptr_t>(s) & 2) == 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = reinterpret_cast<const uint32_t *>(s + c)[e];
        } else {
            const uint32_t *between = reinterpret_cast<const uint32_t *>(s + c + 1);
            const uint32_t x = between[0], y = between[1], z = between[2];
            v[0] = (uint32_t)s[c] | x << 16, v[1] = x >> 16 | y << 16, v[2] = y >> 16 | z << 16, v[3] = z >> 16 | (uint32_t)s[c + 7] << 16;
        }
        *reinterpret_cast<uint4 *>(d + c) = make_uint4(v[0], v[1], v[2], v[3]);
    }
}

}  // namespace

// ------------------------------------------------------------------ host
typedef CUresult (*encode_fn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                              const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

struct cser_xent {
    int device = 0, n = 0, type = 0, sms = 0;
    long long max_tokens = 0, vocab = 0, dim = 0, piece = 0;
    int parts = 0, tp = 0, acc_cols = 0;
    void *work = nullptr;
    float2 *part = nullptr;
    float *z_target = nullptr, *ratio = nullptr, *row_unscale = nullptr, *acc = nullptr;
    WorkerScale *scale = nullptr;
    unsigned *ticket = nullptr;
    char *dz = nullptr, *dz_rows = nullptr;
    uint16_t *h_clean = nullptr;
    CUtensorMap *h_clean_map = nullptr;
    void *pack_h = nullptr, *pack_w = nullptr;     // made on the first call that needs them
    encode_fn encode = nullptr;
    unsigned *err_host = nullptr, *err_dev = nullptr;
    long long launches = 0;
};

namespace {

int splits_of(const cser_xent *h, long long tokens) {
    // Few tiles of dh and a long inner dimension: the vocabulary is split so that every SM has a share, each of 8 stages at least;
    // fewer than 24 are left whole: joining takes 3 us, as much as 8 stages (2 x 5 tokens x 3000 x 2000, gradients: 40 us by 16, 35 by 8;
    // 3 x 77 x 1003 x 201, 16 stages: 27 whole, 30 in two; 50 x 100 x 1200 x 256, 19 stages: 34 and 50; 8 x 100 x 1200 x 2048: 40 and 60).
    const long long tiles = h->n * (up(tokens, 128) / 128) * (up(h->dim, 256) / 256), stages = up(h->piece < h->vocab ? h->piece : h->vocab, 64) / 64;
    long long s = tiles >= h->sms ? 1 : h->sms / tiles;
    if (stages < 24) s = 1;
    else if (s > stages / 8) s = stages / 8;
    return s < 1 ? 1 : (int)s;
}

// Tiles of 256 tokens by a pair of CTAs, or of 128 by one.  Up to 128 tokens half of a pair's tile would be padding: loss of
// one token x 30522 x 1024 13.7 us by single CTAs, 20.5 by pairs.  Above, pairs bring half the bytes per product: 4096 x 131072 x
// 4096 2.63 ms against 2.82 (loss), 9.7 against 12.1 (gradient).
bool wide_tiles(long long tokens) { return tokens > 128; }

bool tensor_map(const cser_xent *h, CUtensorMap &m, const void *p, long long rows, long long row_stride, long long worker_stride,
                int workers, long long dim) {
    const cuuint64_t size[3] = {(cuuint64_t)dim, (cuuint64_t)rows, (cuuint64_t)workers};
    const cuuint64_t stride[2] = {(cuuint64_t)row_stride * 2, (cuuint64_t)(workers == 1 ? up(row_stride * rows, 8) : worker_stride) * 2};
    const cuuint32_t box[3] = {64, 64, 1}, step[3] = {1, 1, 1};
    return h->encode(&m, h->type == CSER_TYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
                     const_cast<void *>(p), size, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                     CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The map of an operand, of a packed copy (then `job` says of what, and the address and strides become its) where its rows cannot
// be read in place.
int operand(cser_xent *h, CUtensorMap &m, int &workers, const void *&p, long long rows, long long &row_stride, long long &worker_stride,
            void *&pack, long long pack_rows, PackSource &job, const char *what, cudaStream_t st) {
    workers = h->n == 1 || worker_stride == 0 ? 1 : h->n;
    if (rows == 1) row_stride = up(h->dim, 8);                      // no second row: its distance says nothing
    const bool direct = (uintptr_t)p % 16 == 0 && row_stride % 8 == 0 && row_stride > 0 && (workers == 1 || worker_stride % 8 == 0);
    if (!direct) {
        const long long padded = up(h->dim, 8);
        if (!pack) {
            cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
            TRY(cudaStreamIsCapturing(st, &cap));
            if (cap != cudaStreamCaptureStatusNone)
                return cser_internal_fail(CSER_ERR_INVALID, "%s needs a packing buffer: make the first such call outside a capture", what);
            TRY(cudaMalloc(&pack, (size_t)h->n * pack_rows * padded * 2));
        }
        job = {static_cast<const uint16_t *>(p), row_stride, worker_stride, (int)rows, (int)(workers * rows), static_cast<uint16_t *>(pack)};
        p = pack, row_stride = padded, worker_stride = padded * rows;
    }
    if (!tensor_map(h, m, p, rows, row_stride, worker_stride, workers, h->dim))
        return cser_internal_fail(CSER_ERR_INVALID, "%s: no tensor map for this address and these strides", what);
    return CSER_OK;
}

int prepare_call(cser_xent *h, const cser_xent_inputs *in, const char *what, XentArgs &a, cudaStream_t st) {
    if (!h) return cser_internal_fail(CSER_ERR_INVALID, "%s: NULL handle", what);
    if (!in) return cser_internal_fail(CSER_ERR_INVALID, "%s: NULL inputs", what);
    int dev = -1;
    TRY(cudaGetDevice(&dev));
    if (dev != h->device)
        return cser_internal_fail(CSER_ERR_INVALID, "handle belongs to device %d, current device is %d", h->device, dev);
    if (*reinterpret_cast<volatile unsigned *>(h->err_host))
        return cser_internal_fail(CSER_ERR_CUDA, "a device-side wait ran out in an earlier call: its results are incomplete");
    if (in->tokens < 0 || in->tokens > h->max_tokens)
        return cser_internal_fail(CSER_ERR_INVALID, "%s: tokens must be in 0..%lld", what, h->max_tokens);
    a = XentArgs{};
    a.n = h->n, a.tokens = (int)in->tokens, a.vocab = (int)h->vocab, a.dim = (int)h->dim;
    if (in->tokens == 0) return CSER_OK;
    if (in->hidden_row_stride < 0 || in->hidden_worker_stride < 0 || in->weight_row_stride < 0 || in->weight_worker_stride < 0)
        return cser_internal_fail(CSER_ERR_INVALID, "%s: strides must not be negative", what);
    if (int rc = cser_internal_check_ptr(in->hidden, "hidden")) return rc;
    if (int rc = cser_internal_check_ptr(in->weight, "weight")) return rc;
    if (int rc = cser_internal_check_ptr(in->target, "target")) return rc;
    if ((uintptr_t)in->hidden % 2 || (uintptr_t)in->weight % 2 || (uintptr_t)in->target % 8)
        return cser_internal_fail(CSER_ERR_INVALID, "%s: a pointer is not aligned to its element type", what);
    PackSource pack[2] = {};
    const void *hid = in->hidden, *wei = in->weight;
    long long h_row = in->hidden_row_stride, h_worker = in->hidden_worker_stride, w_row = in->weight_row_stride, w_worker = in->weight_worker_stride;
    if (int rc = operand(h, a.h, a.h_workers, hid, in->tokens, h_row, h_worker, h->pack_h, h->max_tokens, pack[0], "hidden", st)) return rc;
    if (int rc = operand(h, a.w, a.w_workers, wei, h->vocab, w_row, w_worker, h->pack_w, h->vocab, pack[1], "weight", st)) return rc;
    a.h_at = static_cast<const uint16_t *>(hid), a.h_row = h_row, a.h_worker = a.h_workers == 1 ? 0 : h_worker;
    a.h_clean = h->h_clean, a.h_clean_map = h->h_clean_map, a.clean_rows = (int)up(h->max_tokens, 64);
    if (pack[0].all + pack[1].all > 0) {
        const int chunks = (int)(up(h->dim, 8) / 8), per = chunks < 256 ? chunks : 256, rows = 256 / per;
        TRY(launch_kernel(xent_pack_kernel, (unsigned)(((long long)pack[0].all + pack[1].all + rows - 1) / rows), 256, 0, 1, true, st, pack[0],
                          pack[1], (int)h->dim, (int)up(h->dim, 8), per));
        h->launches++;
    }
    a.bf16 = h->type == CSER_TYPE_BF16;
    a.tp = h->tp, a.part = h->part, a.parts = h->parts, a.z_target = h->z_target, a.target = in->target, a.ignore = in->ignore_index;
    a.ratio = h->ratio, a.scale = h->scale, a.row_unscale = h->row_unscale, a.dz = h->dz, a.dz_rows = h->dz_rows, a.dz_worker = (size_t)(h->piece / 64) * h->tp * 128;
    a.ticket = h->ticket, a.acc = h->acc, a.acc_rows = (int)up(a.tokens, 256), a.acc_cols = h->acc_cols, a.err = h->err_dev;
    return CSER_OK;
}

template <int CG, typename K, typename... Args>
cudaError_t tiles_launch(cser_xent *h, K kernel, size_t shared, long long tiles, cudaStream_t st, Args... args) {
    const long long most = h->sms / CG;
    h->launches++;
    return launch_kernel(kernel, (unsigned)((tiles < most ? tiles : most) * CG), kThreads, shared, CG, true, st, args...);
}

template <int CG>
cudaError_t kernels_setup() {
    const int b = (int)Pipe<CG>::kSharedBytes;
    cudaError_t e = cudaFuncSetAttribute(xent_logits_kernel<CG, kLoss>, cudaFuncAttributeMaxDynamicSharedMemorySize, b);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(xent_logits_kernel<CG, kLongLoss>, cudaFuncAttributeMaxDynamicSharedMemorySize, b);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(xent_logits_kernel<CG, kGrad>, cudaFuncAttributeMaxDynamicSharedMemorySize, b);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(xent_logits_kernel<CG, kLongGrad>, cudaFuncAttributeMaxDynamicSharedMemorySize, b);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(xent_grad_kernel<CG>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)GradPipe<CG>::kSharedBytes);
    return e;
}

template <int CG>
int loss_launch(cser_xent *h, XentArgs &a, cudaStream_t st) {
    a.token_tiles = (int)(up(a.tokens, 128 * CG) / (128 * CG)), a.piece0 = 0, a.piece_n = a.vocab;
    const auto kernel = a.dim > loss_chunk(CG) * kStageK ? xent_logits_kernel<CG, kLongLoss> : xent_logits_kernel<CG, kLoss>;
    TRY((tiles_launch<CG>(h, kernel, Pipe<CG>::kSharedBytes, (long long)a.n * a.token_tiles * ((a.vocab + 255) / 256), st, a)));
    if ((long long)a.n * a.tokens > kJoinRows) {
        TRY(launch_kernel(xent_join_kernel, (unsigned)(((long long)a.n * a.tokens + 31) / 32), 1024, 0, 1, true, st, a));
        h->launches++;
    }
    return CSER_OK;
}

// The map of a result that lies dense for each worker; 0: its address or rows do not allow one.
int result_map(const cser_xent *h, CUtensorMap &m, void *p, long long rows, long long worker_stride) {
    if (!p || (uintptr_t)p % 16 || h->dim % 8 || (h->n > 1 && worker_stride % 8)) return 0;
    const cuuint64_t size[3] = {(cuuint64_t)h->dim, (cuuint64_t)rows, (cuuint64_t)h->n};
    const cuuint64_t stride[2] = {(cuuint64_t)h->dim * 2, (cuuint64_t)(h->n > 1 ? worker_stride : rows * h->dim) * 2};
    const cuuint32_t box[3] = {64, 32, 1}, step[3] = {1, 1, 1};
    return h->encode(&m, h->type == CSER_TYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, p, size, stride,
                     box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int CG>
int grad_launch(cser_xent *h, XentArgs &a, cudaStream_t st) {
    a.token_tiles = (int)(up(a.tokens, 128 * CG) / (128 * CG));
    a.splits = splits_of(h, a.tokens);
    if (a.tokens > kOwnRatio) {
        TRY(launch_kernel(xent_ratio_kernel, (unsigned)a.n, 1024, 0, 1, true, st, a));
        h->launches++;
    }
    const long long dim_tiles = up(a.dim, 256) / 256;
    for (long long v = 0; v < h->vocab; v += h->piece) {
        a.piece0 = (int)v, a.piece_n = (int)(h->vocab - v < h->piece ? h->vocab - v : h->piece);
        a.first_piece = v == 0, a.last_piece = v + h->piece >= h->vocab;
        // The last piece can have fewer stages than there are shares: a tile without a stage would have no accumulator.  The
        // sums of the shares that it leaves out are complete with the pieces before.
        const int stages = (a.piece_n + 63) / 64;
        a.shares = a.splits < stages ? a.splits : stages;
        const long long vt = up(a.piece_n, 128 * CG) / (128 * CG);
        const auto kernel = a.dim > loss_chunk(CG) * kStageK ? xent_logits_kernel<CG, kLongGrad> : xent_logits_kernel<CG, kGrad>;
        TRY((tiles_launch<CG>(h, kernel, Pipe<CG>::kSharedBytes, (long long)a.n * a.token_tiles * ((a.piece_n + 255) / 256), st, a)));
        const long long n_dh = a.dh ? (long long)a.n * a.token_tiles * a.shares * dim_tiles : 0, n_dw = a.dw ? a.n * vt * dim_tiles : 0;
        TRY((tiles_launch<CG>(h, xent_grad_kernel<CG>, GradPipe<CG>::kSharedBytes, n_dh + n_dw, st, a, (int)n_dh, (int)n_dw)));
    }
    if (a.dh && a.splits > 1) {
        const long long e = (long long)a.n * a.tokens * ((a.dim + 3) / 4);
        TRY(launch_kernel(xent_join_dh_kernel, (unsigned)((e + 31) / 32), 256, 0, 1, true, st, a));
        h->launches++;
    }
    return CSER_OK;
}

}  // namespace

extern "C" {

cser_xent_handle cser_xent_create(int32_t n_workers, int64_t max_tokens, int64_t vocab, int64_t dim, int32_t type,
                                  int64_t piece) {
    auto bad = [](int code, const char *what) { cser_internal_fail(code, "cser_xent_create: %s", what); return nullptr; };
    if (n_workers < 1 || max_tokens < 1 || n_workers > (1 << 24) / max_tokens)
        return bad(CSER_ERR_INVALID, "n_workers and max_tokens must be positive and their product at most 2^24");
    if (vocab < 1 || vocab > (1 << 24) || dim < 1 || dim > 65536)
        return bad(CSER_ERR_INVALID, "vocab must be in 1..2^24, dim in 1..65536");
    if ((long long)n_workers * vocab > (1 << 30) || up(max_tokens, 128) / 128 * n_workers * (up(vocab, 256) / 256) > (1 << 30))
        return bad(CSER_ERR_INVALID, "n_workers * vocab, and the tiles of all logits, must be at most 2^30");
    if (type != CSER_TYPE_BF16 && type != CSER_TYPE_F16) return bad(CSER_ERR_INVALID, "type must be CSER_TYPE_BF16 or CSER_TYPE_F16");
    if (piece < 0) return bad(CSER_ERR_INVALID, "piece must not be negative");
    cser_xent *h = new (std::nothrow) cser_xent;
    if (!h) return bad(CSER_ERR_NOMEM, "host allocation failed");
    auto drop = [&](cudaError_t e) {
        cser_internal_fail(e == cudaErrorMemoryAllocation ? CSER_ERR_NOMEM : CSER_ERR_CUDA, "cser_xent_create: %s", cudaGetErrorString(e));
        cser_xent_destroy(h);
        return nullptr;
    };
    h->n = n_workers, h->max_tokens = max_tokens, h->vocab = vocab, h->dim = dim, h->type = type;
    cudaError_t e = cudaGetDevice(&h->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&h->sms, cudaDevAttrMultiProcessorCount, h->device);
    if (e == cudaSuccess) e = kernels_setup<1>();
    if (e == cudaSuccess) e = kernels_setup<2>();
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
    if (e == cudaSuccess) e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found);
    if (e == cudaSuccess && (!fn || found != cudaDriverEntryPointSuccess)) e = cudaErrorNotSupported;
    if (e != cudaSuccess) return drop(e);
    h->encode = reinterpret_cast<encode_fn>(fn);
    const long long rows = (long long)n_workers * max_tokens;
    h->tp = (int)up(max_tokens, 256), h->acc_cols = (int)up(dim, 128), h->parts = (int)(4 * (up(vocab, 256) / 256));
    const long long fit = (long long)(kPieceBytes / ((size_t)h->n * h->tp * 2)) / 256 * 256;
    h->piece = piece ? up(piece < vocab ? piece : vocab, 256) : fit < 2048 ? 2048 : fit;
    if (h->piece > up(vocab, 256)) h->piece = up(vocab, 256);
    long long acc_rows = 0;                        // the most that any number of tokens asks for
    for (long long t = 128; t < max_tokens + 128; t += 128) {
        const int k = splits_of(h, t < max_tokens ? t : max_tokens);
        if ((k > 1 || h->piece < vocab) && k * up(t, 256) > acc_rows) acc_rows = k * up(t, 256);
    }
    size_t at = 0;
    auto place = [&](size_t b) { const size_t p = at; at += (b + 1023) / 1024 * 1024; return p; };
    const size_t o_part = place((size_t)rows * h->parts * 8), o_zt = place((size_t)rows * 4), o_ratio = place((size_t)rows * 4),
                 o_un = place((size_t)n_workers * sizeof(WorkerScale)), o_run = place((size_t)rows * 4), o_tick = place(4),
                 o_dz = place((size_t)n_workers * (h->piece / 64) * h->tp * 128), dz_bytes = at - o_dz,
                 o_dzr = place(type == CSER_TYPE_F16 ? dz_bytes : 0),
                 o_map = place(sizeof(CUtensorMap)), o_clean = place((size_t)n_workers * up(max_tokens, 64) * up(dim, 8) * 2),
                 o_acc = place((size_t)n_workers * acc_rows * h->acc_cols * 4);
    e = cudaMalloc(&h->work, at);
    if (dim % 8) {                                 // dense rows of this length need packing
        if (e == cudaSuccess) e = cudaMalloc(&h->pack_h, (size_t)rows * up(dim, 8) * 2);
        if (e == cudaSuccess) e = cudaMalloc(&h->pack_w, (size_t)n_workers * vocab * up(dim, 8) * 2);
    }
    if (e == cudaSuccess) e = cser_internal_take_word(&h->err_host, &h->err_dev);
    if (e != cudaSuccess) return drop(e);
    char *w = static_cast<char *>(h->work);
    h->ticket = reinterpret_cast<unsigned *>(w + o_tick);
    e = cudaMemset(h->ticket, 0, 4);
    if (e != cudaSuccess) return drop(e);
    h->part = reinterpret_cast<float2 *>(w + o_part), h->z_target = reinterpret_cast<float *>(w + o_zt);
    h->ratio = reinterpret_cast<float *>(w + o_ratio), h->row_unscale = reinterpret_cast<float *>(w + o_run);
    h->scale = reinterpret_cast<WorkerScale *>(w + o_un);
    h->h_clean = reinterpret_cast<uint16_t *>(w + o_clean);
    h->h_clean_map = reinterpret_cast<CUtensorMap *>(w + o_map);
    CUtensorMap map;
    const bool made = tensor_map(h, map, h->h_clean, up(max_tokens, 64), up(dim, 8), up(max_tokens, 64) * up(dim, 8), n_workers, dim);
    e = made ? cudaMemcpy(h->h_clean_map, &map, sizeof(map), cudaMemcpyHostToDevice) : cudaErrorInvalidValue;
    if (e != cudaSuccess) return drop(e);
    h->dz = w + o_dz, h->dz_rows = type == CSER_TYPE_F16 ? w + o_dzr : nullptr, h->acc = reinterpret_cast<float *>(w + o_acc);
    return h;
}

int cser_xent_loss(cser_xent_handle h, const cser_xent_inputs *in, float *loss, float *lse, void *stream) {
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    XentArgs a;
    if (int rc = prepare_call(h, in, "cser_xent_loss", a, st)) return rc;
    if (a.tokens == 0) return CSER_OK;
    if (int rc = cser_internal_check_ptr(lse, "cser_xent_loss: lse")) return rc;
    if (loss)
        if (int rc = cser_internal_check_ptr(loss, "cser_xent_loss: loss")) return rc;
    if ((uintptr_t)lse % 4 || (uintptr_t)loss % 4)
        return cser_internal_fail(CSER_ERR_INVALID, "cser_xent_loss: a pointer is not aligned to its element type");
    a.loss = loss, a.lse_out = lse;
    return wide_tiles(a.tokens) ? loss_launch<2>(h, a, st) : loss_launch<1>(h, a, st);
}

int cser_xent_grad(cser_xent_handle h, const cser_xent_inputs *in, const float *lse, const float *dloss, void *dhidden,
                   void *dweight, int64_t dweight_stride, void *stream) {
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    XentArgs a;
    if (int rc = prepare_call(h, in, "cser_xent_grad", a, st)) return rc;
    if (!dhidden && !dweight) return CSER_OK;
    if (dweight) {
        if (int rc = cser_internal_check_ptr(dweight, "cser_xent_grad: dweight")) return rc;
        if (h->n > 1 && dweight_stride < h->vocab * h->dim)
            return cser_internal_fail(CSER_ERR_INVALID, "cser_xent_grad: dweight_stride must be at least vocab * dim");
    }
    if ((uintptr_t)dweight % 2 || (uintptr_t)dhidden % 2)
        return cser_internal_fail(CSER_ERR_INVALID, "cser_xent_grad: a pointer is not aligned to its element type");
    if (a.tokens == 0) {
        if (dweight)
            for (int w = 0; w < h->n; ++w)
                TRY(cudaMemsetAsync(static_cast<uint16_t *>(dweight) + w * dweight_stride, 0, (size_t)h->vocab * h->dim * 2, st));
        return CSER_OK;
    }
    if (int rc = cser_internal_check_ptr(lse, "cser_xent_grad: lse")) return rc;
    if (int rc = cser_internal_check_ptr(dloss, "cser_xent_grad: dloss")) return rc;
    if (dhidden)
        if (int rc = cser_internal_check_ptr(dhidden, "cser_xent_grad: dhidden")) return rc;
    if ((uintptr_t)lse % 4 || (uintptr_t)dloss % 4)
        return cser_internal_fail(CSER_ERR_INVALID, "cser_xent_grad: a pointer is not aligned to its element type");
    a.lse = lse, a.dloss = dloss, a.dh = dhidden, a.dw = dweight, a.dw_stride = dweight_stride;
    if (wide_tiles(a.tokens)) return grad_launch<2>(h, a, st);
    a.dh_boxes = result_map(h, a.dh_map, dhidden, a.tokens, (long long)a.tokens * h->dim);
    a.dw_boxes = result_map(h, a.dw_map, dweight, h->vocab, dweight_stride);
    return grad_launch<1>(h, a, st);
}

void cser_xent_destroy(cser_xent_handle h) {
    if (!h) return;
    for (void *p : {h->work, h->pack_h, h->pack_w})
        if (p) cudaFree(p);
    if (h->err_host) cser_internal_give_word(h->err_host);
    delete h;
}

int64_t cser_xent_launch_count(cser_xent_handle h) { return h ? h->launches : 0; }

}  // extern "C"
