/*
 * cser_layers.h - C ABI of the layers that stand between the matrix products of the n workers' models: dropout whose mask is
 * drawn from a counter-based generator and never stored, and group norm with an activation, channels last, each with its gradient.
 * They make the activations that the gradients of cser_step come from.
 *
 * Same library (libcser.so), error codes, cser_last_error(), element types and conventions as cser.h and cser_train.h: pointers are device
 * memory of the GPU that was current when the handle was created; `stream` is a cudaStream_t as void* (NULL = legacy default
 * stream); a call only enqueues work and returns; calls on one handle must not overlap, on the host or on the GPU (a handle's
 * workspace serves one call at a time).  Calls may be captured in a CUDA graph and replayed.  No call aborts, throws or
 * traps on the device, and no kernel waits for another.  Results are the same from call to call, bit for bit.
 *
 * A handle is made once for many calls: on a B200 0.03 to 0.35 ms for a workspace of more than 1 MB, and as much to
 * destroy.  The first call of a kind loads its kernel, 2 to 4 ms once in a process.
 */
#ifndef CSER_LAYERS_H_
#define CSER_LAYERS_H_

#include "cser_train.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Dropout.  Worker i's array is [rows, cols]; element e = row * cols + col of it (its place, whatever the strides) has the draw
 *     word e & 3 of Philox4x32-10, key = (seed low, seed high), counter = (e >> 2, step low, step high, 4096 * site + first_worker + i)
 * and is kept where the draw is at least floor(p * 2^32).  A counter's last word is 4096 or more, that of the step's block masks
 * (cser.h) 0 or 1: one seed serves both.  The same (seed, step, site, worker) gives the same mask on any GPU, in any call and for any
 * division of the workers over handles.
 *     y = residual + keep * (x + bias) / (1 - p)          bias, residual: none, one or both
 *     dx = keep * dy / (1 - p) ,   dbias = sum over rows of dx ,   (dresidual = dy)
 * A dropped element counts as 0 whatever its value, an infinity or NaN too.  Where workers share an array (a worker stride of 0), gradients are
 * still each worker's own.
 *
 * Arithmetic.  x, residual, y, dy and dx are of one type, F32, BF16 or F16; computed in fp32 and rounded once.  bias and dbias are
 * fp32; the sums are fp32, of values before their rounding, in a fixed order.
 */
typedef struct cser_drop *cser_drop_handle;

/* [n_workers, rows, cols] with any strides, in elements; the innermost dimension is contiguous.  Strides of what is read may be 0, none
 * may be negative.  Any alignment works. */
typedef struct cser_rows {
    void *data;
    int64_t row_stride, worker_stride;
} cser_rows;

/*
 * Handle for up to max_rows rows a worker.  0 <= p < 1 (and floor(p * 2^32) < 2^32); 1 <= site < 2^20: one number for each place of the
 * model that drops; first_worker >= 0 and first_worker + n_workers <= 4096; max_rows * cols <= 2^34.
 * The workspace, for sums of dbias, is none for a single row a worker, else 4 bytes for every 128 elements, up to 1.3 MB more where there are few, and
 * for each worker 1 KB and 4 bytes for each element of two of its rows, or of nine (five in 32 bits) where it has that many and 16 bytes do
 * not divide them.  Returns NULL on failure.
 */
cser_drop_handle cser_drop_create(int32_t n_workers, int64_t max_rows, int64_t cols, double p, uint64_t seed, uint32_t site,
                                  int32_t first_worker, int32_t type);
/*
 * step: 64 bits, any; step_at: NULL, or device memory holding a number that is added to step (modulo 2^64) when the call runs, so that a
 * replayed graph draws anew.  bias: fp32 [n_workers][cols], bias_stride elements from one worker's to the next (a part of the flat
 * state, say), or NULL.  residual: or NULL.  y may be x or residual itself (same pointer and strides); otherwise what a call writes must not
 * share memory with its other arrays (here and below).  Refused where the two have the same strides or one has no gaps.
 */
int cser_drop_apply(cser_drop_handle h, int64_t rows, uint64_t step, const uint64_t *step_at, const cser_rows *x,
                    const float *bias, int64_t bias_stride, const cser_rows *residual, const cser_rows *y, void *stream);
/* dx: or NULL; may be dy itself.  dbias: fp32 [n_workers][cols], dbias_stride (>= cols) elements from one worker's to the next (a part of
 * the flat gradient, say), or NULL.  With rows = 0 dbias becomes 0. */
int cser_drop_grad(cser_drop_handle h, int64_t rows, uint64_t step, const uint64_t *step_at, const cser_rows *dy,
                   const cser_rows *dx, float *dbias, int64_t dbias_stride, void *stream);
void cser_drop_destroy(cser_drop_handle h);
/* Number of kernels launched on behalf of the handle. */
int64_t cser_drop_launch_count(cser_drop_handle h);

/*
 * Group norm with an activation.  x is [n_workers, samples, pixels, channels], channels last; channel c belongs to group
 * c / (channels / groups).  With mean and var (of all values, not one fewer) over the pixels and channels of a group of one sample,
 *     rstd = 1 / sqrt(var + eps) ,  xhat = (x - mean) * rstd ,  z = xhat * weight + bias ,  y = act(z)
 * and for the upstream gradient dy, with N the values of a group,
 *     dz = dy * act'(z) ,  dweight = sum dz * xhat ,  dbias = sum dz                     over a worker's samples and pixels
 *     dx = rstd * (dz * weight - (sum dz * weight + xhat * sum dz * weight * xhat) / N)      sums over the group
 * act: none, relu (slope 0 at 0) or silu, z / (1 + exp(-z)).  With a dropout, x is dropout(x) in all of this, before its rounding: the
 * array is taken as [n_workers, samples * pixels, channels], and dx is the gradient for what was dropped from.
 *
 * Arithmetic.  x, y, dy and dx are of one type, F32, BF16 or F16.  Everything else is fp32; variances are sums of squares about means,
 * joined pairwise, so they do not cancel where the mean is large.  An infinity or NaN spoils its own group (and its worker's dweight and
 * dbias).
 */
#define CSER_ACT_NONE 0
#define CSER_ACT_RELU 1
#define CSER_ACT_SILU 2
typedef struct cser_norm *cser_norm_handle;

/* [n_workers, samples, pixels, channels] with any strides, in elements, as cser_rows. */
typedef struct cser_pixels {
    void *data;
    int64_t pixel_stride, sample_stride, worker_stride;
} cser_pixels;

/* What both calls read.  weight, bias: fp32 [n_workers][channels], weight_stride and bias_stride elements from one worker's to the next
 * (0 shares one), or NULL for 1 and 0. */
typedef struct cser_norm_inputs {
    cser_pixels x;
    const float *weight, *bias;
    int64_t weight_stride, bias_stride;
    int64_t samples, pixels;         /* samples: 0 .. max_samples of the handle; pixels: 0 .. 2^31 - 1 */
    uint64_t step;                   /* of the dropout, as in cser_drop_apply; not read without one */
    const uint64_t *step_at;
} cser_norm_inputs;

/*
 * 1 <= channels <= 65536, a multiple of groups; n_workers <= 4096, n_workers * max_samples <= 2^24, and times groups below 2^31; eps >= 0 and
 * finite.  drop: NULL, or a dropout for the same number of workers, of the same type and with `channels` columns; it is copied and may be
 * destroyed.  Its limit of rows does not matter here, but samples * pixels * channels <= 2^34 does.  The workspace is 8 bytes for each channel of
 * n_workers * max_samples + 1184 samples and 8 for each group of n_workers * max_samples.  Returns NULL on failure.
 */
cser_norm_handle cser_norm_create(int32_t n_workers, int64_t max_samples, int64_t channels, int64_t groups, int32_t act, float eps,
                                  int32_t type, cser_drop_handle drop);
/* stats: fp32 [2, n_workers, samples, groups], dense: mean, then rstd; what cser_norm_grad takes.  y may be x itself (same pointer and
 * strides).  With pixels = 0 the stats become 0. */
int cser_norm_apply(cser_norm_handle h, const cser_norm_inputs *in, const cser_pixels *y, float *stats, void *stream);
/* stats: as cser_norm_apply gave them for the same inputs.  dx: or NULL; may be x or dy itself.  dweight, dbias: fp32 [n_workers][channels],
 * dweight_stride and dbias_stride (>= channels) elements from one worker's to the next, or NULL; 0 where samples or pixels are 0. */
int cser_norm_grad(cser_norm_handle h, const cser_norm_inputs *in, const float *stats, const cser_pixels *dy, const cser_pixels *dx,
                   float *dweight, int64_t dweight_stride, float *dbias, int64_t dbias_stride, void *stream);
void cser_norm_destroy(cser_norm_handle h);
int64_t cser_norm_launch_count(cser_norm_handle h);

#ifdef __cplusplus
}
#endif
#endif /* CSER_LAYERS_H_ */
