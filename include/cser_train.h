/*
 * cser_train.h - C ABI of the operators of a training step around the optimizer step of cser.h: the loss of a language
 * model's head with its gradient, where the gradients begin, and the orthogonalisation of the matrices inside them,
 * which turns a gradient (with its momentum) into the update that cser_step communicates and applies.
 *
 * Same library (libcser.so), error codes, cser_last_error() and conventions as cser.h: pointers are device memory of
 * the GPU that was current when the handle was created; `stream` is a cudaStream_t as void* (NULL = legacy default
 * stream); a call only enqueues work and returns; calls on one handle must not overlap, on the host or on the GPU (a
 * handle's workspace serves one call at a time).  Calls may be captured in a CUDA
 * graph and replayed (but see cser_xent_create for unaligned inputs).  No call aborts, throws or traps on the device.  Every wait inside a
 * kernel is bounded to about a second; one that ran out (the GPU withheld from part of a launch, say) ends the kernel and every
 * later call on the handle returns CSER_ERR_CUDA, the results of that call being incomplete.
 *
 * A handle is made once for many calls: creation allocates, copies its tables and asks the driver about kernels, and destruction waits for
 * the GPU.  On a B200 0.4 to 1 ms for the cross entropy and 0.8 to 2.8 ms for a plan, up to 17 ms for a process's first (its kernels
 * are loaded), 0.3 to 3.3 ms to destroy: more than many a call takes.
 */
#ifndef CSER_TRAIN_H_
#define CSER_TRAIN_H_

#include "cser.h"

#ifdef __cplusplus
extern "C" {
#endif

/* element types */
#define CSER_TYPE_F32  0
#define CSER_TYPE_BF16 1
#define CSER_TYPE_F16  2

/*
 * Orthogonalised updates.  A plan lists n_matrices matrices inside a flat vector of ld elements, which n_workers
 * workers hold as an [n_workers, ld] array (row i is worker i's vector, the layout of cser_step's grad).  For every
 * matrix of every worker cser_orth_apply computes
 *     u = g                                       without momentum (m = NULL)
 *     m <- mu*m + g ;  u = g + mu*m               with momentum (Nesterov's form, as in step 1 of cser.h)
 *     X = u / (|u|_F + 1e-7)
 *     `steps` times:  X <- a X + (b A + c A A) X, A = X X^T     (rows <= cols; else X <- X (a I + b A + c A A), A = X^T X)
 *                     (a, b, c) = (3.4445, -4.7750, 2.0315)
 *     out = scale * X
 * which drives the singular values of u towards 1 (to within 0.68 .. 1.21 for those that five steps reach) and keeps
 * its singular vectors.  A matrix of zeros gives zeros.  Infinities and NaN spoil their own matrix only.
 * Momenta and outputs outside the listed matrices are neither read nor written.
 *
 * Arithmetic.  in_type F32, BF16 or F16; momentum fp32.  Matrices with a short side of at most 64 go through their Gram
 * matrix in 64 bits.  Others: norms and sums fp32, so |u|_F below 2^64 (from there on the result is 0), and X in fp16's range: a matrix with |u|_F
 * below about 1e-15 sqrt(rows cols), of which 1e-7 leaves next to nothing, keeps fewer bits in a 16-bit result; out_type BF16 or F16: the products take
 * fp16 operands (11 bits), with the remainder of X and the diagonals of A and b A + c A A carried in addition, which
 * leaves about 1e-3 relative error at most before the rounding of the result.  out_type F32: the operands are pairs of
 * fp16 (22 bits) and each product is three, about 1e-6.  Results are the same from call to call, bit for bit.
 */
typedef struct cser_orth *cser_orth_handle;

/*
 * n_workers * ld at most 2^46.  offset[k], rows[k], cols[k]: where matrix k begins in a worker's vector and its shape (row-major),
 * 1 <= rows, cols <= 65536.  row_stride[k] >= cols[k]: elements from one row to the next (NULL: cols[k]).  scale[k]: finite factor of the
 * result (NULL: 1).  Matrices must lie inside the vector and share no element.  steps: 1..16.  The arrays are host memory
 * and are copied.  The plan owns a workspace of about 8 bytes per element (16 for a 32-bit result) for all matrices of all workers or 2 GB,
 * whichever is less (more only where one matrix needs more), and at most 20 MB for sums that CTAs share.  Matrices that do not fit
 * these 2 GB together go through it in groups, of three kernels each; those with a short side of at most 64 take up to three more.  Returns
 * NULL on failure.
 */
cser_orth_handle cser_orth_create(int32_t n_workers, int64_t ld, int32_t n_matrices, const int64_t *offset,
                                  const int64_t *rows, const int64_t *cols, const int64_t *row_stride,
                                  const float *scale, int32_t steps, int32_t in_type, int32_t out_type);
/*
 * grad: [n_workers, ld] of in_type.  m: fp32 [n_workers, ld], updated in place, or NULL (then mu is ignored).  0 <= mu < 1.
 * out: [n_workers, ld] of out_type; may be grad itself where the types are the same.  Otherwise the three arrays must not overlap from the
 * first matrix's beginning to the last one's end.
 */
int cser_orth_apply(cser_orth_handle h, const void *grad, float *m, float mu, void *out, void *stream);
void cser_orth_destroy(cser_orth_handle h);
/*
 * Test hook for the bounded waits.  In the NEXT cser_orth_apply the tiled kernel waits for something that does not happen, and every wait is
 * limited to wait_mcycles million SM clock cycles (1 .. 2000; the normal limit is 2000, about a second).  The wait runs out, the
 * kernel ends, and every later cser_orth_apply on the plan returns CSER_ERR_CUDA.  Nothing traps and the CUDA context stays
 * usable.  CSER_ERR_INVALID where all matrices have a short side of at most 64: no kernel waits then.
 */
int cser_orth_debug_stall_next(cser_orth_handle h, unsigned wait_mcycles);
/* Number of kernels launched on behalf of the plan. */
int64_t cser_orth_launch_count(cser_orth_handle h);

/*
 * Softmax cross entropy of a linear head over a large vocabulary, in pieces of the vocabulary; the logits are never
 * kept.  For worker i, token t:
 *     z_v = <hidden[i,t,:], weight[i,v,:]> ,   lse = log sum_v exp z_v ,   loss = lse - z_target
 * and for the upstream gradients dloss[i,t]:
 *     dz_v = (exp(z_v - lse) - [v = target]) * dloss ,   dhidden = sum_v dz_v weight[v] ,   dweight[v] = sum_t dz_v hidden[t]
 * A token whose target is ignore_index has loss 0 and adds nothing to the gradients, even where its hidden state is not finite; nor does
 * one whose dloss is 0.  A target outside 0..vocab-1 that is not ignore_index makes that token's loss NaN, its row of dhidden NaN and its
 * worker's dweight NaN; so does, for the gradients, a dloss that is not finite of a token that counts.
 *
 * Arithmetic.  hidden, weight, dhidden and dweight are of one type, BF16 or F16.  Logits, sums, lse and loss are fp32.  dz is
 * held in the operands' type between the products (up to 32 tokens with what that rounding leaves), relative to the worker's largest finite |dloss|, so a uniform dloss (the mean
 * over the tokens) adds no rounding; F16: where the |dloss| of a worker's tokens are more than 2^6 apart, a second time relative to each
 * token's own for dhidden, so that its rows are as exact whatever their weight.  Sums over pieces are fp32, in
 * a fixed order: results are the same from call to call.
 */
typedef struct cser_xent *cser_xent_handle;

/* What both calls read.  Strides in elements; the innermost dimension is contiguous.  A worker stride of 0 shares one
 * array between the workers.  Any alignment and stride works; 16-byte aligned pointers and strides need no repacking. */
typedef struct cser_xent_inputs {
    const void *hidden;             /* [n_workers, tokens, dim] */
    int64_t hidden_row_stride, hidden_worker_stride;
    const void *weight;             /* [n_workers, vocab, dim] */
    int64_t weight_row_stride, weight_worker_stride;
    const int64_t *target;          /* [n_workers, tokens], dense */
    int64_t ignore_index;
    int64_t tokens;                 /* 0 .. max_tokens of the handle */
} cser_xent_inputs;

/*
 * Handle for up to max_tokens tokens per worker.  piece: vocabulary entries per piece of the gradient (rounded up to a multiple of
 * 256), 0 = as many as 256 MB of dz hold, but 2048 at least.  The workspace, all of it allocated here, with T = max_tokens rounded up to
 * 256: dz, n_workers * T * piece * 2 bytes (twice for F16); parts of the losses, n_workers * max_tokens * vocab / 8; a copy of the
 * hidden states; and, where the vocabulary is gone through in several pieces or dhidden has few tiles, its fp32 sums.  1 <= vocab <= 2^24, 1 <= dim <= 65536,
 * 1 <= n_workers * max_tokens <= 2^24, n_workers * vocab and n_workers * ceil(max_tokens / 128) * ceil(vocab / 256) at most 2^30.
 * hidden or weights whose rows are not a multiple of 16 bytes apart (or not 16-byte aligned) are first copied: the buffer for that is
 * allocated with the handle where dim is no multiple of 8, else on the first such call, which must not be under stream capture.  Returns
 * NULL on failure.
 */
cser_xent_handle cser_xent_create(int32_t n_workers, int64_t max_tokens, int64_t vocab, int64_t dim, int32_t type,
                                  int64_t piece);
/* loss, lse: fp32 [n_workers, tokens], dense.  lse is what cser_xent_grad takes; loss may be NULL. */
int cser_xent_loss(cser_xent_handle h, const cser_xent_inputs *in, float *loss, float *lse, void *stream);
/*
 * lse: as cser_xent_loss gave it for the same inputs.  dloss: fp32 [n_workers, tokens], dense.
 * dhidden: [n_workers, tokens, dim], dense, or NULL.  dweight: [n_workers][vocab, dim], each worker's dense, dweight_stride
 * elements (>= vocab*dim) from one worker to the next, or NULL.  With tokens = 0, dweight becomes 0.  What is written must not overlap
 * what is read.
 */
int cser_xent_grad(cser_xent_handle h, const cser_xent_inputs *in, const float *lse, const float *dloss, void *dhidden,
                   void *dweight, int64_t dweight_stride, void *stream);
void cser_xent_destroy(cser_xent_handle h);
int64_t cser_xent_launch_count(cser_xent_handle h);

#ifdef __cplusplus
}
#endif
#endif /* CSER_TRAIN_H_ */
