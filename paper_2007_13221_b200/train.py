"""ctypes binding of the operators of ``include/cser_train.h`` - argument marshalling only.

They live in the same ``libcser.so`` as the optimizer step (``binding``) and surround it in a training step:
``LinearCrossEntropy`` gives the loss of a language model's head and its gradient, ``Orthogonalizer`` turns the
matrices inside the flat [n_workers, d] gradient into orthogonalised updates that ``binding.CSER.step`` takes.

``stream``: where a call runs (default: torch's current stream).  What it reads has to be ready there; results that it makes
are made there, and the caller orders their use elsewhere.  Memory is safe without that: tensors may be dropped after the call.
"""
import ctypes

import torch

from .binding import CSERError, _check, _release, _stream, cser_last_error
from .binding import lib as _base_lib

TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}

_lib = None


class _XentInputs(ctypes.Structure):
    _fields_ = [("hidden", ctypes.c_void_p), ("hidden_row_stride", ctypes.c_int64),
                ("hidden_worker_stride", ctypes.c_int64), ("weight", ctypes.c_void_p),
                ("weight_row_stride", ctypes.c_int64), ("weight_worker_stride", ctypes.c_int64),
                ("target", ctypes.c_void_p), ("ignore_index", ctypes.c_int64), ("tokens", ctypes.c_int64)]


def lib():
    """libcser.so with the signatures of cser_train.h."""
    global _lib
    if _lib is not None:
        return _lib
    L, c = _base_lib(), ctypes
    p, i32, i64, f32 = c.c_void_p, c.c_int32, c.c_int64, c.c_float
    for name, res, args in (
            ("cser_orth_create", p, [i32, i64, i32, p, p, p, p, p, i32, i32, i32]),
            ("cser_orth_apply", c.c_int, [p, p, p, f32, p, p]),
            ("cser_orth_destroy", None, [p]),
            ("cser_orth_debug_stall_next", c.c_int, [p, c.c_uint]),
            ("cser_orth_launch_count", i64, [p]),
            ("cser_xent_create", p, [i32, i64, i64, i64, i32, i64]),
            ("cser_xent_loss", c.c_int, [p, c.POINTER(_XentInputs), p, p, p]),
            ("cser_xent_grad", c.c_int, [p, c.POINTER(_XentInputs), p, p, p, p, i64, p]),
            ("cser_xent_destroy", None, [p]),
            ("cser_xent_launch_count", i64, [p])):
        f = getattr(L, name)
        f.restype, f.argtypes = res, args
    _lib = L
    return L


def _want(ok, what):
    if not ok:
        raise CSERError(what)


def _on(stream, call, *args):
    """call(...) with `stream` as the current one.  The allocator does not give out the arguments' memory again before `stream` has
    passed this point, nor the results' before the caller's stream has passed the place where they are dropped."""
    here = torch.cuda.current_stream()
    if not isinstance(stream, torch.cuda.Stream):    # another package's, known by its cuda_stream
        stream = torch.cuda.ExternalStream(stream.cuda_stream)
    for t in args:
        if torch.is_tensor(t) and t.is_cuda:
            t.record_stream(stream)
    with torch.cuda.stream(stream):
        got = call(*args)
    for t in got if isinstance(got, tuple) else (got,):
        if t is not None:
            t.record_stream(here)
    return got


class Orthogonalizer:
    """Plan for the matrices ``[(offset, rows, cols), ...]`` inside each row of an [n_workers, ld] array.

    ``row_strides``: elements from one row of a matrix to the next (default: cols); ``scales``: factor of each
    result (default: 1).  See cser_orth_create.
    """

    def __init__(self, matrices, n_workers, ld, in_dtype=torch.float32, out_dtype=torch.float32, row_strides=None,
                 scales=None, steps=5):
        self.h = None
        _want(in_dtype in TYPES and out_dtype in TYPES, "Orthogonalizer: types are float32, bfloat16 and float16")
        k = len(matrices)
        i64 = ctypes.c_int64 * max(1, k)
        for name, extra in (("row_strides", row_strides), ("scales", scales)):
            _want(extra is None or len(extra) == k, f"Orthogonalizer: {name} needs one value per matrix")
        self.n, self.ld, self.in_dtype, self.out_dtype = int(n_workers), int(ld), in_dtype, out_dtype
        off, rows, cols = (i64(*(int(m[j]) for m in matrices)) for j in range(3))
        stride = i64(*map(int, row_strides)) if row_strides is not None else None
        scale = (ctypes.c_float * max(1, k))(*map(float, scales)) if scales is not None else None
        h = lib().cser_orth_create(self.n, self.ld, k, off, rows, cols, stride, scale, int(steps), TYPES[in_dtype],
                                   TYPES[out_dtype])
        if not h:
            raise CSERError(f"cser_orth_create failed: {cser_last_error()}")
        self.h = ctypes.c_void_p(h)

    def apply(self, grad, out=None, momentum=None, mu=0.0, stream=None):
        """grad [n, ld] -> out [n, ld] (made if not given: zeros outside the matrices); momentum is updated in place."""
        if stream is not None:
            return _on(stream, self.apply, grad, out, momentum, mu)
        size = (self.n, self.ld)
        if not (grad.is_cuda and grad.dtype == self.in_dtype and grad.shape == size and grad.is_contiguous()):
            raise CSERError(f"Orthogonalizer: grad must be a contiguous CUDA {self.in_dtype} tensor of shape {size}")
        if out is None:
            out = torch.zeros(size, dtype=self.out_dtype, device=grad.device)
        if not (out.is_cuda and out.dtype == self.out_dtype and out.shape == size and out.is_contiguous()):
            raise CSERError(f"Orthogonalizer: out must be a contiguous CUDA {self.out_dtype} tensor of shape {size}")
        if momentum is not None and not (momentum.is_cuda and momentum.dtype == torch.float32 and momentum.shape == size and
                                         momentum.is_contiguous()):
            raise CSERError(f"Orthogonalizer: momentum must be a contiguous CUDA float32 tensor of shape {size}")
        _check(_lib.cser_orth_apply(self.h, grad.data_ptr(), None if momentum is None else momentum.data_ptr(), mu,
                                    out.data_ptr(), _stream()), "cser_orth_apply")
        return out

    @property
    def launches(self):
        return int(lib().cser_orth_launch_count(self.h))

    def close(self):
        if self.h is not None:
            h, self.h = self.h, None
            _release(lib().cser_orth_destroy, h)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class LinearCrossEntropy:
    """Softmax cross entropy of hidden @ weight^T against targets, in pieces of the vocabulary, and its gradient.

    Workspace for up to ``max_tokens`` tokens of each of ``n_workers`` workers; ``piece``: vocabulary entries per piece
    of the gradient (0: chosen by size).  hidden is [n, tokens, dim], weight [n, vocab, dim] (an ``expand``ed leading
    dimension shares one array), target int64 [n, tokens].  See cser_xent_create.
    """

    def __init__(self, n_workers, max_tokens, vocab, dim, dtype=torch.bfloat16, piece=0):
        self.h = None
        _want(dtype in TYPES, "LinearCrossEntropy: types are bfloat16 and float16")
        self.n, self.max_tokens, self.vocab, self.dim = int(n_workers), int(max_tokens), int(vocab), int(dim)
        self.dtype = dtype
        h = lib().cser_xent_create(self.n, self.max_tokens, self.vocab, self.dim, TYPES[dtype], int(piece))
        if not h:
            raise CSERError(f"cser_xent_create failed: {cser_last_error()}")
        self.h = ctypes.c_void_p(h)

    def _inputs(self, hidden, weight, target, ignore_index):
        n, dim = self.n, self.dim
        if not (target.is_cuda and target.dtype == torch.int64 and target.dim() == 2 and target.shape[0] == n and
                target.shape[1] <= self.max_tokens and target.is_contiguous()):
            raise CSERError(f"LinearCrossEntropy: target must be a contiguous CUDA int64 tensor [{n}, at most {self.max_tokens}]")
        t = target.shape[1]
        hs, ws = hidden.stride(), weight.stride()
        if not (hidden.is_cuda and hidden.dtype == self.dtype and hidden.shape == (n, t, dim) and (hs[2] == 1 or dim == 1)):
            raise CSERError(f"LinearCrossEntropy: hidden must be a CUDA {self.dtype} tensor of shape {(n, t, dim)} with a contiguous "
                            "last dimension")
        if not (weight.is_cuda and weight.dtype == self.dtype and weight.shape == (n, self.vocab, dim) and (ws[2] == 1 or dim == 1)):
            raise CSERError(f"LinearCrossEntropy: weight must be a CUDA {self.dtype} tensor of shape {(n, self.vocab, dim)} with a "
                            "contiguous last dimension")
        return _XentInputs(hidden.data_ptr(), hs[1], hs[0], weight.data_ptr(), ws[1], ws[0], target.data_ptr(), ignore_index, t)

    def loss(self, hidden, weight, target, ignore_index=-100, stream=None):
        """(loss, lse), each fp32 [n, tokens]; lse is what grad takes."""
        if stream is not None:
            return _on(stream, self.loss, hidden, weight, target, ignore_index)
        args = self._inputs(hidden, weight, target, ignore_index)
        loss, lse = torch.empty_like(target, dtype=torch.float32), torch.empty_like(target, dtype=torch.float32)
        _check(_lib.cser_xent_loss(self.h, ctypes.byref(args), loss.data_ptr(), lse.data_ptr(), _stream()), "cser_xent_loss")
        return loss, lse

    def grad(self, hidden, weight, target, lse, dloss, ignore_index=-100, dhidden=None, dweight=None, need_dhidden=True,
             need_dweight=True, stream=None):
        """(dhidden, dweight) of sum(dloss * loss); dweight may be a [n, vocab, dim] view of a larger [n, d] array."""
        if stream is not None:
            return _on(stream, self.grad, hidden, weight, target, lse, dloss, ignore_index, dhidden, dweight, need_dhidden, need_dweight)
        args = self._inputs(hidden, weight, target, ignore_index)
        for a in (lse, dloss):
            if not (a.is_cuda and a.dtype == torch.float32 and a.shape == target.shape and a.is_contiguous()):
                raise CSERError("LinearCrossEntropy: lse and dloss must be contiguous CUDA float32 tensors of target's shape")
        if need_dhidden:
            if dhidden is None:
                dhidden = torch.empty_like(hidden, memory_format=torch.contiguous_format)   # half the time of empty()
            elif not (dhidden.is_cuda and dhidden.dtype == self.dtype and dhidden.shape == hidden.shape and dhidden.is_contiguous()):
                raise CSERError(f"LinearCrossEntropy: dhidden must be a contiguous CUDA {self.dtype} tensor of hidden's shape")
        if need_dweight:
            if dweight is None:
                dweight = torch.empty_like(weight, memory_format=torch.contiguous_format)
            elif not (dweight.is_cuda and dweight.dtype == self.dtype and dweight.shape == weight.shape and
                      (self.dim == 1 or dweight.stride(2) == 1) and (self.vocab == 1 or dweight.stride(1) == self.dim) and
                      (self.n == 1 or dweight.stride(0) >= self.vocab * self.dim)):
                raise CSERError(f"LinearCrossEntropy: dweight must be a CUDA {self.dtype} tensor of weight's shape, dense for each worker")
        _check(_lib.cser_xent_grad(self.h, ctypes.byref(args), lse.data_ptr(), dloss.data_ptr(),
                                   dhidden.data_ptr() if need_dhidden else None,
                                   dweight.data_ptr() if need_dweight else None,
                                   max(dweight.stride(0), self.vocab * self.dim) if need_dweight else 0, _stream()),
               "cser_xent_grad")
        return dhidden if need_dhidden else None, dweight if need_dweight else None

    @property
    def launches(self):
        return int(lib().cser_xent_launch_count(self.h))

    def close(self):
        if self.h is not None:
            h, self.h = self.h, None
            _release(lib().cser_xent_destroy, h)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
