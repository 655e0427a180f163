"""ctypes binding of the layers of ``include/cser_layers.h`` - argument marshalling only.

They live in the same ``libcser.so`` as the optimizer step (``binding``) and stand between the matrix products of the n
workers' models: ``Dropout`` draws its mask from a counter-based generator and never stores it, ``GroupNorm`` is group norm with an
activation, channels last.  Parameters and their gradients are fp32 [n, channels] and may be views of the flat [n, d] state and
gradient of ``binding.CSER``.

``stream``: where a call runs (default: torch's current stream), as in ``train``.
"""
import ctypes

import torch

from .binding import CSERError, _check, _release, cser_last_error
from .binding import lib as _base_lib
from .train import TYPES, _on, _want

ACTIVATIONS = {"none": 0, None: 0, "relu": 1, "silu": 2}

_lib = None


class _Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("worker_stride", ctypes.c_int64)]


class _Pixels(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("pixel_stride", ctypes.c_int64), ("sample_stride", ctypes.c_int64),
                ("worker_stride", ctypes.c_int64)]


class _NormInputs(ctypes.Structure):
    _fields_ = [("x", _Pixels), ("weight", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("weight_stride", ctypes.c_int64),
                ("bias_stride", ctypes.c_int64), ("samples", ctypes.c_int64), ("pixels", ctypes.c_int64),
                ("step", ctypes.c_uint64), ("step_at", ctypes.c_void_p)]


def lib():
    """libcser.so with the signatures of cser_layers.h."""
    global _lib
    if _lib is not None:
        return _lib
    L, c = _base_lib(), ctypes
    p, i32, i64, u32, u64 = c.c_void_p, c.c_int32, c.c_int64, c.c_uint32, c.c_uint64
    rows, pixels, inputs = c.POINTER(_Rows), c.POINTER(_Pixels), c.POINTER(_NormInputs)
    for name, res, args in (
            ("cser_drop_create", p, [i32, i64, i64, c.c_double, u64, u32, i32, i32]),
            ("cser_drop_apply", c.c_int, [p, i64, u64, p, rows, p, i64, rows, rows, p]),
            ("cser_drop_grad", c.c_int, [p, i64, u64, p, rows, rows, p, i64, p]),
            ("cser_drop_destroy", None, [p]),
            ("cser_drop_launch_count", i64, [p]),
            ("cser_norm_create", p, [i32, i64, i64, i64, i32, c.c_float, i32, p]),
            ("cser_norm_apply", c.c_int, [p, inputs, pixels, p, p]),
            ("cser_norm_grad", c.c_int, [p, inputs, p, pixels, pixels, p, i64, p, i64, p]),
            ("cser_norm_destroy", None, [p]),
            ("cser_norm_launch_count", i64, [p])):
        f = getattr(L, name)
        f.restype, f.argtypes = res, args
    _lib = L
    return L


def _merged(name, shape, stride, first, last):
    """Size and stride of the axes first .. last - 1 taken as one."""
    size, step = 1, 0
    for k in range(last - 1, first - 1, -1):
        if shape[k] == 1:
            continue
        if size > 1 and stride[k] != size * step:
            raise CSERError(f"{name}: its middle dimensions cannot be taken as one; make it contiguous")
        if size == 1:
            step = stride[k]
        size *= shape[k]
    return size, step


def _number(what, v, bits=64):
    """v as a signed number of so many bits, which ctypes would cut without a word."""
    v = int(v)
    _want(-1 << bits - 1 <= v < 1 << bits - 1, f"{what} is out of range")
    return v


def _step(step):
    """(64 bits of the number, device pointer) of a step given as a number or as an int64 CUDA tensor of one element."""
    if torch.is_tensor(step):
        _want(step.is_cuda and step.dtype == torch.int64 and step.numel() == 1, "step must be a number or a CUDA int64 tensor of one element")
        return 0, step.data_ptr()
    return int(step) & 0xFFFFFFFFFFFFFFFF, None


def _params(name, t, n, cols):
    """(pointer, worker stride) of an fp32 [n, cols] tensor or None."""
    if t is None:
        return None, 0
    stride = t.stride()
    if not (t.dtype is torch.float32 and t.shape == (n, cols) and (stride[1] == 1 or cols == 1) and t.is_cuda):
        raise CSERError(f"{name} must be a CUDA float32 tensor of shape {(n, cols)} with a contiguous last dimension")
    return t.data_ptr(), stride[0]


def _like(t):
    """A dense tensor of t's shape and type."""
    return torch.empty_like(t) if t.is_contiguous() else torch.empty_like(t, memory_format=torch.contiguous_format)


def _raw_stream(t):
    """The current stream of t's device."""
    return torch._C._cuda_getCurrentRawStream(t.get_device())


class _Handle:
    """What both kinds of handle do at their end."""

    @property
    def launches(self):
        return int(getattr(lib(), f"cser_{self._kind}_launch_count")(self.h))

    def close(self):
        if self.h is not None:
            h, self.h = self.h, None
            _release(getattr(lib(), f"cser_{self._kind}_destroy"), h)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Dropout(_Handle):
    """Dropout of [n, ..., cols] arrays of up to ``max_rows`` rows a worker, with a bias before and a residual after it where wanted.

    The mask is a function of (seed, step, site, worker, place): ``site`` is a number of 1 or more for each place of the model that
    drops, ``first_worker`` the number of the first of these workers among all.  See cser_drop_create.
    """
    _kind = "drop"

    def __init__(self, n_workers, max_rows, cols, p, seed, site, dtype=torch.bfloat16, first_worker=0):
        self.h = None
        _want(dtype in TYPES, "Dropout: types are float32, bfloat16 and float16")
        _want(0 <= site < 2 ** 32, "Dropout: site must be in 1..2^20-1")
        self.n, self.max_rows, self.cols = _number("Dropout: n_workers", n_workers, 32), _number("Dropout: max_rows", max_rows), _number("Dropout: cols", cols)
        self.p, self.dtype = float(p), dtype
        h = lib().cser_drop_create(self.n, self.max_rows, self.cols, self.p, int(seed) & 0xFFFFFFFFFFFFFFFF, int(site),
                                   _number("Dropout: first_worker", first_worker, 32), TYPES[dtype])
        if not h:
            raise CSERError(f"cser_drop_create failed: {cser_last_error()}")
        self.h = ctypes.c_void_p(h)

    def _array(self, name, t, like=None):
        shape = t.shape
        if (t.dtype is self.dtype and t.is_contiguous() and t.is_cuda and
                (shape == like.shape if like is not None else len(shape) >= 2 and shape[0] == self.n and shape[-1] == self.cols)):
            each = t.numel() // self.n                    # the ordinary case, without its strides
            return each // self.cols, _Rows(t.data_ptr(), self.cols, each)
        if not (t.is_cuda and t.dtype == self.dtype and t.dim() >= 2 and shape[0] == self.n and shape[-1] == self.cols and
                (like is None or shape == like.shape)):
            raise CSERError(f"Dropout: {name} must be a CUDA {self.dtype} tensor of shape " +
                            (f"[{self.n}, ..., {self.cols}]" if like is None else f"{tuple(like.shape)}"))
        stride = t.stride()
        _want(stride[-1] == 1 or self.cols == 1, f"Dropout: the last dimension of {name} must be contiguous")
        if t.dim() == 3:
            rows, step = shape[1], stride[1]
        else:
            rows, step = _merged(f"Dropout: {name}", shape, stride, 1, t.dim() - 1)
        return rows, _Rows(t.data_ptr(), step, stride[0])

    def apply(self, x, step, bias=None, residual=None, out=None, stream=None):
        """residual + dropout(x + bias); bias fp32 [n, cols], residual like x.  out may be x or residual."""
        if stream is not None:
            return _on(stream, self.apply, x, step, bias, residual, out)
        rows, xs = self._array("x", x)
        step, step_at = _step(step)
        b, b_stride = _params("Dropout: bias", bias, self.n, self.cols)
        rs = None if residual is None else self._array("residual", residual, x)[1]
        if out is None:
            out = _like(x)
            ys = _Rows(out.data_ptr(), self.cols, rows * self.cols)
        else:
            ys = self._array("out", out, x)[1]
        rc = _lib.cser_drop_apply(self.h, rows, step, step_at, xs, b, b_stride, rs, ys, _raw_stream(x))
        if rc:
            _check(rc, "cser_drop_apply")
        return out

    def grad(self, dy, step, dx=None, dbias=None, need_dx=True, need_dbias=False, stream=None):
        """(dx, dbias) of sum(dy * apply(x, step, bias, residual)); the residual's gradient is dy.  dx may be dy; dbias (None unless
        given or needed) may be a view of a flat [n, d] gradient."""
        if stream is not None:
            return _on(stream, self.grad, dy, step, dx, dbias, need_dx, need_dbias)
        rows, ds = self._array("dy", dy)
        step, step_at = _step(step)
        xs = None
        if need_dx:
            if dx is None:
                dx = _like(dy)
                xs = _Rows(dx.data_ptr(), self.cols, rows * self.cols)
            else:
                xs = self._array("dx", dx, dy)[1]
        if dbias is None and need_dbias:
            dbias = torch.empty((self.n, self.cols), dtype=torch.float32, device=dy.device)
        b, b_stride = _params("Dropout: dbias", dbias, self.n, self.cols)
        _check(_lib.cser_drop_grad(self.h, rows, step, step_at, ds, xs, b, b_stride, _raw_stream(dy)), "cser_drop_grad")
        return dx if need_dx else None, dbias


class GroupNorm(_Handle):
    """Group norm with an activation ("none", "relu" or "silu") of [n, samples, ..., channels] arrays, up to ``max_samples`` a worker.

    dropout: a ``Dropout`` for the same workers, channels and type; x then counts as dropout(x), and every call needs the dropout's step.
    It is copied.  See cser_norm_create.
    """
    _kind = "norm"

    def __init__(self, n_workers, max_samples, channels, groups, activation="none", eps=1e-5, dtype=torch.bfloat16, dropout=None):
        self.h = None
        _want(dtype in TYPES, "GroupNorm: types are float32, bfloat16 and float16")
        _want(activation in ACTIVATIONS, 'GroupNorm: activations are "none", "relu" and "silu"')
        _want(dropout is None or dropout.h is not None, "GroupNorm: the dropout is closed")
        self.n, self.max_samples = _number("GroupNorm: n_workers", n_workers, 32), _number("GroupNorm: max_samples", max_samples)
        self.channels, self.groups = _number("GroupNorm: channels", channels), _number("GroupNorm: groups", groups)
        self.dtype, self.drops = dtype, dropout is not None
        h = lib().cser_norm_create(self.n, self.max_samples, self.channels, self.groups, ACTIVATIONS[activation], float(eps), TYPES[dtype],
                                   None if dropout is None else dropout.h)
        if not h:
            raise CSERError(f"cser_norm_create failed: {cser_last_error()}")
        self.h = ctypes.c_void_p(h)

    def _array(self, name, t, like=None):
        shape = t.shape
        if (t.dtype is self.dtype and t.is_contiguous() and t.is_cuda and
                (shape == like.shape if like is not None else len(shape) >= 3 and shape[0] == self.n and shape[-1] == self.channels)):
            each = t.numel() // self.n                    # the ordinary case, without its strides
            sample = each // shape[1] if each else 0
            if each or shape[1] == 0:
                return sample // self.channels, _Pixels(t.data_ptr(), self.channels, sample, each)
        if not (t.is_cuda and t.dtype == self.dtype and t.dim() >= 3 and shape[0] == self.n and shape[-1] == self.channels and
                (like is None or shape == like.shape)):
            raise CSERError(f"GroupNorm: {name} must be a CUDA {self.dtype} tensor of shape " +
                            (f"[{self.n}, samples, ..., {self.channels}]" if like is None else f"{tuple(like.shape)}"))
        stride = t.stride()
        _want(stride[-1] == 1 or self.channels == 1, f"GroupNorm: the last dimension of {name} must be contiguous")
        pixels, step = _merged(f"GroupNorm: {name}", shape, stride, 2, t.dim() - 1)
        return pixels, _Pixels(t.data_ptr(), step, stride[1], stride[0])

    def _dense(self, t, args):
        """A dense array of x's shape, as just made."""
        sample = args.pixels * self.channels
        return _Pixels(t.data_ptr(), self.channels, sample, sample * args.samples)

    def _new_params(self, like, x):
        if like is not None and like.is_contiguous():
            return torch.empty_like(like)                 # half the time of empty()
        return torch.empty((self.n, self.channels), dtype=torch.float32, device=x.device)

    def _inputs(self, x, weight, bias, step):
        if step is None:                                  # (one left out would mean one mask for ever, or another one in the gradient)
            _want(not self.drops, "GroupNorm: with a dropout each call needs its step")
            step = 0
        pixels, xs = self._array("x", x)
        step, step_at = _step(step)
        w, w_stride = _params("GroupNorm: weight", weight, self.n, self.channels)
        b, b_stride = _params("GroupNorm: bias", bias, self.n, self.channels)
        return _NormInputs(xs, w, b, w_stride, b_stride, x.shape[1], pixels, step, step_at)

    def apply(self, x, weight=None, bias=None, step=None, out=None, stream=None):
        """(act(norm(x) * weight + bias), stats); weight and bias fp32 [n, channels] or None.  stats, fp32 [2, n, samples, groups] (mean and
        1 / deviation), is what grad takes.  step: of the dropout, where there is one.  out may be x."""
        if stream is not None:
            return _on(stream, self.apply, x, weight, bias, step, out)
        args = self._inputs(x, weight, bias, step)
        if out is None:
            out = _like(x)
            ys = self._dense(out, args)
        else:
            ys = self._array("out", out, x)[1]
        size = (2, self.n, args.samples, self.groups)
        stats = torch.empty(size, dtype=torch.float32, device=x.device) if weight is None else weight.new_empty(size)
        _check(_lib.cser_norm_apply(self.h, args, ys, stats.data_ptr(), _raw_stream(x)), "cser_norm_apply")
        return out, stats

    def grad(self, x, dy, stats, weight=None, bias=None, step=None, dx=None, dweight=None, dbias=None, need_dx=True, need_params=True,
             stream=None):
        """(dx, dweight, dbias) of sum(dy * apply(x, weight, bias, step)[0]).  dx may be x or dy; dweight and dbias may be views of a flat
        [n, d] gradient."""
        if stream is not None:
            return _on(stream, self.grad, x, dy, stats, weight, bias, step, dx, dweight, dbias, need_dx, need_params)
        args = self._inputs(x, weight, bias, step)
        ds = self._array("dy", dy, x)[1]
        if not (stats.is_cuda and stats.dtype == torch.float32 and stats.shape == (2, self.n, x.shape[1], self.groups) and
                stats.is_contiguous()):
            raise CSERError("GroupNorm: stats must be what apply returned for x")
        xs = None
        if need_dx:
            if dx is None:
                dx = _like(x)
                xs = self._dense(dx, args)
            else:
                xs = self._array("dx", dx, x)[1]
        if need_params:
            if dweight is None:
                dweight = self._new_params(weight, x)
            if dbias is None:
                dbias = self._new_params(bias, x)
            w, w_stride = _params("GroupNorm: dweight", dweight, self.n, self.channels)
            b, b_stride = _params("GroupNorm: dbias", dbias, self.n, self.channels)
        else:
            dweight, dbias, w, w_stride, b, b_stride = None, None, None, 0, None, 0
        _check(_lib.cser_norm_grad(self.h, args, stats.data_ptr(), ds, xs, w, w_stride, b, b_stride, _raw_stream(x)), "cser_norm_grad")
        return dx if need_dx else None, dweight, dbias
