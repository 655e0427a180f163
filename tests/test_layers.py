"""Dropout and group norm (cser_drop_* and cser_norm_* of cser_layers.h) against the formulas in 64 bits and the mask of the oracle's generator.

Tolerances.  u is half a step of the type relative to a value (bf16 2^-8, fp16 2^-11, fp32 2^-24), e = 2^-24, tiny half the spacing of fp16's
smallest numbers (2^-25) or 0.
Dropout: x + bias, the factor and the sum with the residual are each rounded in fp32, then the result in the type:
    u |y| + 4 e (|x| + |bias|) / (1 - p) + 4 e |residual| + tiny;     a sum over rows, in any order: e (rows + 8) sum |dx|
Group norm, with K = 64 roundings in a chain of sums at most, and more where a thread has more pixels than that (`chain`), A the largest
magnitude of a group and s its deviation (with eps): mean and x - mean are off by K e A, so rstd by K e (1 + A / s) of itself, and
    d_xhat = K e (A / s) + K e (1 + A / s) |xhat|,   d_z = |weight| d_xhat + 4 e (|z| + |bias|)
    d_y    = 1.1 d_z + 2^-20 (1 + |z|) |y| + u |y| + tiny       (act's slope is below 1.1; the hardware's exponential: 2^-22 and z's own rounding)
The slope of act is 1.1-Lipschitz, but for relu's within d_z of 0, where it may be 0 or 1:
    d_dz   = |dy| (1.1 d_z + 2^-20 (1 + |z|))  (relu: |dy| where |z| <= d_z)
and sums and products add these up as the formula of dx does; see `Norm`.
"""
import numpy as np
import pytest
import torch

from oracle.philox import philox4x32_10
from paper_2007_13221_b200 import layers
from paper_2007_13221_b200.binding import CSERError

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
U = {BF: 2.0 ** -8, HF: 2.0 ** -11, F32: 2.0 ** -24}
TINY = {BF: 0.0, HF: 2.0 ** -25, F32: 0.0}
E = 2.0 ** -24
SEED, STEP = 0x123456789ABCDEF1, 2 ** 33 + 7


def mask(n, count, p, seed=SEED, step=STEP, site=3, first=0):
    """bool [n, count]: what is kept."""
    q = np.arange((count + 3) // 4, dtype=np.uint64)
    rows = []
    for w in range(first, first + n):
        words = philox4x32_10(seed & 0xFFFFFFFF, seed >> 32, q, step & 0xFFFFFFFF, step >> 32, 4096 * site + w)
        rows.append(np.stack(words, 1).reshape(-1)[:count] >= int(p * 2 ** 32))
    return torch.from_numpy(np.stack(rows)).cuda()


def normal(gen, *size):
    return torch.randn(size, generator=gen, device="cuda")


def gen_of(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def close(got, want, bound):
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), (float((off - bound).max()), float(off.max()))


# ------------------------------------------------------------------ dropout
SIZES = [(1, 1, 1), (1, 1, 4), (2, 1, 3), (1, 3, 8), (3, 5, 7), (2, 33, 64), (4, 1, 1000), (3, 77, 201), (8, 20, 96), (2, 301, 36), (1, 1000, 9),
         (2, 4097, 2), (1, 70, 2056), (5, 64, 520)]


def check_drop(op, x, bias, residual, dy, p, keep, **kw):
    """Both directions of `op` on these arrays against the formula."""
    dt, n = x.dtype, x.shape[0]
    keep = keep.view(x.shape)
    y = op.apply(x, STEP, bias=bias, residual=residual, **kw)
    v = x.double()
    size = x.double().abs()
    if bias is not None:
        b = bias.double().view(n, *([1] * (x.dim() - 2)), -1)
        v, size = v + b, size + b.abs()
    want = torch.where(keep, v / (1 - p), 0.0)
    bound = 4 * E * size / (1 - p)
    if residual is not None:
        want = want + residual.double()
        bound = bound + 4 * E * residual.double().abs()
    assert y.dtype == dt and y.shape == x.shape
    close(y, want, U[dt] * want.abs() * 1.01 + bound + TINY[dt])
    dx, db = op.grad(dy, STEP, need_dbias=bias is not None)
    want = torch.where(keep, dy.double() / (1 - p), 0.0)
    close(dx, want, U[dt] * want.abs() * 1.01 + 4 * E * want.abs() + TINY[dt])
    assert bool((dx[~keep] == 0).all())
    if bias is not None:
        rows = want.view(n, -1, x.shape[-1])
        close(db, rows.sum(1), E * (rows.shape[1] + 8) * rows.abs().sum(1) + 1e-45)
    return y, dx, db


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF, F32], ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_dropout_against_the_formula(size, dtype):
    n, rows, cols = size
    for k, (p, with_bias, with_residual) in enumerate([(0.1, True, True), (0.5, False, True), (0.3, True, False), (0.25, False, False), (0.0, True, True)]):
        gen = gen_of(k)
        x, r, dy = (normal(gen, *size).to(dtype) for _ in range(3))
        bias = normal(gen, n, cols)
        op = layers.Dropout(n, rows, cols, p, SEED, 3, dtype)
        check_drop(op, x, bias if with_bias else None, r if with_residual else None, dy, p, mask(n, rows * cols, p))
        assert op.launches >= 2


@pytest.mark.gpu
def test_masks_are_the_generator_s():
    """Every bit of the mask, at probabilities that differ in their last bits, with both halves of a step and of a seed, and for other workers."""
    n, rows, cols = 3, 11, 65
    x = torch.ones((n, rows, cols), device="cuda")
    for seed, step, site, first, p in ((0, 0, 1, 0, 0.5), (2 ** 64 - 1, 2 ** 64 - 1, 2 ** 20 - 1, 4093, 0.5), (7, 2 ** 32, 5, 17, 2 ** -32),
                                       (7, 1, 5, 17, 1 - 2 ** -32), (7, 1, 5, 17, 0.123456789)):
        op = layers.Dropout(n, rows, cols, p, seed, site, F32, first_worker=first)
        got = op.apply(x, step) != 0
        assert torch.equal(got, mask(n, rows * cols, p, seed, step, site, first).view(x.shape))


@pytest.mark.gpu
def test_masks_do_not_depend_on_how_workers_are_divided():
    n, rows, cols = 6, 40, 130
    x = normal(gen_of(1), n, rows, cols).bfloat16()
    whole = layers.Dropout(n, rows, cols, 0.3, SEED, 2).apply(x, 5)
    for lo, hi in ((0, 1), (1, 4), (4, 6)):
        part = layers.Dropout(hi - lo, rows, cols, 0.3, SEED, 2, first_worker=lo)
        assert torch.equal(part.apply(x[lo:hi], 5), whole[lo:hi])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32], ids=str)
@pytest.mark.parametrize("cols", [64, 36, 33])
def test_dropout_of_strided_arrays_and_flat_parameters(cols, dtype):
    """Columns of wider arrays, rows and workers in either order, parameters inside flat vectors, four dimensions; what lies between is left."""
    n, rows, p = 3, 50, 0.3
    gen = gen_of(cols)
    keep = mask(n, rows * cols, p)
    op = layers.Dropout(n, rows, cols, p, SEED, 3, dtype)
    x, r, dy = (normal(gen, n, rows, cols).to(dtype) for _ in range(3))
    flat = normal(gen, n, cols + 77)
    bias = flat[:, 5:5 + cols]
    want, want_dx, want_db = check_drop(op, x, bias, r, dy, p, keep)

    def inside(t, pad, at, workers_inner=False):
        big = torch.full((rows, n, cols + pad) if workers_inner else (n, rows, cols + pad), 7.0, device="cuda").to(dtype)
        view = big[..., at:at + cols]
        view = view.transpose(0, 1) if workers_inner else view
        view.copy_(t)
        return big, view

    for pad, at, inner in ((8, 8, False), (16, 1, False), (7, 3, True), (64, 0, True)):
        xs, rs, ds = (inside(t, pad, at, inner)[1] for t in (x, r, dy))
        big, out = inside(torch.zeros_like(x), pad, at, inner)
        grads = torch.full((n, cols + 9), 7.0, device="cuda")
        got = op.apply(xs, STEP, bias=bias, residual=rs, out=out)
        dx, db = op.grad(ds, STEP, dbias=grads[:, 4:4 + cols])
        assert got is out and torch.equal(out, want) and torch.equal(dx, want_dx)
        rows_sum = want_dx.double().abs().sum(1)
        close(db, want_db.double(), 2 * E * (rows + 8) * rows_sum + 2 * U[dtype] * rows_sum)
        assert bool((big[..., :at] == 7).all()) and bool((big[..., at + cols:] == 7).all())
        assert bool((grads[:, :4] == 7).all()) and bool((grads[:, 4 + cols:] == 7).all())
    assert torch.equal(op.apply(x.view(n, 5, 10, cols), STEP, bias=bias, residual=r.view(n, 5, 10, cols)), want.view(n, 5, 10, cols))
    spread = x[:1].expand(n, rows, cols)
    assert torch.equal(op.apply(spread, STEP), op.apply(spread.contiguous(), STEP))
    row = dy[:, :1].expand(n, rows, cols)
    assert torch.equal(op.grad(row, STEP, need_dbias=True)[0], op.grad(row.contiguous(), STEP)[0])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF, F32], ids=str)
def test_arrays_that_begin_at_any_element(dtype):
    """All arrays equally far from a 16-byte boundary, and each at another distance."""
    n, rows, cols = 2, 9, 49
    count = n * rows * cols
    gen = gen_of(3)
    op = layers.Dropout(n, rows, cols, 0.3, SEED, 3, dtype)
    x, r = (normal(gen, n, rows, cols).to(dtype) for _ in range(2))
    bias = normal(gen, n, cols)
    want = op.apply(x, STEP, bias=bias, residual=r)
    alone = op.apply(x, STEP)

    def shifted(t, by):
        room = torch.full((count + 24,), 7.0, device="cuda").to(dtype)
        view = room[by:by + count].view(n, rows, cols)
        view.copy_(t)
        return room, view

    for by in range(9):
        for other in (by, (by + 3) % 8):
            room, out = shifted(torch.zeros_like(x), by)
            assert torch.equal(op.apply(shifted(x, by)[1], STEP, bias=bias, residual=shifted(r, other)[1], out=out), want)
            assert bool((room[:by] == 7).all()) and bool((room[by + count:] == 7).all())
            room, out = shifted(torch.zeros_like(x), other)
            assert torch.equal(op.apply(shifted(x, by)[1], STEP, out=out), alone)
            assert bool((room[:other] == 7).all()) and bool((room[other + count:] == 7).all())


@pytest.mark.gpu
def test_dropped_elements_may_be_anything_and_results_may_replace_inputs():
    n, rows, cols = 2, 40, 72
    keep = mask(n, rows * cols, 0.5).view(n, rows, cols)
    gen = gen_of(4)
    x, r, dy = (normal(gen, n, rows, cols).bfloat16() for _ in range(3))
    op = layers.Dropout(n, rows, cols, 0.5, SEED, 3)
    y, (dx, db) = op.apply(x, STEP, residual=r), op.grad(dy, STEP, need_dbias=True)
    for bad in (float("nan"), float("inf"), -float("inf"), 3.3e38):
        spoiled, spoiled_dy = torch.where(keep, x, bad), torch.where(keep, dy, bad)
        assert torch.equal(op.apply(spoiled, STEP, residual=r), y)
        got = op.grad(spoiled_dy, STEP, need_dbias=True)
        assert torch.equal(got[0], dx) and torch.equal(got[1], db)
    into = x.clone()
    assert op.apply(into, STEP, residual=r, out=into) is into and torch.equal(into, y)
    into = r.clone()
    op.apply(x, STEP, residual=into, out=into)
    assert torch.equal(into, y)
    into = dy.clone()
    assert torch.equal(op.grad(into, STEP, dx=into, need_dbias=True)[1], db) and torch.equal(into, dx)
    assert torch.equal(op.grad(dy, STEP, need_dx=False, need_dbias=True)[1], db) and op.grad(dy, STEP, need_dx=False) == (None, None)


@pytest.mark.gpu
def test_dropout_without_rows():
    op = layers.Dropout(2, 4, 10, 0.5, 1, 1)
    none = torch.empty((2, 0, 10), device="cuda", dtype=BF)
    assert op.apply(none, 1).shape == (2, 0, 10)
    db = torch.full((2, 10), 3.0, device="cuda")
    dx, got = op.grad(none, 1, dbias=db)
    assert dx.shape == none.shape and got is db and bool((db == 0).all())


@pytest.mark.gpu
def test_a_replayed_call_draws_anew_with_a_step_on_the_device():
    n, rows, cols = 2, 30, 100
    gen = gen_of(5)
    x, dy = normal(gen, n, rows, cols).bfloat16(), normal(gen, n, rows, cols).bfloat16()
    op = layers.Dropout(n, rows, cols, 0.3, SEED, 3)
    norm = layers.GroupNorm(n, rows, cols, 5, "silu", dropout=op)
    at = torch.zeros(1, dtype=torch.int64, device="cuda")
    y, dx = torch.empty_like(x), torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        op.apply(x, at, out=y)
        op.grad(dy, at, dx=dx, need_dbias=True)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        at += 1
        op.apply(x, at, out=y)
        db = op.grad(dy, at, dx=dx, need_dbias=True)[1]
        z, stats = norm.apply(x.view(n, rows, 1, cols), step=at)
        dz = norm.grad(x.view(n, rows, 1, cols), dy.view(n, rows, 1, cols), stats, step=at)
    for step in (1, 2, 3):
        graph.replay()
        want_dx, want_db = op.grad(dy, step, need_dbias=True)
        assert torch.equal(y, op.apply(x, step)) and torch.equal(dx, want_dx) and torch.equal(db, want_db)
        want, s = norm.apply(x.view(n, rows, 1, cols), step=step)
        assert torch.equal(z, want) and torch.equal(stats, s)
        assert all(torch.equal(a, b) for a, b in zip(dz, norm.grad(x.view(n, rows, 1, cols), dy.view(n, rows, 1, cols), s, step=step)))
    at.fill_(2 ** 63 - 1)                                # the 64 bits as they are
    assert torch.equal(op.apply(x, at), op.apply(x, 2 ** 63 - 1))
    at.fill_(-1)
    assert torch.equal(op.apply(x, at), op.apply(x, 2 ** 64 - 1))


@pytest.mark.gpu
def test_dropout_s_gradient_is_its_difference():
    """Linear in x and in the bias for a fixed mask: <dy, y(x + h) - y(x)> = <dx, h>, in 32 bits."""
    n, rows, cols = 2, 31, 45
    gen = gen_of(6)
    x, h, dy = (normal(gen, n, rows, cols) for _ in range(3))
    bias, hb = normal(gen, n, cols), normal(gen, n, cols)
    op = layers.Dropout(n, rows, cols, 0.4, SEED, 3, F32)
    dx, db = op.grad(dy, 9, need_dbias=True)
    moved = (op.apply(x + h, 9, bias=bias + hb).double() - op.apply(x, 9, bias=bias).double())
    left, right = (moved * dy.double()).sum((1, 2)), (dx.double() * h.double()).sum((1, 2)) + (db.double() * hb.double()).sum(1)
    size = ((x.abs() + h.abs() + 4).double() * dy.abs().double()).sum((1, 2))
    assert bool(((left - right).abs() <= 64 * E * size).all())


# ------------------------------------------------------------------ group norm
class Norm:
    """The formula in 64 bits with how far each result may be off."""

    def __init__(self, x, weight, bias, dy, groups, act, eps, keep, p, chain=0):
        n, b, c = x.shape[0], x.shape[1], x.shape[-1]
        dt, k = x.dtype, (64 + chain) * E
        size = (n, b, -1, groups, c // groups)

        def mean(t):
            return t.mean((2, 4), keepdim=True)

        v = x.double().reshape(size)
        m = None if keep is None else keep.view(v.shape).double() / (1 - p)
        v = v if m is None else v * m
        self.mean, var = mean(v), (v - mean(v)).square().mean((2, 4), keepdim=True)
        std = (var + eps).sqrt()
        hat = (v - self.mean) / std
        a = v.abs().amax((2, 4), keepdim=True) / std
        w = torch.ones((n, 1, 1, groups, c // groups), device="cuda").double() if weight is None else weight.double().view(n, 1, 1, groups, -1)
        o = torch.zeros_like(w) if bias is None else bias.double().view(n, 1, 1, groups, -1)
        z = hat * w + o
        d_hat = k * a + k * (1 + a) * hat.abs()
        d_z = w.abs() * d_hat + 4 * E * (z.abs() + o.abs())
        gate = torch.sigmoid(z)
        approx = 2.0 ** -20 * (1 + z.abs()) if act == "silu" else torch.zeros_like(z)
        y = {"none": z, "relu": z.clamp(min=0), "silu": z * gate}[act]
        self.y = y.reshape(x.shape)
        self.d_y = ((1.1 * d_z + approx * y.abs()) * 1.01 + 1.01 * U[dt] * y.abs() + TINY[dt]).reshape(x.shape)
        self.rstd = 1 / std
        self.d_mean, self.d_rstd = k * a * std, k * (1 + a) / std
        if dy is None:
            return
        g = dy.double().reshape(v.shape)
        slope = {"none": torch.ones_like(z), "relu": (z > 0).double(), "silu": gate * (1 + z * (1 - gate))}[act]
        dz = g * slope
        jump = (z.abs() <= d_z).double() if act == "relu" else 1.1 * d_z + approx if act == "silu" else torch.zeros_like(z)
        d_dz = g.abs() * jump + 4 * E * dz.abs()
        self.db, self.dw = dz.sum((1, 2)).view(n, c), (dz * hat).sum((1, 2)).view(n, c)
        self.d_db = ((d_dz + k * dz.abs()).sum((1, 2))).view(n, c) * 1.01 + 1e-45
        self.d_dw = ((d_dz * hat.abs() + dz.abs() * d_hat + k * (dz * hat).abs()).sum((1, 2))).view(n, c) * 1.01 + 1e-45
        t = dz * w
        d_t = d_dz * w.abs() + 4 * E * t.abs()
        m2 = mean(t * hat)
        dx = (t - mean(t) - hat * m2) / std
        d_m1, d_m2 = mean(d_t + k * t.abs()), mean(d_t * hat.abs() + t.abs() * d_hat + k * (t * hat).abs())
        d_dx = (d_t + d_m1 + hat.abs() * d_m2 + d_hat * (m2.abs() + d_m2) + 4 * E * (t.abs() + mean(t).abs() + (hat * m2).abs())) / std
        d_dx = d_dx * (1 + k * (1 + a)) + k * (1 + a) * dx.abs()
        if m is not None:
            dx, d_dx = dx * m, d_dx * m + 4 * E * (dx * m).abs()
        self.dx = dx.reshape(x.shape)
        self.d_dx = (d_dx * 1.01 + 1.01 * U[dt] * dx.abs() + TINY[dt]).reshape(x.shape)


def check_norm(op, x, weight, bias, dy, groups, act, eps=1e-5, keep=None, p=0.0, chain=0):
    want = Norm(x, weight, bias, dy, groups, act, eps, keep, p, chain)
    y, stats = op.apply(x, weight, bias, step=STEP)
    assert y.dtype == x.dtype and y.shape == x.shape and stats.dtype == F32
    close(stats[0], want.mean.view(stats[0].shape), want.d_mean.view(stats[0].shape))
    close(stats[1], want.rstd.view(stats[0].shape), want.d_rstd.view(stats[0].shape))
    close(y, want.y, want.d_y)
    if dy is None:
        return y, stats
    dx, dw, db = op.grad(x, dy, stats, weight, bias, step=STEP)
    assert dx.dtype == x.dtype and dx.shape == x.shape
    close(dx, want.dx, want.d_dx)
    close(dw, want.dw, want.d_dw)
    close(db, want.db, want.d_db)
    return y, stats, dx, dw, db


def norm_inputs(seed, n, samples, pixels, channels, dtype):
    gen = gen_of(seed)
    shape = (n, samples, *pixels, channels)
    x = (normal(gen, *shape) * (0.5 + torch.rand((channels,), generator=gen, device="cuda")) + normal(gen, channels)).to(dtype)
    return x, normal(gen, n, channels) * 0.3 + 1, normal(gen, n, channels) * 0.3, normal(gen, *shape).to(dtype)


NORMS = [  # n, samples, pixels, channels, groups
    (1, 1, (8, 8), 64, 32), (1, 1, (1,), 32, 4), (2, 3, (1, 1), 512, 1), (1, 2, (5, 3), 8, 8), (3, 5, (13, 9), 60, 12), (2, 4, (7, 7), 96, 32),
    (1, 3, (4, 5), 13, 1), (2, 2, (6, 6), 14, 7), (2, 1, (33,), 1, 1), (8, 2, (16, 16), 32, 8), (1, 1, (56, 56), 40, 4), (2, 7, (2, 2), 1000, 8),
    (1, 1, (65, 64), 24, 3), (4, 16, (3, 5), 20, 5), (1, 2, (30, 31), 320, 32), (1, 1, (100, 101), 128, 4), (3, 1, (2,), 2056, 257)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF, F32], ids=str)
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("size", NORMS, ids=str)
def test_norm_against_the_formula(size, act, dtype):
    n, samples, pixels, c, groups = size
    x, weight, bias, dy = norm_inputs(1, n, samples, pixels, c, dtype)
    op = layers.GroupNorm(n, samples, c, groups, act, dtype=dtype)
    check_norm(op, x, weight, bias, dy, groups, act)
    if act == "silu":
        check_norm(op, x, None, bias, dy, groups, act)
        check_norm(op, x, weight, None, dy, groups, act)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF, F32], ids=str)
@pytest.mark.parametrize("size", NORMS, ids=str)
def test_norm_of_a_dropout(size, dtype):
    """Against the formula with the oracle's mask, and the mask against the dropout's own."""
    n, samples, pixels, c, groups = size
    x, weight, bias, dy = norm_inputs(2, n, samples, pixels, c, dtype)
    p, rows = 0.3, samples * int(np.prod(pixels))
    drop = layers.Dropout(n, rows, c, p, SEED, 3, dtype)
    op = layers.GroupNorm(n, samples, c, groups, "silu", dtype=dtype, dropout=drop)
    drop.close()
    keep = mask(n, rows * c, p).view(x.shape)
    got = check_norm(op, x, weight, bias, dy, groups, "silu", keep=keep, p=p)
    assert bool((got[2][~keep] == 0).all())
    spoiled = torch.where(keep, x, float("nan"))
    assert torch.equal(op.apply(spoiled, weight, bias, step=STEP)[0], got[0])
    assert torch.equal(op.grad(spoiled, dy, got[1], weight, bias, step=STEP)[0], got[2])


@pytest.mark.gpu
def test_a_mean_far_from_zero_keeps_the_variance():
    """Values 1e4 deviations from 0 in 32 bits: sums of squares would lose all of it."""
    gen = gen_of(7)
    for pixels in ((8, 8), (60, 60)):
        x = normal(gen, 2, 3, *pixels, 64) + 1e4
        check_norm(layers.GroupNorm(2, 3, 64, 8, "silu", dtype=F32), x, None, None, normal(gen, *x.shape), 8, "silu")
        x[:, :, 0, 0] = 3e6                              # and where the first pixel is far from the others
        check_norm(layers.GroupNorm(2, 3, 64, 8, "none", dtype=F32), x, None, None, normal(gen, *x.shape), 8, "none")


@pytest.mark.gpu
def test_groups_of_equal_values_and_spoiled_groups():
    gen = gen_of(8)
    x, weight, bias, dy = norm_inputs(3, 2, 3, (6, 6), 48, BF)
    x[0, 1, :, :, 8:16] = 2.5                            # one group without variance
    op = layers.GroupNorm(2, 3, 48, 6, "relu")
    y, stats, dx, dw, db = check_norm(op, x, weight, bias, dy, 6, "relu")
    assert float(stats[1, 0, 1, 1]) == pytest.approx(1e-5 ** -0.5, rel=1e-6)
    for bad in (float("nan"), float("inf")):
        z = x.clone()
        z[1, 2, 3, 3, 20] = bad
        y2, s2 = op.apply(z, weight, bias)
        g2 = op.grad(z, dy, s2, weight, bias)
        clean = torch.ones_like(x, dtype=torch.bool)
        clean[1, 2, :, :, 16:24] = False
        assert torch.equal(y2[clean], y[clean]) and torch.equal(g2[0][clean], dx[clean])
        assert not bool(y2[1, 2, 3, 3, 20].isfinite()) and not bool(g2[0][1, 2, :, :, 16:24].isfinite().any())
        assert torch.equal(g2[1][0], dw[0]) and torch.equal(g2[1][1, 24:], dw[1, 24:]) and torch.equal(g2[2][1, :16], db[1, :16])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32], ids=str)
def test_norm_of_strided_arrays_and_flat_parameters(dtype):
    """Channels of wider arrays, any order of workers and samples, parameters and their gradients inside flat vectors, results in place."""
    n, b, h, w, c, groups = 2, 3, 6, 5, 48, 6
    x, weight, bias, dy = norm_inputs(4, n, b, (h, w), c, dtype)
    op = layers.GroupNorm(n, b, c, groups, "silu", dtype=dtype)
    want = check_norm(op, x, weight, bias, dy, groups, "silu")
    for pad, at in ((16, 8), (7, 3), (4, 4)):
        big = torch.full((b, n, h, w, c + pad), 7.0, device="cuda").to(dtype)
        gap = torch.full((n, b, h, w, c + pad), 7.0, device="cuda").to(dtype)
        xs, out = big[..., at:at + c].transpose(0, 1), gap[..., at:at + c]
        xs.copy_(x)
        state = torch.full((n, 400), 7.0, device="cuda")
        ws, bs = state[:, 31:31 + c], state[:, 101:101 + c]
        ws.copy_(weight), bs.copy_(bias)
        grads = torch.full((n, 400), 7.0, device="cuda")
        y, stats = op.apply(xs, ws, bs, out=out)
        close(y, want[0].double(), 2 * U[dtype] * want[0].double().abs() + 1e-5 * (1 + want[0].double().abs()))
        got = op.grad(xs, dy, stats, ws, bs, dx=out, dweight=grads[:, 31:31 + c], dbias=grads[:, 101:101 + c])
        check = Norm(x, weight, bias, dy, groups, "silu", 1e-5, None, 0.0)
        close(got[0], check.dx, check.d_dx), close(got[1], check.dw, check.d_dw), close(got[2], check.db, check.d_db)
        assert bool((gap[..., :at] == 7).all()) and bool((gap[..., at + c:] == 7).all())
        used = torch.zeros(400, dtype=torch.bool, device="cuda")
        used[31:31 + c], used[101:101 + c] = True, True
        assert bool((grads[:, ~used] == 7).all())
    shared = weight[:1].expand(n, c)                     # one weight for all workers
    assert torch.equal(op.apply(x, shared, bias)[0], op.apply(x, shared.contiguous(), bias)[0])
    flat = torch.ones((n, 1, 1, 1, 1), device="cuda").to(dtype).expand(n, b, h, w, c)
    with pytest.raises(CSERError, match="contiguous"):
        op.grad(x, flat, want[1], weight, bias)          # the upstream gradient of a sum has no contiguous dimension
    ones = torch.ones((n, b, 1, 1, c), device="cuda").to(dtype).expand(n, b, h, w, c)
    got, plain = op.grad(x, ones, want[1], weight, bias), op.grad(x, ones.contiguous(), want[1], weight, bias)
    assert all(torch.equal(p, q) for p, q in zip(got, plain))
    into = x.clone()
    assert op.apply(into, weight, bias, out=into)[0] is into and torch.equal(into, want[0])
    for which in (0, 1):
        ax, ad = x.clone(), dy.clone()
        assert torch.equal(op.grad(ax, ad, want[1], weight, bias, dx=(ax, ad)[which])[0], want[2])


@pytest.mark.gpu
def test_parts_of_the_gradient_alone():
    x, weight, bias, dy = norm_inputs(5, 2, 3, (9, 9), 40, BF)
    op = layers.GroupNorm(2, 3, 40, 5, "silu")
    y, stats = op.apply(x, weight, bias)
    dx, dw, db = op.grad(x, dy, stats, weight, bias)
    a = op.grad(x, dy, stats, weight, bias, need_params=False)
    b = op.grad(x, dy, stats, weight, bias, need_dx=False)
    assert torch.equal(a[0], dx) and a[1:] == (None, None) and b[0] is None and torch.equal(b[1], dw) and torch.equal(b[2], db)


@pytest.mark.gpu
def test_norm_without_samples_or_pixels():
    op = layers.GroupNorm(2, 4, 24, 3)
    none = torch.empty((2, 0, 5, 24), device="cuda", dtype=BF)
    y, stats = op.apply(none)
    assert y.shape == none.shape and stats.shape == (2, 2, 0, 3)
    assert all(bool((g == 0).all()) for g in op.grad(none, none, stats)[1:])
    none = torch.empty((2, 3, 0, 24), device="cuda", dtype=BF)
    y, stats = op.apply(none)
    assert y.shape == none.shape and bool((stats == 0).all())
    assert all(bool((g == 0).all()) for g in op.grad(none, none, stats)[1:])


@pytest.mark.gpu
def test_fewer_samples_than_the_handle_is_for():
    op = layers.GroupNorm(3, 20, 64, 16, "silu")
    for samples in (20, 1, 7):
        x, weight, bias, dy = norm_inputs(6 + samples, 3, samples, (5, 5), 64, BF)
        check_norm(op, x, weight, bias, dy, 16, "silu")


@pytest.mark.gpu
def test_norm_s_gradient_is_its_difference():
    """Central differences of <dy, y> in 32 bits along random directions of x, weight and bias: h = 2^-7 leaves h^2 of the third derivative
    and 2^-24 / h of the values."""
    n, b, h, w, c, groups = 2, 2, 5, 7, 24, 6
    for act in ("none", "silu"):
        x, weight, bias, dy = norm_inputs(9, n, b, (h, w), c, F32)
        op = layers.GroupNorm(n, b, c, groups, act, dtype=F32)
        dx, dw, db = op.grad(x, dy, op.apply(x, weight, bias)[1], weight, bias)
        gen = gen_of(10)
        for k in range(3):
            t = 2.0 ** -7
            move = [normal(gen, *a.shape) if k == j else torch.zeros_like(a) for j, a in enumerate((x, weight, bias))]
            up, down = (op.apply(x + s * t * move[0], weight + s * t * move[1], bias + s * t * move[2])[0].double() for s in (1, -1))
            left = ((up - down) * dy.double()).sum() / (2 * t)
            right = sum((g.double() * m.double()).sum() for g, m in zip((dx, dw, db), move))
            size = float((dy.double().abs() * (1 + up.abs())).sum())
            assert abs(float(left - right)) <= size * (8 * t * t + 8 * E / t), (act, k)


# ------------------------------------------------------------------ refusals
@pytest.mark.parametrize("args", [(0, 1, 1, 0.5, 1), (1, 0, 1, 0.5, 1), (1, 1, 0, 0.5, 1), (1, 1, 1, 1.0, 1), (1, 1, 1, -0.1, 1), (1, 1, 1, float("nan"), 1),
                                  (1, 1, 1, 0.5, 0), (1, 1, 1, 0.5, 2 ** 20), (4097, 1, 1, 0.5, 1), (1, 2 ** 33, 3, 0.5, 1), (1, 1, 1, 0.5, -1)], ids=str)
def test_dropout_refuses(args):
    n, rows, cols, p, site = args
    with pytest.raises(CSERError):
        layers.Dropout(n, rows, cols, p, 0, site)


def test_handles_refuse_other_arguments():
    with pytest.raises(CSERError, match="types"):
        layers.Dropout(1, 1, 1, 0.5, 0, 1, torch.float64)
    with pytest.raises(CSERError, match="first_worker"):
        layers.Dropout(2, 1, 1, 0.5, 0, 1, first_worker=4095)
    for args in ((0, 1, 8, 2), (1, 0, 8, 2), (1, 1, 8, 3), (1, 1, 0, 1), (1, 1, 8, 0), (1, 1, 65544, 8), (2 ** 13, 2 ** 12, 8, 2)):
        with pytest.raises(CSERError):
            layers.GroupNorm(*args)
    for kw in (dict(eps=-1.0), dict(eps=float("inf")), dict(eps=float("nan")), dict(activation="tanh"), dict(dtype=torch.int8)):
        with pytest.raises(CSERError):
            layers.GroupNorm(1, 1, 8, 2, **kw)


@pytest.mark.gpu
def test_calls_refuse_what_they_cannot_take():
    op = layers.Dropout(2, 10, 16, 0.5, 0, 1)
    x = torch.zeros((2, 10, 16), device="cuda", dtype=BF)
    bias = torch.zeros((2, 16), device="cuda")
    for call in (lambda: op.apply(x.float(), 0), lambda: op.apply(x.cpu(), 0), lambda: op.apply(x[:1], 0), lambda: op.apply(x[..., :8], 0),
                 lambda: op.apply(torch.zeros((2, 11, 16), device="cuda", dtype=BF), 0), lambda: op.apply(x.transpose(1, 2), 0),
                 lambda: op.apply(x, 0, bias=bias.bfloat16()), lambda: op.apply(x, 0, bias=bias[:1]), lambda: op.apply(x, 0, residual=x[:, :5]),
                 lambda: op.apply(x, 0, out=x[:1].expand(2, 10, 16)), lambda: op.apply(x, 0, out=x[:, :1].expand(2, 10, 16)),
                 lambda: op.apply(x, torch.zeros(2, dtype=torch.int64, device="cuda")), lambda: op.apply(x, torch.zeros(1, dtype=torch.int64)),
                 lambda: op.grad(x, 0, dbias=bias[:1].expand(2, 16)), lambda: op.grad(x, 0, dx=x[:, :5])):
        with pytest.raises(CSERError):
            call()
    norm = layers.GroupNorm(2, 3, 16, 4)
    x = torch.zeros((2, 3, 5, 5, 16), device="cuda", dtype=BF)
    y, stats = norm.apply(x)
    for call in (lambda: norm.apply(x.half()), lambda: norm.apply(x[:1]), lambda: norm.apply(x[..., :8]), lambda: norm.apply(x, weight=bias.half()),
                 lambda: norm.apply(torch.zeros((2, 4, 5, 5, 16), device="cuda", dtype=BF)), lambda: norm.apply(x.permute(0, 1, 4, 2, 3)),
                 lambda: norm.apply(torch.zeros((2, 3, 5, 8, 16), device="cuda", dtype=BF)[:, :, :, :5]),
                 lambda: norm.apply(x, out=x[:1].expand(2, 3, 5, 5, 16)), lambda: norm.grad(x, x[:, :2], stats), lambda: norm.grad(x, x, stats[:1]),
                 lambda: norm.grad(x, x, stats, dx=x[:, :1].expand(2, 3, 5, 5, 16)), lambda: norm.grad(x, x, stats, dweight=bias[:1].expand(2, 16)),
                 lambda: layers.GroupNorm(2, 3, 16, 4, dropout=layers.Dropout(2, 10, 8, 0.5, 0, 1)),
                 lambda: layers.GroupNorm(2, 3, 16, 4, dropout=layers.Dropout(1, 10, 16, 0.5, 0, 1)),
                 lambda: layers.GroupNorm(2, 3, 16, 4, dropout=layers.Dropout(2, 10, 16, 0.5, 0, 1, F32))):
        with pytest.raises(CSERError):
            call()
    op.close()
    with pytest.raises(CSERError):
        layers.GroupNorm(2, 3, 16, 4, dropout=op)
    with pytest.raises(CSERError, match="NULL handle"):
        op.apply(torch.zeros((2, 10, 16), device="cuda", dtype=BF), 0)
