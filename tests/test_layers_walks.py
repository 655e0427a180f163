"""Group norm of samples that fit no cluster: the kernels for moments, join and result, and for the gradient's sums, join and result, at every vector
length, with several chunks of pixels and several blocks of columns.

Groups of more than 128 vectors reach them at few pixels; that it is they is seen from the number of kernels, 3 forward and 4 for the gradient
(the fourth adds up the workers' dweight and dbias).  Formulas and bounds are those of test_layers.
"""
import pytest
import torch
from test_layers import BF, F32, HF, SEED, STEP, Norm, check_norm, close, mask, norm_inputs

from paper_2007_13221_b200 import layers

pytestmark = pytest.mark.gpu

# channels of a group, type: 130 vectors of 8, 129 of 4 and of 2 16-bit elements; of 4, 2 and 1 32-bit ones
VECTORS = [(1040, BF), (1040, HF), (516, BF), (516, HF), (258, BF), (258, HF), (516, F32), (258, F32), (129, F32)]


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("wide", VECTORS, ids=str)
def test_wide_groups_in_several_walks(wide, act):
    """Ten chunks of 30 pixels; two groups."""
    c, dtype = wide
    n, b, pixels, groups = 2, 2, 300, 2
    x, weight, bias, dy = norm_inputs(1, n, b, (pixels,), c * groups, dtype)
    op = layers.GroupNorm(n, b, c * groups, groups, act, dtype=dtype)
    got = check_norm(op, x, weight, bias, dy, groups, act)
    assert op.launches == 3 + 4
    if act == "silu":
        check_norm(op, x, None, None, dy, groups, act)
        again = op.grad(x, dy, got[1], weight, bias)
        assert torch.equal(op.apply(x, weight, bias)[0], got[0]) and all(torch.equal(p, q) for p, q in zip(again, got[2:]))
        into, at = x.clone(), dy.clone()
        assert torch.equal(op.apply(into, weight, bias, out=into)[0], got[0])
        assert torch.equal(op.grad(x, at, got[1], weight, bias, dx=at)[0], got[2])
        assert torch.equal(op.grad(x, dy, got[1], weight, bias, need_params=False)[0], got[2])
        only = op.grad(x, dy, got[1], weight, bias, need_dx=False)
        assert torch.equal(only[1], got[3]) and torch.equal(only[2], got[4])


@pytest.mark.parametrize("wide", VECTORS, ids=str)
def test_wide_groups_of_a_dropout_in_several_walks(wide):
    c, dtype = wide
    n, b, pixels, p = 2, 3, 77, 0.3
    x, weight, bias, dy = norm_inputs(2, n, b, (pixels,), c, dtype)
    drop = layers.Dropout(n, b * pixels, c, p, SEED, 3, dtype)
    op = layers.GroupNorm(n, b, c, 1, "silu", dtype=dtype, dropout=drop)
    keep = mask(n, b * pixels * c, p).view(x.shape)
    got = check_norm(op, x, weight, bias, dy, 1, "silu", keep=keep, p=p)
    assert op.launches == 3 + 4 and bool((got[2][~keep] == 0).all())
    spoiled = torch.where(keep, x, float("nan"))
    assert torch.equal(op.apply(spoiled, weight, bias, step=STEP)[0], got[0])
    assert torch.equal(op.grad(spoiled, dy, got[1], weight, bias, step=STEP)[0], got[2])


@pytest.mark.parametrize("wide", [(1040, BF), (516, HF), (258, BF), (516, F32), (129, F32)], ids=str)
def test_threads_of_more_pixels_than_are_joined_at_a_time(wide):
    """Two chunks of 400 pixels, 50 a thread: its moments are joined after 32."""
    c, dtype = wide
    n, b, pixels = 2, 148, 800
    if c > 1000:
        n, b, pixels = 1, 296, 530
    x, weight, bias, dy = norm_inputs(3, n, b, (pixels,), c, dtype)
    x[:, :, 0] += 30                                     # and the first of them is far from the others
    op = layers.GroupNorm(n, b, c, 1, "silu", dtype=dtype)
    check_norm(op, x, weight, bias, dy, 1, "silu", chain=64)
    assert op.launches == 3 + 4


@pytest.mark.parametrize("size", [(1, 1, (120, 1001), 8, 1, BF), (1, 2, (444, 444), 6, 3, HF), (2, 1, (150000,), 4, 2, F32)], ids=str)
def test_large_images_of_few_channels(size):
    """One block of columns, 4 pixels a thread, many chunks, groups narrower than a vector."""
    n, b, pixels, c, groups, dtype = size
    x, weight, bias, dy = norm_inputs(4, n, b, pixels, c, dtype)
    for act in ("none", "silu"):
        op = layers.GroupNorm(n, b, c, groups, act, dtype=dtype)
        check_norm(op, x, weight, bias, dy, groups, act, chain=64)
        assert op.launches == 3 + 4


def test_strided_arrays_in_several_walks():
    """Whole vectors at other strides, parameters inside flat vectors; what lies between is left as it was."""
    n, b, pixels, c, dtype = 2, 3, 65, 1040, BF
    x, weight, bias, dy = norm_inputs(5, n, b, (pixels,), c, dtype)
    op = layers.GroupNorm(n, b, c, 1, "silu", dtype=dtype)
    want = check_norm(op, x, weight, bias, dy, 1, "silu")
    for pad, at in ((16, 8), (4, 4), (3, 1)):            # vectors of 8, 4 and 1
        wide = torch.full((b, n, pixels, c + pad), 7.0, device="cuda").to(dtype)
        gap = torch.full((n, b, pixels, c + pad), 7.0, device="cuda").to(dtype)
        xs, out = wide[..., at:at + c].transpose(0, 1), gap[..., at:at + c]
        xs.copy_(x)
        state, grads = torch.full((n, 2400), 7.0, device="cuda"), torch.full((n, 2400), 7.0, device="cuda")
        ws, bs = state[:, 31:31 + c], state[:, 1101:1101 + c]
        ws.copy_(weight), bs.copy_(bias)
        check = Norm(x, weight, bias, dy, 1, "silu", 1e-5, None, 0.0)
        y, stats = op.apply(xs, ws, bs, out=out)
        close(y, check.y, check.d_y)
        got = op.grad(xs, dy, stats, ws, bs, dx=out, dweight=grads[:, 31:31 + c], dbias=grads[:, 1101:1101 + c])
        close(got[0], check.dx, check.d_dx), close(got[1], check.dw, check.d_dw), close(got[2], check.db, check.d_db)
        assert bool((gap[..., :at] == 7).all()) and bool((gap[..., at + c:] == 7).all())
        used = torch.zeros(2400, dtype=torch.bool, device="cuda")
        used[31:31 + c], used[1101:1101 + c] = True, True
        assert bool((grads[:, ~used] == 7).all())
    assert torch.equal(op.apply(x, weight, bias)[0], want[0])


def test_an_infinity_spoils_its_group_alone():
    x, weight, bias, dy = norm_inputs(6, 1, 2, (90,), 1040 * 2, BF)
    op = layers.GroupNorm(1, 2, 1040 * 2, 2, "silu", dtype=BF)
    y, stats = op.apply(x, weight, bias)
    dx = op.grad(x, dy, stats, weight, bias)[0]
    for bad in (float("inf"), float("nan")):
        z = x.clone()
        z[0, 1, 50, 1500] = bad
        y2, s2 = op.apply(z, weight, bias)
        dx2 = op.grad(z, dy, s2, weight, bias)[0]
        clean = torch.ones_like(x, dtype=torch.bool)
        clean[0, 1, :, 1040:] = False
        assert torch.equal(y2[clean], y[clean]) and torch.equal(dx2[clean], dx[clean])
        assert not bool(y2[0, 1, :, 1040:].isfinite().any()) and not bool(dx2[0, 1, :, 1040:].isfinite().any())
