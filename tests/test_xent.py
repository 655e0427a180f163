"""Linear cross entropy (cser_xent_* of cser_train.h) against the formula in 64 bits, and its gradient against differences.

Tolerances.  loss and lse: logits are sums of exact products in fp32 whose partial sums are truncated, at most
2^-23 * dim / 16 of the sum of magnitudes, and the sum of exponentials adds a few 2^-24: 1e-5 of 1 + |value| is allowed.
Gradients: dz and the result are each rounded to the type, by u = 2^-8 (bf16) or 2^-11 (fp16) of a value at most.  In the
2-norm over all, where the two are independent: u * sqrt(2) * 1.1.  For every entry, where terms may cancel, the sum of
    u |dz|                              rounding of dz, times |W| (or |h|), summed
    2e-5 (1 + |lse|) p |dloss|          what the tolerance of z and lse above makes of p, likewise
    2^-37 max |dloss|                   half the spacing of fp16's smallest numbers, 2^12 under dz, likewise
    u |result| + 2^-25 (fp16)           rounding of the result, and half that spacing
and a tenth more for the products of these.
"""
import pytest
import torch

from paper_2007_13221_b200 import train
from paper_2007_13221_b200.binding import CSERError

BF, HF = torch.bfloat16, torch.float16
GRAD = {BF: 2.0 ** -8 * 1.56, HF: 2.0 ** -11 * 1.56}
IGN = -100


def exact(h, w, y, dloss, ignore=IGN):
    """loss, lse, dhidden, dweight in float64, one worker after the other, and how far each entry of the gradients
    may be off."""
    loss, lse, dh, dw, bh, bw = [], [], [], [], [], []
    for i in range(h.shape[0]):
        hi, wi = h[i].double(), w[i].double()
        z = hi @ wi.t()
        l = torch.logsumexp(z, 1)
        ok = y[i] != ignore
        at = torch.where(ok, y[i], 0)
        loss.append(torch.where(ok, l - z.gather(1, at[:, None])[:, 0], 0.0))
        lse.append(l)
        dz = torch.exp(z - l[:, None])
        dz[torch.arange(len(at), device=z.device), at] -= 1
        dz *= (dloss[i].double() * ok)[:, None]
        dh.append(dz @ wi)
        dw.append(dz.t() @ hi)
        u, tiny = (2.0 ** -8, 0.0) if h.dtype == BF else (2.0 ** -11, 2.0 ** -25)
        g = (dloss[i].double().abs() * ok)[:, None]
        off = u * dz.abs() + 2e-5 * (1 + l.abs())[:, None] * torch.exp(z - l[:, None]) * g + 2.0 ** -37 * g.max()
        bh.append(1.1 * (off @ wi.abs() + u * dh[-1].abs() + tiny))
        bw.append(1.1 * (off.t() @ hi.abs() + u * dw[-1].abs() + tiny))
    return tuple(map(torch.stack, (loss, lse, dh, dw, bh, bw)))


def inputs(n, t, v, d, dtype, seed=0, ignored=0.2, spread=2.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 1000003 * t + 7919 * v + d)
    h = torch.randn((n, t, d), generator=gen, device="cuda")
    w = (torch.randn((n, v, d), generator=gen, device="cuda") * spread / d ** 0.5).to(dtype)
    y = torch.randint(0, v, (n, t), generator=gen, device="cuda")
    h = (h + 1.5 * torch.stack([w[i][y[i]].float() for i in range(n)])).to(dtype)
    y = torch.where(torch.rand((n, t), generator=gen, device="cuda") < ignored, IGN, y)
    dloss = torch.randn((n, t), generator=gen, device="cuda")
    return h, w, y, dloss


def far(got, want):
    scale = want.norm()
    return float((got.double() - want).norm() / scale) if scale else float(got.double().abs().max())


def check(op, h, w, y, dloss, dtype, **kw):
    loss, lse = op.loss(h, w, y, **kw)
    dh, dw = op.grad(h, w, y, lse, dloss, **kw)
    e_loss, e_lse, e_dh, e_dw, b_dh, b_dw = exact(h, w, y, dloss, **({"ignore": kw["ignore_index"]} if kw else {}))
    assert loss.dtype == lse.dtype == torch.float32 and dh.dtype == dw.dtype == dtype
    assert bool(((loss.double() - e_loss).abs() <= 1e-5 * (1 + e_lse.abs())).all())
    assert bool(((lse.double() - e_lse).abs() <= 1e-5 * (1 + e_lse.abs())).all())
    assert far(dh, e_dh) < GRAD[dtype] and far(dw, e_dw) < GRAD[dtype]
    for got, want, bound in ((dh, e_dh, b_dh), (dw, e_dw, b_dw)):
        assert bool(((got.double() - want).abs() <= bound).all())
    return loss, lse, dh, dw


SIZES = [  # n, tokens, vocab, dim
    (1, 1, 1, 1), (1, 1, 2, 8), (2, 3, 5, 7), (1, 1, 1000, 64), (1, 7, 257, 64), (3, 64, 256, 128), (1, 128, 512, 256), (1, 129, 513, 65),
    (2, 127, 255, 200), (1, 300, 2000, 72), (2, 77, 1003, 201), (1, 16, 5000, 264), (8, 5, 700, 96), (1, 513, 1100, 520), (1, 1000, 300, 1032)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF], ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_against_the_formula(size, dtype):
    n, t, v, d = size
    h, w, y, dloss = inputs(n, t, v, d, dtype)
    op = train.LinearCrossEntropy(n, t, v, d, dtype)
    check(op, h, w, y, dloss, dtype)
    assert op.launches >= 3                           # loss, dz, the gradients


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF], ids=str)
@pytest.mark.parametrize("size", [(1, 1, 134, 279), (4, 1, 1000, 64), (1, 17, 700, 520), (2, 31, 2000, 136), (1, 32, 5000, 264)], ids=str)
def test_few_tokens_round_once(size, dtype):
    """Up to 32 tokens dz keeps what its rounding left: u^2 |dz| in place of u |dz|, and the truncation of the products'
    partial sums, 2^-23 of the sum of magnitudes for each of two per 16 of the inner dimension, no longer vanishes beside it."""
    n, t, v, d = size
    h, w, y, dloss = inputs(n, t, v, d, dtype)
    op = train.LinearCrossEntropy(n, 40, v, d, dtype)
    loss, lse, dh, dw = check(op, h, w, y, dloss, dtype)
    u, tiny = (2.0 ** -8, 0.0) if dtype == BF else (2.0 ** -11, 2.0 ** -25)
    for i in range(n):
        hi, wi = h[i].double(), w[i].double()
        ok = y[i] != IGN
        z = hi @ wi.t()
        l = torch.logsumexp(z, 1)[:, None]
        p = torch.exp(z - l)
        dz = p.clone()
        dz[torch.arange(t, device="cuda"), torch.where(ok, y[i], 0)] -= 1
        g = (dloss[i].double() * ok)[:, None]
        dz *= g
        off = 2e-5 * (1 + l.abs()) * p * g.abs() + 2.0 ** -37 * g.abs().max()
        for got, mine, other, of in ((dh[i], dz, wi, off), (dw[i], dz.t(), hi, off.t())):
            sums = 2.0 ** -23 * 2 * (mine.shape[1] // 16 + 1)
            want = mine @ other
            bound = 1.1 * ((of + (u * u + sums) * mine.abs()) @ other.abs() + u * want.abs() + tiny)
            assert bool(((got.double() - want).abs() <= bound).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF], ids=str)
@pytest.mark.parametrize("piece", [1, 256, 512, 1024])
def test_pieces_of_the_vocabulary(piece, dtype):
    n, t, v, d = 2, 200, 1700, 136
    h, w, y, dloss = inputs(n, t, v, d, dtype)
    check(train.LinearCrossEntropy(n, t, v, d, dtype, piece=piece), h, w, y, dloss, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("piece", [1700, 1701, 2 ** 40, 2 ** 63 - 1])
def test_pieces_longer_than_the_vocabulary(piece):
    n, t, v, d = 2, 200, 1700, 136
    h, w, y, dloss = inputs(n, t, v, d, BF)
    got = check(train.LinearCrossEntropy(n, t, v, d, BF, piece=piece), h, w, y, dloss, BF)
    want = check(train.LinearCrossEntropy(n, t, v, d, BF), h, w, y, dloss, BF)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF], ids=str)
@pytest.mark.parametrize("size", [  # n, tokens, vocab, dim, piece: the last piece has 1, 2, 3, 4 stages of 64 or one more than shares
    (1, 10, 2049, 64, 2048), (1, 10, 2100, 64, 2048), (1, 10, 2048 + 65, 72, 2048), (2, 40, 4096 + 129, 64, 2048), (1, 10, 2048 + 256, 64, 2048),
    (1, 10, 2048 + 257, 64, 2048), (1, 200, 2049, 64, 2048), (2, 300, 2048 + 129, 264, 2048), (1, 130, 4096 + 193, 201, 2048),
    (8, 16, 65600, 64, 0), (1, 1200, 104800, 200, 0)], ids=str)
def test_a_last_piece_shorter_than_the_shares_of_the_others(size, dtype):
    """dh's inner dimension is summed in shares where it has few tiles; every share has a stage, in the last piece too."""
    n, t, v, d, piece = size
    h, w, y, dloss = inputs(n, t, v, d, dtype)
    op = train.LinearCrossEntropy(n, t, v, d, dtype, piece=piece)
    loss, lse, dh, _ = check(op, h, w, y, dloss, dtype)
    assert torch.equal(op.grad(h, w, y, lse, dloss, need_dweight=False)[0], dh)


@pytest.mark.gpu
def test_fewer_tokens_than_the_handle_was_made_for():
    n, v, d = 2, 900, 160
    op = train.LinearCrossEntropy(n, 700, v, d, BF)
    for t in (700, 1, 130, 0, 256, 700):
        h, w, y, dloss = inputs(n, t, v, d, BF)
        if t:
            check(op, h, w, y, dloss, BF)
        else:
            loss, lse = op.loss(h, w, y)
            dh, dw = op.grad(h, w, y, lse, dloss, dweight=torch.ones_like(w))
            assert loss.numel() == lse.numel() == dh.numel() == 0 and bool((dw == 0).all())


@pytest.mark.gpu
def test_a_mean_over_the_tokens_is_not_rounded_twice():
    """Uniform dloss = 1/3 (not representable): the same bits as dloss = 1 gives, scaled."""
    h, w, y, _ = inputs(1, 150, 600, 128, BF)
    op = train.LinearCrossEntropy(1, 150, 600, 128, BF)
    _, lse = op.loss(h, w, y)
    ones = torch.ones((1, 150), device="cuda")
    a = op.grad(h, w, y, lse, ones / 4)
    b = op.grad(h, w, y, lse, ones)
    for p, q in zip(a, b):
        assert torch.equal(p * 4, q)
    check(op, h, w, y, ones / 3, BF)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF], ids=str)
@pytest.mark.parametrize("size", [(1, 150, 600, 128), (2, 300, 700, 264), (1, 4096, 1000, 64)], ids=str)
def test_a_uniform_dloss_adds_no_rounding(size, dtype):
    """dz is that of dloss = 1 whatever dloss is: three times the result for 1/3 differs from the result for 1 by the roundings of
    these two results, u each, alone.  Were p / 3 rounded itself, entries whose terms cancel would be off by u of the terms."""
    n, t, v, d = size
    h, w, y, _ = inputs(n, t, v, d, dtype)
    op = train.LinearCrossEntropy(n, t, v, d, dtype)
    _, lse = op.loss(h, w, y)
    ones = torch.ones((n, t), device="cuda")
    third, whole = op.grad(h, w, y, lse, ones / 3), op.grad(h, w, y, lse, ones)
    u, tiny = (2.0 ** -8, 0.0) if dtype == BF else (2.0 ** -11, 2.0 ** -25)
    for a, b in zip(third, whole):
        a, b = a.double(), b.double()
        assert bool(((3 * a - b).abs() <= 2.02 * u * b.abs() + 4 * tiny).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF], ids=str)
def test_ignored_tokens_other_indices_and_targets_out_of_range(dtype):
    n, t, v, d = 2, 90, 400, 64
    h, w, y, dloss = inputs(n, t, v, d, dtype, ignored=0.0)
    op = train.LinearCrossEntropy(n, t, v, d, dtype)
    y[:, ::3] = 7                                     # an index inside the vocabulary can be the one that is ignored
    loss, _, dh, dw = check(op, h, w, y, dloss, dtype, ignore_index=7)
    assert bool((loss[y == 7] == 0).all()) and bool((dh[y == 7] == 0).all())
    none = torch.full_like(y, IGN)                    # nothing left to learn from
    loss, lse = op.loss(h, w, none)
    dh, dw = op.grad(h, w, none, lse, dloss)
    assert bool((loss == 0).all()) and bool((dh == 0).all()) and bool((dw == 0).all())
    bad = y.clone()
    bad[1, 5], bad[1, 6] = v, -1
    loss, lse = op.loss(h, w, bad)
    dh, dw = op.grad(h, w, bad, lse, dloss)
    assert loss.isnan().nonzero().tolist() == [[1, 5], [1, 6]] and bool(lse.isfinite().all())
    assert bool(dh[1, 5:7].isnan().all()) and bool(dh[0].isfinite().all()) and bool(dw[0].isfinite().all()) and bool(dw[1].isnan().any())
    zero = torch.zeros_like(dloss)
    dh, dw = op.grad(h, w, y, lse, zero)
    assert bool((dh == 0).all()) and bool((dw == 0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF], ids=str)
@pytest.mark.parametrize("size", [(2, 20, 300, 64), (2, 90, 700, 72), (2, 300, 700, 201)], ids=str)
def test_a_dloss_that_is_not_finite_stays_in_its_row(size, dtype):
    """Its token's row of dhidden and its worker's dweight; tokens that do not count have no dloss."""
    n, t, v, d = size
    h, w, y, dloss = inputs(n, t, v, d, dtype)
    op = train.LinearCrossEntropy(n, t, v, d, dtype)
    loss, lse = op.loss(h, w, y)
    y[:, 4:8] = 1
    y[:, 9], y[:, 12] = IGN, IGN
    loss, lse = op.loss(h, w, y)
    hurt = dloss.clone()
    hurt[0, 5], hurt[0, 6], hurt[0, 7] = float("inf"), -float("inf"), float("nan")
    hurt[:, 9], hurt[:, 12] = float("inf"), float("nan")
    dh, dw = op.grad(h, w, y, lse, hurt)
    zero = torch.where(hurt.isfinite(), hurt, 0.0)
    _, _, e_dh, e_dw, b_dh, b_dw = exact(h, w, y, zero)
    rows = torch.ones_like(y, dtype=torch.bool)
    rows[0, 5:8] = False
    assert bool(((dh.double() - e_dh).abs() <= b_dh)[rows].all())
    assert not bool(dh[0, 5:8].isfinite().all(1).any())
    assert not bool(dw[0].isfinite().all(1).any())
    assert bool(((dw.double() - e_dw).abs() <= b_dw)[1].all())


@pytest.mark.gpu
@pytest.mark.parametrize("size", [(1, 20, 20000, 64), (1, 70, 20000, 72), (2, 300, 20000, 64), (1, 100, 9000, 1032), (1, 9, 60000, 64)], ids=str)
@pytest.mark.parametrize("dtype", [BF, HF], ids=str)
def test_rows_of_tokens_with_little_weight(size, dtype):
    """dloss of 1 to 2^-20 of the largest: a row of dhidden is as exact relative to its own dloss.  The weights have a common
    part, so that the many small p of a row add up.  Every entry: u |dz| |W| + 2e-5 (1 + |lse|) p |dloss| |W| + the result's
    rounding as elsewhere, and the spacing of the smallest dz, 2^-37 of the largest dloss of which the token's is 1/64 at
    least, or of the token's own: 2^-31 |dloss|."""
    n, t, v, d = size
    h, w, y, _ = inputs(n, t, v, d, dtype, spread=0.5)
    w = (w.float() + 0.5).to(dtype)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(t)
    dloss = 4096 * torch.exp2(-20 * torch.rand((n, t), generator=gen, device="cuda")) * torch.randint(0, 2, (n, t), generator=gen, device="cuda").mul(2).sub(1)
    dloss[:, 0], dloss[:, 1], dloss[:, 2] = 4096, 4096 * 2.0 ** -20, 0
    op = train.LinearCrossEntropy(n, t, v, d, dtype)
    _, lse = op.loss(h, w, y)
    dh, dw = op.grad(h, w, y, lse, dloss)
    u, tiny = (2.0 ** -8, 0.0) if dtype == BF else (2.0 ** -11, 2.0 ** -25)
    for i in range(n):
        hi, wi = h[i].double(), w[i].double()
        ok = y[i] != IGN
        z = hi @ wi.t()
        l = torch.logsumexp(z, 1)[:, None]
        p = torch.exp(z - l)
        g = (dloss[i].double() * ok)[:, None]
        off = 2e-5 * (1 + l.abs()) * p * g.abs() + 2.0 ** -31 * g.abs()
        p[torch.arange(t, device="cuda"), torch.where(ok, y[i], 0)] -= 1
        dz = p * g
        want = dz @ wi
        bound = 1.1 * ((off + u * dz.abs()) @ wi.abs() + u * want.abs() + tiny)
        assert bool(((dh[i].double() - want).abs() <= bound).all())
        # and as a whole, row by row: roundings of dz and of the result are independent of one another
        live = ok & (dloss[i].abs() > 0)
        err = (dh[i].double() - want)[live].norm(dim=1)
        size_of = u * (dz[live].square() @ wi.square()).sum(1).sqrt() + u * want[live].norm(dim=1) + (off[live] @ wi.abs()).norm(dim=1) + tiny * d ** 0.5
        assert bool((err <= 1.1 * size_of).all())
    _, _, _, e_dw, _, b_dw = exact(h, w, y, dloss)
    assert bool(((dw.double() - e_dw).abs() <= b_dw).all())


@pytest.mark.gpu
@pytest.mark.parametrize("t", [3, 50, 200])
def test_logits_of_any_finite_size(t):
    """Rows whose logits all lie near the type's lowest value, beside ordinary ones."""
    n, v, d = 1, 300, 16
    h, w, y, dloss = inputs(n, t, v, d, BF)
    w = w.float()
    w[..., 0] = 1 + torch.arange(v, device="cuda") / 64.0
    h = h.float()
    h[0, 1, :], h[0, 1, 0] = 0, -1e35
    h[0, 2, :], h[0, 2, 0] = 0, -1e38 / 4
    h, w = h.bfloat16(), w.bfloat16()
    y[0, 1], y[0, 2] = 0, 5
    op = train.LinearCrossEntropy(n, t, v, d, BF)
    check(op, h, w, y, dloss, BF)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF], ids=str)
@pytest.mark.parametrize("size", [(2, 20, 300, 64, 0), (2, 32, 300, 72, 0), (3, 90, 700, 201, 256), (2, 300, 700, 136, 0), (2, 333, 3000, 264, 1024),
                                  (1, 70, 50, 1, 0)], ids=str)
def test_hidden_states_of_tokens_that_do_not_count_may_be_anything(size, dtype):
    """The same gradients, bit for bit, as with zeros there."""
    n, t, v, d, piece = size
    h, w, y, dloss = inputs(n, t, v, d, dtype)
    y[:, :8] = 1
    y[:, 3], y[0, 5], y[:, t - 1] = IGN, IGN, IGN
    dloss[:, 6] = 0
    op = train.LinearCrossEntropy(n, t, v, d, dtype, piece=piece)
    blank = h.clone()
    blank[:, 3], blank[0, 5], blank[:, t - 1], blank[:, 6] = 0, 0, 0, 0
    odd = blank.clone()
    odd[:, 3], odd[0, 5, 0], odd[:, t - 1], odd[:, 6] = float("nan"), float("inf"), -float("inf"), float("nan")
    if d > 1:
        odd[:, t - 1, 1] = float("inf")
    loss, lse = op.loss(blank, w, y)
    want = op.grad(blank, w, y, lse, dloss)
    check(op, blank, w, y, dloss, dtype)
    loss2, lse2 = op.loss(odd, w, y)
    counted = torch.ones_like(y, dtype=torch.bool)
    counted[:, 6] = False
    assert torch.equal(loss2[counted], loss[counted])
    got = op.grad(odd, w, y, lse2, dloss)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    got = op.grad(odd, w, y, lse2, dloss, need_dhidden=False)
    assert torch.equal(got[1], want[1])
    again = op.grad(blank, w, y, lse, dloss)
    assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])
    # one array of hidden states for all workers: where another worker counts the token, its gradient is spoiled, and only its
    if n > 1:
        shared = odd[:1].expand(n, -1, -1)
        y2 = y.clone()
        y2[1, 3] = 2
        _, lse3 = op.loss(shared, w, y2)
        got = op.grad(shared, w, y2, lse3, dloss)
        base = blank[:1].expand(n, -1, -1)
        _, lse4 = op.loss(base, w, y2)
        want = op.grad(base, w, y2, lse4, dloss)
        assert torch.equal(got[0][0], want[0][0]) and torch.equal(got[1][0], want[1][0])
        assert bool(got[1][1].isnan().any()) and bool(got[0][1, 3].isnan().any())


@pytest.mark.gpu
def test_large_logits_and_values_that_are_not_finite():
    n, t, v, d = 1, 70, 500, 64
    h, w, y, dloss = inputs(n, t, v, d, BF, spread=60.0)
    op = train.LinearCrossEntropy(n, t, v, d, BF)
    check(op, h, w, y, dloss, BF)
    for value in (float("nan"), float("inf")):
        g = h.clone()
        g[0, 3, 9] = value
        loss, lse = op.loss(g, w, torch.zeros_like(y))
        keep = torch.arange(t, device="cuda") != 3
        assert bool(loss[0, 3].isnan()) and bool(loss[0, keep].isfinite().all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF], ids=str)
def test_strides_alignment_and_shared_weights(dtype):
    n, t, v, d = 3, 60, 300, 104
    h, w, y, dloss = inputs(n, t, v, d, dtype)
    op = train.LinearCrossEntropy(n, t, v, d, dtype)

    def inside(a, extra, shift):
        big = torch.zeros((a.shape[0], a.shape[1] + 2, a.shape[2] + extra), dtype=dtype, device="cuda")
        view = big[:, 1:-1, shift:shift + a.shape[2]]
        view.copy_(a)
        return view

    base = check(op, h, w, y, dloss, dtype)
    for extra, shift in ((8, 0), (24, 8), (3, 0), (16, 5)):
        loss, lse = op.loss(inside(h, extra, shift), inside(w, extra, shift), y)
        got = op.grad(inside(h, extra, shift), inside(w, extra, shift), y, lse, dloss)
        assert torch.equal(loss, base[0]) and torch.equal(got[0], base[2]) and torch.equal(got[1], base[3])
    shared = w[:1].expand(n, -1, -1)
    check(op, h, shared, y, dloss, dtype)
    check(op, h[:1].expand(n, -1, -1), w, y, dloss, dtype)
    check(op, h[:, :1].expand(-1, t, -1), w, y, dloss, dtype)
    # into a slice of each worker's flat gradient, at an odd place
    flat = torch.full((n, v * d + 37), 3.0, dtype=dtype, device="cuda")
    place = flat[:, 5:5 + v * d].view(n, v, d) if n == 1 else flat.as_strided((n, v, d), (v * d + 37, d, 1), 5)
    loss, lse = op.loss(h, w, y)
    op.grad(h, w, y, lse, dloss, dweight=place)
    assert torch.equal(place, base[3]) and bool((flat[:, :5] == 3).all()) and bool((flat[:, 5 + v * d:] == 3).all())
    only_h = op.grad(h, w, y, lse, dloss, need_dweight=False)
    only_w = op.grad(h, w, y, lse, dloss, need_dhidden=False)
    assert only_h[1] is None and only_w[0] is None
    assert torch.equal(only_h[0], base[2]) and torch.equal(only_w[1], base[3])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF], ids=str)
@pytest.mark.parametrize("size", [(3, 20, 1700, 264), (2, 100, 900, 328), (1, 300, 700, 264), (2, 33, 515, 201)], ids=str)
@pytest.mark.parametrize("piece", [0, 256])
def test_gradients_inside_larger_arrays(size, piece, dtype):
    """Gradients in the middle of larger arrays, as parts of a flat gradient are: what lies around them stays."""
    n, t, v, d = size
    h, w, y, dloss = inputs(n, t, v, d, dtype)
    op = train.LinearCrossEntropy(n, t, v, d, dtype, piece=piece)
    loss, lse = op.loss(h, w, y)
    gap = 64
    flat = torch.full((n, gap + v * d + gap), 7.0, dtype=dtype, device="cuda")
    around = torch.full((gap + n * t * d + gap,), 7.0, dtype=dtype, device="cuda")
    dw = flat[:, gap:gap + v * d].view(n, v, d)
    dh = around[gap:gap + n * t * d].view(n, t, d)
    op.grad(h, w, y, lse, dloss, dhidden=dh, dweight=dw)
    plain_dh, plain_dw = op.grad(h, w, y, lse, dloss)
    assert torch.equal(dw, plain_dw) and torch.equal(dh, plain_dh)
    assert bool((flat[:, :gap] == 7).all()) and bool((flat[:, gap + v * d:] == 7).all())
    assert bool((around[:gap] == 7).all()) and bool((around[-gap:] == 7).all())
    check(op, h, w, y, dloss, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF], ids=str)
@pytest.mark.parametrize("size", [(1, 2, 2933), (1, 3, 4096), (150, 4, 2048), (2, 500, 1024)], ids=str)
def test_tokens_that_are_nearly_certain(size, dtype):
    """A loss near 0 and p - 1 are small differences of large logits.  z is the same in loss and gradient, so that what is off in
    it (1e-5 of 1 + |lse|) moves 1 - p, and the loss, by its share of them only; beside that there is the rounding of lse and the
    exponential's, 2^-24 |lse| + 2^-22 at most, of which a 1e-6 of 1 + |lse| is allowed."""
    t, v, d = size
    gen = torch.Generator(device="cuda")
    gen.manual_seed(d)
    w = (torch.randn((1, v, d), generator=gen, device="cuda") * 2 / d ** 0.5).to(dtype)
    y = torch.randint(0, v, (1, t), generator=gen, device="cuda")
    h = (0.4 * torch.randn((1, t, d), generator=gen, device="cuda") + 2.2 * w[0][y[0]].float()).to(dtype)
    dloss = torch.ones((1, t), device="cuda")
    op = train.LinearCrossEntropy(1, t, v, d, dtype)
    loss, lse = op.loss(h, w, y)
    dh, dw = op.grad(h, w, y, lse, dloss)
    e_loss, e_lse, e_dh, e_dw, _, _ = exact(h, w, y, dloss)
    size_of = 1 + float(e_lse.abs().max())
    left = -torch.expm1(-e_loss)                                     # 1 - p
    assert bool(((loss.double() - e_loss).abs() <= (1e-5 * left + 2.0 ** -22) * size_of).all())
    off = GRAD[dtype] + 1e-5 * size_of + 1e-6 * size_of * t ** 0.5 / float(left.norm())
    assert far(dh, e_dh) < off and far(dw, e_dw) < off


@pytest.mark.gpu
def test_gradient_against_differences():
    """Central differences of the op's own loss along random directions: fp16 inputs moved by amounts they hold exactly."""
    n, t, v, d = 1, 40, 120, 32
    h, w, y, _ = inputs(n, t, v, d, HF, ignored=0.1)
    op = train.LinearCrossEntropy(n, t, v, d, HF)
    h, w = (h * 256).round().div(256).to(HF), (w * 256).round().div(256).to(HF)
    h.clamp_(-4, 4), w.clamp_(-4, 4)
    dloss = torch.ones((n, t), device="cuda")
    _, lse = op.loss(h, w, y)
    dh, dw = op.grad(h, w, y, lse, dloss)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    eps = 2.0 ** -6
    for x, g, which in ((h, dh, 0), (w, dw, 1)):
        for _ in range(4):
            step = torch.randint(0, 2, x.shape, generator=gen, device="cuda").to(HF).mul_(2).sub_(1)
            moved = [op.loss(*((x + s * eps * step, w) if which == 0 else (h, x + s * eps * step)), y)[0].double().sum()
                     for s in (1, -1)]
            slope = float((moved[0] - moved[1]) / (2 * eps))
            said = float((g.double() * step.double()).sum())
            # third derivatives of 36 terms of order eps^2 |direction|^3, and fp32 sums of losses of about 5
            assert abs(slope - said) <= 0.02 * abs(said) + 0.02 * float(g.double().norm()) + 0.05


@pytest.mark.gpu
def test_calls_are_repeatable_on_any_stream_and_in_a_graph():
    n, t, v, d = 2, 260, 1500, 264
    two = [inputs(n, t, v, d, BF, seed=s) for s in (1, 2)]
    op = train.LinearCrossEntropy(n, t, v, d, BF, piece=512)

    def call(h, w, y, dloss):
        loss, lse = op.loss(h, w, y)
        return [loss, *op.grad(h, w, y, lse, dloss)]

    want = [call(*x) for x in two]
    for _ in range(3):
        for x, q in zip(two, want):
            assert all(torch.equal(a, b) for a, b in zip(call(*x), q))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = call(*two[0])
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want[0]))
    bufs = [x.clone() for x in two[0]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(*bufs)
    for x, q in zip(two, want):
        for b, s in zip(bufs, x):
            b.copy_(s)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(out, q))


@pytest.mark.gpu
@pytest.mark.parametrize("size", [(60, 20, 1100, 200), (8, 100, 1200, 2048), (1, 100, 1535, 16384), (1, 5, 1500, 64), (2, 5, 1000, 520)], ids=str)
def test_inner_dimensions_of_fewer_than_24_stages_are_left_whole(size):
    """However many SMs that leaves idle: the gradients are two kernels, with none that joins shares.  (1535 entries are 24.)"""
    n, t, v, d = size
    h, w, y, dloss = inputs(n, t, v, d, BF)
    op = train.LinearCrossEntropy(n, t, v, d, BF)
    _, lse, _, _ = check(op, h, w, y, dloss, BF)
    before = op.launches
    op.grad(h, w, y, lse, dloss)
    assert op.launches - before == (2 if (v + 63) // 64 < 24 else 3)


@pytest.mark.gpu
@pytest.mark.parametrize("size", [(1, 40, 50000, 64), (2, 300, 30000, 72)], ids=str)
def test_a_long_kernel_ahead_that_lets_the_next_one_be_set_up(size):
    """The time that the kernel ahead takes, about 1.6 s here, is no wait that could run out (those may take about one)."""
    import ctypes
    import __graft_entry__
    ahead = ctypes.CDLL(f"{__graft_entry__.ROOT}/tests/libearly_trigger.so")
    ahead.early_trigger.argtypes = [ctypes.c_longlong, ctypes.c_void_p]
    n, t, v, d = size
    h, w, y, dloss = inputs(n, t, v, d, BF)
    op = train.LinearCrossEntropy(n, t, v, d, BF)
    loss, lse = op.loss(h, w, y)
    want = op.grad(h, w, y, lse, dloss)
    stream = torch.cuda.current_stream().cuda_stream
    assert ahead.early_trigger(3_000_000_000, stream) == 0
    got = op.loss(h, w, y)
    assert ahead.early_trigger(3_000_000_000, stream) == 0
    got += op.grad(h, w, y, lse, dloss)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, (loss, lse, *want)))
    op.loss(h, w, y)                                  # and nothing was reported


@pytest.mark.gpu
@pytest.mark.parametrize("size", [(1, 600, 40000, 256), (8, 130, 3001, 128)], ids=str)
def test_many_tiles(size):
    n, t, v, d = size
    h, w, y, dloss = inputs(n, t, v, d, BF)
    check(train.LinearCrossEntropy(n, t, v, d, BF), h, w, y, dloss, BF)


@pytest.mark.gpu
@pytest.mark.parametrize("size", [(1, 40, 700, 2112), (1, 150, 520, 4104), (1, 3, 1000, 8192)], ids=str)
def test_long_inner_dimensions(size):
    """Losses as exact as for short ones: 2e-6 of 1 + |lse| whatever the dimension (partial sums taken out of the tensor cores)."""
    n, t, v, d = size
    h, w, y, dloss = inputs(n, t, v, d, BF)
    loss, lse, _, _ = check(train.LinearCrossEntropy(n, t, v, d, BF), h, w, y, dloss, BF)
    e_loss, e_lse = exact(h, w, y, dloss)[:2]
    assert bool(((lse.double() - e_lse).abs() <= 2e-6 * (1 + e_lse.abs())).all())


@pytest.mark.gpu
def test_refusals():
    ok = dict(n_workers=2, max_tokens=8, vocab=30, dim=16, dtype=BF)
    op = train.LinearCrossEntropy(**ok)
    h, w, y, dloss = inputs(2, 8, 30, 16, BF)
    _, lse = op.loss(h, w, y)
    for args in ((h.float(), w, y), (h, w.float(), y), (h, w, y.int()), (h[:1], w, y), (h, w[:, :29], y), (h, w, y[:, :7]), (h.cpu(), w, y),
                 (h, w, y.t()), (h.transpose(1, 2), w, y), (torch.cat([h, h], 1), w, torch.cat([y, y], 1))):
        with pytest.raises(CSERError):
            op.loss(*args)
    for args, kw in (((lse.double(), dloss), {}), ((lse, dloss[:, :7]), {}), ((lse, dloss.cpu()), {}), ((lse, dloss), dict(dhidden=h.float())),
                     ((lse, dloss), dict(dweight=w.transpose(0, 1))), ((lse, dloss), dict(dweight=w[:1]))):
        with pytest.raises(CSERError):
            op.grad(h, w, y, *args, **kw)
    L = train.lib()
    import ctypes
    args = op._inputs(h, w, y, IGN)
    p = lse.data_ptr()
    assert L.cser_xent_loss(None, ctypes.byref(args), p, p, None) == -1
    assert L.cser_xent_loss(op.h, None, p, p, None) == -1
    assert L.cser_xent_loss(op.h, ctypes.byref(args), p, None, None) == -1
    assert L.cser_xent_grad(op.h, ctypes.byref(args), p, None, None, w.data_ptr(), 480, None) == -1
    assert L.cser_xent_grad(op.h, ctypes.byref(args), p, p, None, w.data_ptr(), 479, None) == -1
    for name, value in (("tokens", 9), ("tokens", -1), ("hidden_row_stride", -16), ("hidden", None), ("hidden", 3), ("target", None)):
        args = op._inputs(h, w, y, IGN)
        setattr(args, name, value)
        assert L.cser_xent_loss(op.h, ctypes.byref(args), p, p, None) == -1, name
    L.cser_xent_destroy(None)


def test_refusals_need_no_gpu():
    """Arguments are checked before the first CUDA call."""
    ok = dict(n_workers=2, max_tokens=8, vocab=30, dim=16, dtype=BF)
    for bad in (dict(n_workers=0), dict(max_tokens=0), dict(vocab=0), dict(dim=0), dict(dim=70000), dict(vocab=2 ** 24 + 1), dict(piece=-1),
                dict(max_tokens=2 ** 24), dict(dtype=torch.float32), dict(dtype=torch.float64), dict(n_workers=2 ** 10, vocab=2 ** 24)):
        with pytest.raises(CSERError):
            train.LinearCrossEntropy(**{**ok, **bad})
    assert train.lib().cser_xent_launch_count(None) == 0
