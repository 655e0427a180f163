"""Orthogonalised updates (cser_orth_* of cser_train.h) against the formula in 64 bits.

Tolerances, relative to the 2-norm of the exact result.  16-bit results: the products' own error, at most 2e-3 for
inputs like these (fp16 operands with remainder and diagonals apart), plus the rounding of the result, 2^-8 (bf16) or
2^-11 (fp16) of each value.  32-bit results: operands of 22 bits and at most 256 terms to an accumulator whose partial sums are
truncated at 2^-24 leave about 1e-6 for each of the last steps' products; 5e-6 is allowed.
"""
import numpy as np
import pytest
import torch

from paper_2007_13221_b200 import train
from paper_2007_13221_b200.binding import CSERError

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
OUT = {BF: 2e-3 + 2.0 ** -8, HF: 2e-3 + 2.0 ** -11, F32: 5e-6}


def exact(u, steps=5, scale=1.0):
    """X (a I + b K + c K K), K = X^T X, in float64 (the other grouping of the same polynomial when the matrix is wide)."""
    x = u.double()
    x = x / (x.square().sum().sqrt() + 1e-7)
    for _ in range(steps):
        k = x.t() @ x
        x = 3.4445 * x + x @ (-4.7750 * k + 2.0315 * (k @ k))
    return scale * x


def matrix(gen, r, c, kind="mixed"):
    x = torch.randn((r, c), generator=gen, device="cuda")
    if kind == "mixed" and min(r, c) > 8:
        x = 0.3 * x + torch.randn((r, 4), generator=gen, device="cuda") @ torch.randn((4, c), generator=gen, device="cuda") / 2
    if kind == "low rank":
        x = 0.02 * x + torch.randn((r, 4), generator=gen, device="cuda") @ torch.randn((4, c), generator=gen, device="cuda") / 2
    return x * 0.01


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def far(got, want):
    return float((got.double() - want).norm() / want.norm())


SHAPES = [(1, 1), (1, 77), (77, 1), (2, 3), (16, 1024), (1024, 16), (64, 64), (63, 65), (127, 129), (128, 128), (129, 127),
          (128, 256), (256, 128), (257, 640), (640, 257), (300, 1500), (1100, 513), (1, 5000),
          (8, 200), (9, 40), (24, 24), (200, 25), (32, 33), (40, 500), (48, 48), (56, 300), (64, 4000)]


@pytest.mark.gpu
@pytest.mark.parametrize("types", [(BF, BF), (F32, F32), (F32, BF), (HF, HF)], ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_one_matrix(shape, types):
    r, c = shape
    u = matrix(generator(r * 7919 + c), r, c).to(types[0])
    o = train.Orthogonalizer([(0, r, c)], 1, r * c, *types)
    got = o.apply(u.reshape(1, -1)).view(r, c)
    assert got.dtype == types[1]
    assert far(got, exact(u)) < OUT[types[1]]
    assert o.launches > 0


@pytest.mark.gpu
@pytest.mark.parametrize("out", [BF, F32], ids=str)
@pytest.mark.parametrize("kind", ["low rank", "noise"])
def test_other_spectra(kind, out):
    for r, c in ((256, 512), (700, 320)):
        u = matrix(generator(5), r, c, kind)
        got = train.Orthogonalizer([(0, r, c)], 1, r * c, F32, out).apply(u.reshape(1, -1)).view(r, c)
        assert far(got, exact(u)) < OUT[out]


@pytest.mark.gpu
@pytest.mark.parametrize("out", [BF, HF], ids=str)
@pytest.mark.parametrize("kind", ["mixed", "noise", "low rank"])
@pytest.mark.parametrize("shape", [(384, 512), (1000, 300), (1024, 1024), (2048, 512)], ids=str)
def test_products_of_16_bit_results_leave_a_thousandth(shape, kind, out):
    """1e-3 before the rounding of the result, whose 2-norm is 2^-p / sqrt(7) of the result's for p bits (half an ulp, uniform, of values
    spread evenly over a binade), the two independent; a tenth for how values really lie in their binades."""
    u = matrix(generator(sum(shape)), *shape, kind)
    got = train.Orthogonalizer([(0, *shape)], 1, u.numel(), F32, out).apply(u.reshape(1, -1)).view(shape)
    rounding = 2.0 ** (-8 if out == BF else -11) / 7 ** 0.5
    assert far(got, exact(u)) < 1.1 * (1e-6 + rounding ** 2) ** 0.5


@pytest.mark.gpu
def test_singular_values_come_near_one():
    u = matrix(generator(1), 192, 384, "noise")
    got = train.Orthogonalizer([(0, 192, 384)], 1, u.numel(), F32, F32).apply(u.reshape(1, -1)).view(192, 384)
    s = torch.linalg.svdvals(got.double())
    assert float(s.max()) < 1.22 and float(s.min()) > 0.65


@pytest.mark.gpu
@pytest.mark.parametrize("steps", [1, 2, 3, 7])
def test_steps_and_scales(steps):
    gen = generator(steps)
    shapes, scales = [(96, 200), (200, 96)], [0.2, -3.0]
    us = [matrix(gen, *s) for s in shapes]
    flat = torch.cat([u.reshape(-1) for u in us]).reshape(1, -1)
    o = train.Orthogonalizer([(0, 96, 200), (96 * 200, 200, 96)], 1, flat.numel(), F32, F32, scales=scales, steps=steps)
    out = o.apply(flat)
    for k, (u, s) in enumerate(zip(us, scales)):
        assert far(out[0, k * 19200:(k + 1) * 19200].view(u.shape), exact(u, steps, s)) < OUT[F32]


@pytest.mark.gpu
@pytest.mark.parametrize("types", [(BF, BF), (F32, F32), (F32, HF)], ids=str)
@pytest.mark.parametrize("mu", [0.0, 0.95])
def test_many_matrices_of_many_workers_with_strides_gaps_and_momentum(types, mu):
    n, gen = 3, generator(11)
    #        offset, rows, cols, row stride
    plan = [(5, 40, 33, 33), (1400, 17, 129, 140), (4001, 130, 70, 70), (13200, 1, 9, 9), (13213, 256, 64, 72), (32000, 64, 264, 264)]
    ld = 32000 + 64 * 264 + 3
    grad = (torch.randn((n, ld), generator=gen, device="cuda") * 0.02).to(types[0])
    m = (torch.randn((n, ld), generator=gen, device="cuda") * 0.02) if mu else None
    m0 = m.clone() if mu else None
    out = torch.full((n, ld), 7.0, dtype=types[1], device="cuda")
    keep = torch.ones(ld, dtype=torch.bool, device="cuda")
    o = train.Orthogonalizer([p[:3] for p in plan], n, ld, *types, row_strides=[p[3] for p in plan])
    assert o.apply(grad, out, momentum=m, mu=mu) is out
    for at, r, c, st in plan:
        where = at + torch.arange(r, device="cuda")[:, None] * st + torch.arange(c, device="cuda")[None, :]
        keep[where.reshape(-1)] = False
        for i in range(n):
            u = grad[i][where].double()
            if mu:
                want_m = mu * m0[i][where].double() + u
                assert torch.allclose(m[i][where].double(), want_m, rtol=2.0 ** -22, atol=2.0 ** -24 * 0.1)
                u = u + mu * want_m
            assert far(out[i][where], exact(u)) < OUT[types[1]], (at, i)
    assert bool((out[:, keep] == 7.0).all())
    if mu:
        assert torch.equal(m[:, keep], m0[:, keep])


@pytest.mark.gpu
def test_zeros_and_values_that_are_not_finite_stay_in_their_matrix():
    for out_t in (BF, F32):
        u = torch.cat([matrix(generator(3), 80, 100).reshape(-1) for _ in range(4)]).reshape(1, -1).clone()
        u[0, :8000] = 0
        u[0, 8000 + 57] = float("nan")
        u[0, 16000 + 99] = float("inf")
        got = train.Orthogonalizer([(k * 8000, 80, 100) for k in range(4)], 1, 32000, F32, out_t).apply(u)[0]
        assert bool((got[:8000] == 0).all())
        assert bool(got[8000:16000].isnan().any()) and bool(got[16000:24000].isnan().any())
        assert far(got[24000:].view(80, 100), exact(u[0, 24000:].view(80, 100))) < OUT[out_t]


@pytest.mark.gpu
@pytest.mark.parametrize("size", [1e-3, 1e15])
def test_magnitudes(size):
    u = matrix(generator(9), 100, 150) * size
    got = train.Orthogonalizer([(0, 100, 150)], 1, 15000, F32, F32).apply(u.reshape(1, -1)).view(100, 150)
    assert far(got, exact(u)) < OUT[F32]


@pytest.mark.gpu
@pytest.mark.parametrize("out_t", [BF, F32], ids=str)
def test_calls_are_repeatable_on_any_stream_and_in_a_graph(out_t):
    shapes, n = [(130, 300), (513, 90), (256, 256), (64, 700)], 2
    mats, at = [], 0
    for r, c in shapes:
        mats.append((at, r, c))
        at += r * c
    gen = generator(2)
    grads = [torch.randn((n, at), generator=gen, device="cuda") for _ in range(2)]
    o = train.Orthogonalizer(mats, n, at, F32, out_t)
    first = [o.apply(g).clone() for g in grads]
    for _ in range(3):
        for g, w in zip(grads, first):
            assert torch.equal(o.apply(g), w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = o.apply(grads[0])
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, first[0])
    buf, out = grads[0].clone(), torch.zeros((n, at), dtype=out_t, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o.apply(buf, out)
    for g, w in zip(grads, first):
        buf.copy_(g)
        graph.replay()
        assert torch.equal(out, w)
    if out_t == F32:                                   # in place
        o.apply(buf, buf)
        assert torch.equal(buf, first[1])


@pytest.mark.gpu
def test_results_do_not_depend_on_what_else_the_plan_holds():
    """More matrices than one group of the workspace holds: each result is what a plan of its own gives."""
    r = c = 2048
    k = 60                                            # 60 x 50 MB of workspace
    grad = torch.randn((1, k * r * c), generator=generator(4), device="cuda").to(BF)
    out = train.Orthogonalizer([(i * r * c, r, c) for i in range(k)], 1, k * r * c, BF, BF).apply(grad)
    alone = train.Orthogonalizer([(0, r, c)], 1, r * c, BF, BF)
    for i in (0, 31, k - 1):
        part = slice(i * r * c, (i + 1) * r * c)
        assert torch.equal(out[:, part], alone.apply(grad[:, part].contiguous()))
    assert far(out[0, :r * c].view(r, c), exact(grad[0, :r * c].view(r, c))) < OUT[BF]


@pytest.mark.gpu
@pytest.mark.parametrize("out_t", [BF, F32], ids=str)
@pytest.mark.parametrize("shapes", [[(500, 1000), (1000, 500)] * 7, [(130, 200), (200, 130)] * 20, [(129, 65)] * 3], ids=lambda s: f"{len(s)}")
def test_plans_of_different_sizes(shapes, out_t):
    """Many large matrices, many small ones, few: tiles are cut differently."""
    gen, mats, at = generator(8), [], 0
    for r, c in shapes:
        mats.append((at, r, c))
        at += r * c
    u = torch.cat([matrix(gen, r, c).reshape(-1) for r, c in shapes] * 2).reshape(2, -1)
    got = train.Orthogonalizer(mats, 2, at, F32, out_t).apply(u)
    for o, r, c in mats:
        for i in range(2):
            assert far(got[i, o:o + r * c].view(r, c), exact(u[i, o:o + r * c].view(r, c))) < OUT[out_t], (r, c)


@pytest.mark.gpu
@pytest.mark.parametrize("types", [(BF, BF), (F32, F32), (F32, HF)], ids=str)
@pytest.mark.parametrize("shapes", [[(100, 6000)], [(6000, 100), (70, 1025)], [(300, 5003)] * 2, [(512, 16384)] * 2, [(8192, 700), (65, 65)],
                                    [(64, 20000)], [(30001, 7), (40, 9000)], [(33, 9000), (200, 300)]],
                         ids=lambda s: f"{len(s)}x{s[0]}")
def test_long_sides_in_shares(shapes, types):
    """Few and long: the inner dimension of A is summed in shares by several CTAs.  The same bits every time."""
    gen = generator(17)
    ms = [matrix(gen, r, c).to(types[0]) for r, c in shapes]
    at, mats = 0, []
    for r, c in shapes:
        mats.append((at, r, c))
        at += r * c
    flat = torch.cat([m.reshape(-1) for m in ms]).reshape(1, -1)
    o = train.Orthogonalizer(mats, 1, at, *types)
    first = o.apply(flat).clone()
    for (off, r, c), m in zip(mats, ms):
        assert far(first[0, off:off + r * c].view(r, c), exact(m)) < OUT[types[1]]
    for _ in range(3):
        assert torch.equal(o.apply(flat), first)


@pytest.mark.gpu
def test_refusals():
    ok = dict(matrices=[(0, 4, 5)], n_workers=1, ld=20)
    train.Orthogonalizer(**ok)
    for bad in (dict(n_workers=0), dict(ld=19), dict(matrices=[]), dict(matrices=[(0, 0, 5)]), dict(matrices=[(-1, 4, 5)]),
                dict(matrices=[(1, 4, 5)]), dict(matrices=[(0, 70000, 1)], ld=70000), dict(steps=0), dict(steps=17), dict(row_strides=[4]),
                dict(row_strides=[5, 5]), dict(scales=[float("nan")]), dict(in_dtype=torch.float64)):
        with pytest.raises(CSERError):
            train.Orthogonalizer(**{**ok, **bad})
    o = train.Orthogonalizer([(0, 4, 5)], 2, 20, BF, BF)
    g = torch.randn((2, 20), device="cuda").to(BF)
    for args, kw in (((g.float(),), {}), ((g[:1],), {}), ((g.cpu(),), {}), ((g, g.float()), {}), ((g.t(),), {}),
                     ((g,), dict(momentum=g)), ((g,), dict(momentum=g.float(), mu=1.0)), ((g,), dict(momentum=g.float(), mu=-0.1)),
                     ((g,), dict(momentum=g.float(), mu=float("nan")))):
        with pytest.raises(CSERError):
            o.apply(*args, **kw)
    L = train.lib()
    assert L.cser_orth_apply(None, g.data_ptr(), None, 0.0, g.data_ptr(), None) == -1
    assert L.cser_orth_apply(o.h, None, None, 0.0, g.data_ptr(), None) == -1
    host = torch.zeros((2, 20), dtype=BF)
    assert L.cser_orth_apply(o.h, host.data_ptr(), None, 0.0, g.data_ptr(), None) == -1
    assert L.cser_orth_apply(o.h, g.data_ptr() + 1, None, 0.0, g.data_ptr(), None) == -1
    L.cser_orth_destroy(None)
    assert torch.equal(o.apply(g), o.apply(g))


@pytest.mark.gpu
@pytest.mark.parametrize("shapes", [[(200, 300)], [(200, 300), (16, 16)], [(512, 1024)] * 12], ids=lambda s: f"{len(s)}")
@pytest.mark.parametrize("out_t", [BF, F32], ids=str)
def test_a_wait_that_runs_out_ends_the_kernel_and_is_reported(shapes, out_t):
    """Single CTAs and pairs, both results: the context and other plans stay usable."""
    mats, at = [], 0
    for r, c in shapes:
        mats.append((at, r, c))
        at += r * c
    g = torch.randn((1, at), device="cuda")
    o, other = (train.Orthogonalizer(mats, 1, at, F32, out_t) for _ in range(2))
    want = other.apply(g)
    assert torch.equal(o.apply(g), want)
    L = train.lib()
    for bad in (0, 2001):
        assert L.cser_orth_debug_stall_next(o.h, bad) == -1
    assert L.cser_orth_debug_stall_next(o.h, 20) == 0
    o.apply(g)
    torch.cuda.synchronize()
    for _ in range(2):
        with pytest.raises(CSERError, match="wait ran out"):
            o.apply(g)
    assert torch.equal(other.apply(g), want)
    o.close()
    small = train.Orthogonalizer([(0, 8, 8)], 1, 64)
    assert L.cser_orth_debug_stall_next(small.h, 20) == -1 and L.cser_orth_debug_stall_next(None, 20) == -1


@pytest.mark.gpu
def test_arrays_that_overlap_are_refused():
    """From the first matrix's beginning to the last one's end; what lies outside may."""
    n, ld = 2, 400
    o, wide = (train.Orthogonalizer([(40, 10, 12), (200, 8, 9)], n, ld, F32, t) for t in (F32, BF))
    buf = torch.randn(8 * n * ld, generator=generator(1), device="cuda")

    def at(k, t=F32):
        return buf.view(t)[k * 4 // (4 if t == F32 else 2):][:n * ld].view(n, ld)

    grad, size = at(2000), (n - 1) * ld + 200 + 72 - 40             # touched elements
    want = o.apply(grad.clone(), momentum=torch.ones_like(grad), mu=0.5)
    for k in (2000 - size, 2000 + size):                             # just apart
        keep = buf.clone()
        assert torch.equal(o.apply(grad, at(k), momentum=torch.ones_like(grad), mu=0.5)[:, 40:160], want[:, 40:160])
        buf.copy_(keep)
    for k in (2000 - size + 1, 1999, 2001, 2000 + size - 1):
        with pytest.raises(CSERError, match="apart"):
            o.apply(grad, at(k))
        with pytest.raises(CSERError, match="its own"):
            o.apply(grad, momentum=at(k))
        with pytest.raises(CSERError, match="its own"):
            o.apply(grad, at(4800), momentum=at(4800 + k - 2000))
    with pytest.raises(CSERError, match="apart"):
        wide.apply(grad, at(2100, BF))
    with pytest.raises(CSERError):
        wide.apply(grad, at(2000, BF))


def test_refusals_need_no_gpu():
    """Arguments are checked before the first CUDA call."""
    for bad in (dict(n_workers=0), dict(ld=0), dict(matrices=[(0, 4, 6)]), dict(matrices=[(0, 4, 0)]), dict(steps=0)):
        with pytest.raises(CSERError, match="cser_orth_create"):
            train.Orthogonalizer(**{**dict(matrices=[(0, 4, 5)], n_workers=1, ld=20), **bad})
    assert train.lib().cser_orth_launch_count(None) == 0


def test_formula_of_the_exact_form():
    """The tests' own reference against the singular values: every one goes through the quintic, vectors stay."""
    rng = np.random.default_rng(0)
    x = torch.from_numpy(rng.standard_normal((12, 7)))
    u, s, v = torch.linalg.svd(x, full_matrices=False)
    s = s / (x.norm() + 1e-7)
    for _ in range(5):
        s = 3.4445 * s - 4.7750 * s ** 3 + 2.0315 * s ** 5
    assert torch.allclose(exact(x), u @ torch.diag(s) @ v, rtol=1e-10, atol=1e-10)


def test_sizes_whose_sums_would_overflow_are_refused():
    for bad in (dict(matrices=[(0, 3, 1)], ld=2 ** 62, row_strides=[2 ** 62]), dict(ld=2 ** 62, n_workers=4), dict(ld=2 ** 44, n_workers=5),
                dict(matrices=[(2 ** 46 - 1, 4, 5)], ld=2 ** 46), dict(matrices=[(2 ** 63 - 1, 4, 5)])):
        with pytest.raises(CSERError, match="2\\^46|reaches outside"):
            train.Orthogonalizer(**{**dict(matrices=[(0, 4, 5)], n_workers=1, ld=20), **bad})


def test_matrices_that_share_an_element_are_refused():
    for ms, strides in (([(0, 4, 5), (19, 1, 1)], None), ([(0, 4, 5), (0, 4, 5)], None), ([(10, 2, 5), (0, 2, 6)], None),
                        ([(0, 3, 2), (3, 3, 2)], [4, 4]), ([(0, 3, 2), (2, 3, 2), (9, 1, 1)], [4, 4, 1]), ([(0, 100, 1), (99, 1, 1)], [1, 1]),
                        ([(0, 5, 2), (2, 3, 2)], [4, 5])):
        with pytest.raises(CSERError, match="two matrices overlap"):
            train.Orthogonalizer(ms, 2, 100, row_strides=strides)


@pytest.mark.gpu
def test_columns_of_one_array_are_matrices_of_their_own():
    """Interleaved rows, which share no element."""
    gen = generator(21)
    u = torch.stack([matrix(gen, 90, 100 + 70) for _ in range(2)])
    got = train.Orthogonalizer([(0, 90, 100), (100, 90, 70)], 2, 90 * 170, row_strides=[170, 170]).apply(u.reshape(2, -1)).view(2, 90, 170)
    for i in range(2):
        assert far(got[i, :, :100], exact(u[i, :, :100])) < OUT[F32] and far(got[i, :, 100:], exact(u[i, :, 100:])) < OUT[F32]
