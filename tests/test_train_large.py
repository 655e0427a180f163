"""The operators on arrays of more than 2^31 elements: places past 32 bits in every array they read and write.

Tolerances as in test_xent.py and test_orth.py, whose exact forms would not fit: the vocabulary is gone through in pieces here, and
an orthogonalised matrix is compared by its products with a few vectors.
"""
import pytest
import torch

from paper_2007_13221_b200 import train

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
FAR = 2 ** 31


@pytest.fixture(autouse=True)
def free_memory():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def fill(a, gen, scale):
    """Random rows, a part of them at a time."""
    flat = a.view(-1)
    for k in range(0, flat.numel(), 1 << 27):
        part = flat[k:k + (1 << 27)]
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda") * scale)
    return a


@pytest.mark.parametrize("pad", [0, 3], ids=["read in place", "packed"])
def test_weights_and_their_gradient(pad):
    """Two workers of 70000 x 16376, hidden rows 2^31 elements apart; with rows of odd length the operands are packed first."""
    n, t, v, d = 2, 2, 70000, 16376
    gen = torch.Generator(device="cuda")
    gen.manual_seed(pad)
    w = fill(torch.empty((n, v, d + pad), dtype=BF, device="cuda"), gen, 2 / d ** 0.5)[..., :d]
    assert w.stride(0) * n > FAR
    y = torch.tensor([[v - 1, 3], [0, v - 2]], device="cuda")
    h0 = torch.stack([torch.randn((t, d), generator=gen, device="cuda") + 2 * w[i][y[i]].float() for i in range(n)]).to(BF)
    apart = FAR + 8 + pad
    h = torch.empty(apart + 2 * d, dtype=BF, device="cuda").as_strided((n, t, d), (d, apart, 1))
    h.copy_(h0)
    dloss = torch.tensor([[1.0, -0.5], [0.25, 2.0]], device="cuda")
    op = train.LinearCrossEntropy(n, t, v, d)
    loss, lse = op.loss(h, w, y)
    flat = torch.full((n, v * d + 5), 7, dtype=BF, device="cuda")
    dw = flat.as_strided((n, v, d), (v * d + 5, d, 1))
    dh, _ = op.grad(h, w, y, lse, dloss, dweight=dw)
    assert bool((flat[:, v * d:] == 7).all())
    u = 2.0 ** -8
    for i in range(n):
        hi = h0[i].double()
        z = torch.cat([hi @ w[i, k:k + 5000].double().t() for k in range(0, v, 5000)], 1)
        l = torch.logsumexp(z, 1)
        assert bool(((lse[i].double() - l).abs() <= 1e-5 * (1 + l.abs())).all())
        assert bool(((loss[i].double() - (l - z.gather(1, y[i][:, None])[:, 0])).abs() <= 1e-5 * (1 + l.abs())).all())
        p = torch.exp(z - l[:, None])
        dz = p.clone()
        dz[torch.arange(t), y[i]] -= 1
        g = dloss[i].double()[:, None]
        dz *= g
        off = u * dz.abs() + 2e-5 * (1 + l.abs())[:, None] * p * g.abs()
        want_dh, bound_dh = torch.zeros_like(hi), torch.zeros_like(hi)
        for k in range(0, v, 5000):
            part = w[i, k:k + 5000].double()
            want_dh += dz[:, k:k + 5000] @ part
            bound_dh += off[:, k:k + 5000] @ part.abs()
            want = dz[:, k:k + 5000].t() @ hi
            bound = 1.1 * (off[:, k:k + 5000].t() @ hi.abs() + u * want.abs())
            assert bool(((dw[i, k:k + 5000].double() - want).abs() <= bound).all())
        assert bool(((dh[i].double() - want_dh).abs() <= 1.1 * (bound_dh + u * want_dh.abs())).all())


def exact(u):
    x = u.double()
    x = x / (x.square().sum().sqrt() + 1e-7)
    for _ in range(5):
        k = x.t() @ x
        x = 3.4445 * x + x @ (-4.7750 * k + 2.0315 * (k @ k))
    return x


@pytest.mark.parametrize("out_t", [BF, F32], ids=str)
def test_matrices_far_inside_a_vector(out_t):
    """Every kind of matrix (tiled, by Gram matrix, by one CTA) beyond 2^31 elements, with momentum; what lies between stays."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    plan = [(FAR - 100, 150, 200, 200), (FAR + 40001, 300, 129, 140), (FAR + 100000, 33, 1000, 1000), (FAR + 150000, 16, 500, 500)]
    ld = FAR + 160000
    grad = torch.zeros((1, ld), dtype=BF, device="cuda")
    m = torch.zeros((1, ld), device="cuda")
    grad[0, FAR - 1000:] = (torch.randn(ld - FAR + 1000, generator=gen, device="cuda") * 0.02).to(BF)
    m[0, FAR - 1000:] = torch.randn(ld - FAR + 1000, generator=gen, device="cuda") * 0.02
    m0 = m[0, FAR - 1000:].clone()
    out = torch.full((1, ld), 7, dtype=out_t, device="cuda")
    train.Orthogonalizer([p[:3] for p in plan], 1, ld, BF, out_t, row_strides=[p[3] for p in plan]).apply(grad, out, momentum=m, mu=0.9)
    touched = torch.zeros(ld - FAR + 1000, dtype=torch.bool, device="cuda")
    for at, r, c, st in plan:
        where = at - FAR + 1000 + torch.arange(r, device="cuda")[:, None] * st + torch.arange(c, device="cuda")[None, :]
        touched[where.reshape(-1)] = True
        g, new = grad[0, FAR - 1000:][where].double(), m[0, FAR - 1000:][where].double()
        want_m = 0.9 * m0[where].double() + g
        assert torch.allclose(new, want_m, rtol=2.0 ** -22, atol=2.0 ** -24 * 0.1)
        want = exact(g + 0.9 * want_m)
        assert float((out[0, FAR - 1000:][where].double() - want).norm() / want.norm()) < (2e-3 + 2.0 ** -8 if out_t == BF else 5e-6)
    assert bool((out[0, FAR - 1000:][~touched] == 7).all()) and torch.equal(m[0, FAR - 1000:][~touched], m0[~touched])
    assert bool((out[0, :FAR - 1000] == 7).all()) and not bool(m[0, :FAR - 1000].any())


def test_one_matrix_of_more_than_2_31_elements():
    """65536 x 32800, one step: out v = a X v + b X K v + c X K K v with K = X^T X, for a few vectors v."""
    r, c = 65536, 32800
    assert r * c > FAR
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    g = fill(torch.empty((1, r * c), dtype=BF, device="cuda"), gen, 0.01)
    row, col = torch.randn((r, 2), generator=gen, device="cuda"), torch.randn((2, c), generator=gen, device="cuda")
    x = g.view(r, c)
    for k in range(0, r, 8192):                       # a part of low rank, so that the singular values differ
        x[k:k + 8192] += (0.01 * row[k:k + 8192] @ col).to(BF)
    out = train.Orthogonalizer([(0, r, c)], 1, r * c, BF, BF, steps=1).apply(g).view(r, c)
    parts = range(0, r, 8192)
    norm = sum(float(x[k:k + 8192].double().square().sum()) for k in parts) ** 0.5 + 1e-7

    def times(a, v):                                  # a v, and a^T v
        return torch.cat([a[k:k + 8192].double() @ v for k in parts])

    def times_t(a, v):
        return sum(a[k:k + 8192].double().t() @ v[k:k + 8192] for k in parts)

    v = torch.randn((c, 3), generator=gen, device="cuda").double()
    v[:, 2] = col[0].double()
    k1 = times_t(x, times(x, v)) / norm ** 2
    k2 = times_t(x, times(x, k1)) / norm ** 2
    want = (3.4445 * times(x, v) - 4.7750 * times(x, k1) + 2.0315 * times(x, k2)) / norm
    err = (times(out, v) - want).norm(dim=0) / want.norm(dim=0)
    assert bool((err < 2e-3 + 2.0 ** -8).all())
