"""Group norm where there are more units of work than the GPU holds at a time, and the layers' streams, large offsets and use together.

The one-walk kernels keep their blocks and fetch the next unit into the places of this one: sizes here give every block several units, of
equal and of unequal length, for clusters of one block and more, and the results are those of the same samples alone.
"""
import pytest
import torch

from paper_2007_13221_b200 import layers

pytestmark = pytest.mark.gpu
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
LONG = 200_000_000                                    # cycles, about a tenth of a second: what is queued behind it runs late


def inputs(n, b, pixels, c, dtype, seed=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = (torch.randn((n, b, pixels, c), generator=gen, device="cuda") * 1.5 + torch.randn(c, generator=gen, device="cuda")).to(dtype)
    dy = torch.randn((n, b, pixels, c), generator=gen, device="cuda").to(dtype)
    return x, dy, torch.rand((n, c), generator=gen, device="cuda") + 0.5, torch.randn((n, c), generator=gen, device="cuda") * 0.3


# n, samples, pixels, channels, groups, type: clusters of 1, of 2, of 4 and of 8, slices whose last is narrower, groups wider than a slice's 64
# bytes, vectors of 8 and of 4 bytes
MANY = [(8, 60, 64, 256, 32, BF), (2, 200, 1024, 128, 32, BF), (4, 50, 1200, 192, 4, HF), (3, 60, 3136, 64, 32, BF), (2, 40, 5000, 36, 3, HF),
        (1, 40, 12544, 64, 32, HF), (2, 300, 77, 104, 13, F32), (8, 200, 1, 512, 32, BF), (4, 300, 9, 100, 25, BF), (1, 700, 400, 60, 2, F32)]


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("size", MANY, ids=str)
def test_many_units_equal_the_samples_alone(size, act):
    """A sample's result does not depend on what else the call has: bit for bit where it is cut alike, within rounding else."""
    n, b, pixels, c, groups, dtype = size
    x, dy, w, s = inputs(n, b, pixels, c, dtype)
    op = layers.GroupNorm(n, b, c, groups, act, dtype=dtype)
    y, stats = op.apply(x, w, s)
    dx, dw, db = op.grad(x, dy, stats, w, s)
    u = {BF: 2.0 ** -8, HF: 2.0 ** -11, F32: 2.0 ** -24}[dtype]
    hat = (x.double().view(n, b, pixels, groups, -1))
    mean = hat.mean((2, 4), keepdim=True)
    rstd = 1 / (hat.var((2, 4), keepdim=True, correction=0) + 1e-5).sqrt()
    hat = ((hat - mean) * rstd).view(x.shape)
    z = hat * w.double().view(n, 1, 1, c) + s.double().view(n, 1, 1, c)
    gate = torch.sigmoid(z)
    want = z * gate if act == "silu" else z
    # 64 roundings of values of up to 16 deviations before the result's own
    slack = 64 * 16 * 2.0 ** -24
    assert bool(((y.double() - want).abs() <= 1.01 * u * want.abs() + slack * (1 + want.abs()) + 2.0 ** -25).all())
    dz = dy.double() * (gate * (1 + z * (1 - gate)) if act == "silu" else 1)
    t = (dz * w.double().view(n, 1, 1, c)).view(n, b, pixels, groups, -1)
    h5 = hat.view(t.shape)
    wanted = ((t - t.mean((2, 4), keepdim=True) - h5 * (t * h5).mean((2, 4), keepdim=True)) * rstd).view(x.shape)
    size_dx = (rstd * (1 + h5.abs())).expand(t.shape).reshape(x.shape) * (1 + dy.double().abs()) * 4
    assert bool(((dx.double() - wanted).abs() <= 1.01 * u * wanted.abs() + slack * size_dx + 2.0 ** -25).all())
    for got, terms, size in ((db, dz, 1 + dy.double().abs()), (dw, dz * hat, (1 + dy.double().abs()) * (1 + hat.abs()))):
        assert bool(((got.double() - terms.sum((1, 2))).abs() <= (slack + 64 * 2.0 ** -24) * size.sum((1, 2))).all())
    again = op.apply(x, w, s)
    assert torch.equal(again[0], y) and torch.equal(again[1], stats)
    more = op.grad(x, dy, stats, w, s)
    assert all(torch.equal(p, q) for p, q in zip(more, (dx, dw, db)))
    few = layers.GroupNorm(n, 1, c, groups, act, dtype=dtype)
    for k in (0, b // 2, b - 1):
        one, st = few.apply(x[:, k:k + 1], w, s)
        assert bool(((one.double() - y[:, k:k + 1].double()).abs() <= 2.02 * u * one.double().abs() + 2 * slack * (1 + one.double().abs())).all())


@pytest.mark.parametrize("size", MANY[:7], ids=str)
def test_many_units_of_a_dropout(size):
    """The same as norm(dropout(x)) with the dropped array rounded to no fewer bits than it has: a factor of 2 rounds nothing."""
    n, b, pixels, c, groups, dtype = size
    x, dy, w, s = inputs(n, b, pixels, c, dtype, seed=1)
    drop = layers.Dropout(n, b * pixels, c, 0.5, 77, 9, dtype)
    dropped = drop.apply(x, 3)
    fused = layers.GroupNorm(n, b, c, groups, "silu", dtype=dtype, dropout=drop)
    plain = layers.GroupNorm(n, b, c, groups, "silu", dtype=dtype)
    y, stats = fused.apply(x, w, s, step=3)
    y2, stats2 = plain.apply(dropped, w, s)
    u = {BF: 2.0 ** -8, HF: 2.0 ** -11, F32: 2.0 ** -24}[dtype]
    slack = 128 * 16 * 2.0 ** -24
    assert bool(((stats - stats2).abs() <= slack * (1 + stats2.abs())).all())
    assert bool(((y.double() - y2.double()).abs() <= 2.02 * u * y2.double().abs() + slack * (1 + y2.double().abs())).all())
    got = fused.grad(x, dy, stats, w, s, step=3)
    want = plain.grad(dropped, dy, stats2, w, s)
    through = drop.grad(want[0], 3)[0]
    size_dx = 2 * (1 + dy.double().abs()) * (1 + through.double().abs()) * 8
    assert bool(((got[0].double() - through.double()).abs() <= 3.03 * u * through.double().abs() + slack * size_dx).all())
    for g, p in zip(got[1:], want[1:]):
        assert bool(((g - p).abs() <= slack * pixels * b).all())


def test_more_than_2_31_elements():
    """Offsets beyond 32 bits, at both ends of arrays of 2^31 + 2^20 elements, against the same places in small calls."""
    n, rows, cols = 1, 2 ** 21 + 2 ** 10, 1024
    x = torch.zeros((n, rows, cols), dtype=BF, device="cuda")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    head, tail = torch.randn((64, cols), generator=gen, device="cuda").to(BF), torch.randn((64, cols), generator=gen, device="cuda").to(BF)
    x[0, :64], x[0, -64:] = head, tail
    op = layers.Dropout(n, rows, cols, 0.25, 5, 6)
    y = op.apply(x, 11)
    kept = y[0, -64:] != 0
    assert torch.equal(y[0, :64], layers.Dropout(1, 64, cols, 0.25, 5, 6).apply(head[None], 11)[0])
    assert bool((y[0, 64:-64] == 0).all())
    dx, db = op.grad(x, 11, need_dbias=True)
    assert torch.equal(dx, y)
    want = y[0, :64].double().sum(0) + y[0, -64:].double().sum(0)
    size = y[0, :64].double().abs().sum(0) + y[0, -64:].double().abs().sum(0)
    assert bool(((db[0].double() - want).abs() <= size * (2.0 ** -8 + 1e-5)).all())
    import numpy as np
    from oracle.philox import philox4x32_10
    first = (rows - 64) * cols
    q = np.arange(first // 4, rows * cols // 4, dtype=np.uint64)
    words = np.stack(philox4x32_10(5, 0, q, 11, 0, 4096 * 6), 1).reshape(64, cols)
    assert torch.equal(kept, torch.from_numpy(words >= 2 ** 30).cuda() & (tail != 0))
    del y, dx
    norm = layers.GroupNorm(1, rows // 2, cols, 8, "silu")
    z, stats = norm.apply(x.view(1, rows // 2, 2, cols))
    part = layers.GroupNorm(1, 32, cols, 8, "silu").apply(x.view(1, rows // 2, 2, cols)[:, -32:])
    assert bool(((z[:, -32:].double() - part[0].double()).abs() <= 2.0 ** -7 * part[0].double().abs() + 1e-4).all())
    assert bool((z[:, 32:-32] == 0).all())
    grads = norm.grad(x.view(1, rows // 2, 2, cols), z, stats)
    assert bool(grads[0][:, 32:-32].isfinite().all()) and bool((grads[0][:, 32:-32] == 0).all())


def test_calls_on_another_stream():
    """Results are made on the stream; inputs may be dropped after the call, results while the current stream reads them."""
    x, dy, w, s = inputs(2, 6, 300, 64, BF)
    drop = layers.Dropout(2, 6 * 300, 64, 0.3, 1, 2)
    norm = layers.GroupNorm(2, 6, 64, 8, "silu", dropout=drop)
    xs, dys = x.view(2, 1800, 64), dy.view(2, 1800, 64)

    def calls(x, dy, w, s, stream=None):
        y, stats = norm.apply(x, w, s, step=4, stream=stream)
        a = drop.apply(x.view(2, 1800, 64), 4, bias=w, residual=dy.view(2, 1800, 64), stream=stream)
        return (y, stats, a, *norm.grad(x, dy, stats, w, s, step=4, stream=stream),
                *drop.grad(dy.view(2, 1800, 64), 4, need_dbias=True, stream=stream))

    want = calls(x, dy, w, s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    old = [torch.empty_like(a) for a in want]
    torch.cuda._sleep(LONG)
    for a in old:
        a.fill_(7)
    del old                                             # memory that the current stream writes late and its pool gives out at once
    got = calls(x, dy, w, s, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    args = [a.clone() for a in (x, dy, w, s)]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(LONG)
    got = calls(*args, stream=side)
    shapes = [torch.empty_like(a) for a in args]
    del args
    junk = [torch.full_like(a, 3) for a in shapes for _ in range(3)]
    torch.cuda.synchronize()
    del junk
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda._sleep(LONG)
    read = [a.clone() for a in got]
    del got
    with torch.cuda.stream(side):
        junk = [torch.full_like(a, 3) for a in read for _ in range(3)]
    torch.cuda.synchronize()
    del junk
    assert all(torch.equal(a, b) for a, b in zip(read, want))
    assert xs.data_ptr() == x.data_ptr() and dys.data_ptr() == dy.data_ptr()


def test_calls_behind_one_another_and_captured():
    """Kernels are set up while the ones before them end: a chain of calls on the same buffers, replayed and not, gives the same bits."""
    n, b, pixels, c = 2, 40, 49, 96
    x, dy, w, s = inputs(n, b, pixels, c, BF, seed=5)
    drop = layers.Dropout(n, b * pixels, c, 0.3, 1, 2)
    norm = layers.GroupNorm(n, b, c, 12, "silu")
    flat, grads = torch.zeros((n, 500), device="cuda"), torch.zeros((n, 500), device="cuda")
    flat[:, 3:3 + c], flat[:, 200:200 + c] = w, s
    weight, bias, dweight, dbias = flat[:, 3:3 + c], flat[:, 200:200 + c], grads[:, 3:3 + c], grads[:, 200:200 + c]
    h, out, dx = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)

    def chain():
        drop.apply(x, 8, out=h)
        for _ in range(3):
            _, stats = norm.apply(h, weight, bias, out=out)
            norm.grad(h, dy, stats, weight, bias, dx=dx, dweight=dweight, dbias=dbias)
            drop.apply(dx, 9, residual=out, out=h)
        drop.grad(h, 10, dx=dx, dbias=grads[:, 400:400 + c])

    chain()
    torch.cuda.synchronize()
    want = [a.clone() for a in (h, out, dx, grads)]
    for _ in range(5):
        chain()
    assert all(torch.equal(a, b) for a, b in zip((h, out, dx, grads), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        chain()
    for a in (h, out, dx, grads):
        a.zero_()
    for _ in range(3):
        graph.replay()
    assert all(torch.equal(a, b) for a, b in zip((h, out, dx, grads), want))


def test_a_handle_may_go_while_a_graph_is_captured():
    x, dy, w, s = inputs(1, 2, 9, 16, BF)
    norm, other, drop = layers.GroupNorm(1, 2, 16, 4), layers.GroupNorm(1, 2, 16, 4), layers.Dropout(1, 18, 16, 0.5, 1, 1)
    want = norm.apply(x, w, s)[0]
    out = torch.zeros_like(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        other.close()
        norm.apply(x, w, s, out=out)
        del drop
    graph.replay()
    assert torch.equal(out, want) and other.h is None


def test_between_the_other_operators():
    """Behind and before the cross entropy, whose kernels too are set up while the ones before them end: the same bits as one after the other."""
    from paper_2007_13221_b200 import train
    n, t, v, d = 2, 96, 700, 128
    gen = torch.Generator(device="cuda")
    gen.manual_seed(9)
    x = torch.randn((n, t, d), generator=gen, device="cuda").to(BF)
    w = (torch.randn((n, v, d), generator=gen, device="cuda") * 0.1).to(BF)
    y = torch.randint(0, v, (n, t), generator=gen, device="cuda")
    mean = torch.full((n, t), 1.0 / t, device="cuda")
    drop, head = layers.Dropout(n, t, d, 0.2, 3, 1), train.LinearCrossEntropy(n, t, v, d)
    norm = layers.GroupNorm(n, t, d, 4, "silu")

    def step(wait):
        out = []
        h, stats = norm.apply(x.view(n, t, 1, d))
        wait()
        h = drop.apply(h.view(n, t, d), 6, residual=x)
        wait()
        loss, lse = head.loss(h, w, y)
        wait()
        dh, dw = head.grad(h, w, y, lse, mean)
        wait()
        dz, db = drop.grad(dh, 6, need_dbias=True)
        wait()
        out += [loss, dw, dz, db, *norm.grad(x.view(n, t, 1, d), dz.view(n, t, 1, d), stats)]
        return out

    want = step(torch.cuda.synchronize)
    for _ in range(20):
        got = step(lambda: None)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_sample_of_so_many_pixels_that_no_thread_has_slots_for_its_own():
    """More than 2^16 pixels a thread of a cluster: three kernels forward.  A thread of theirs has about 112 pixels, then 600 parts are joined."""
    from test_layers import check_norm, norm_inputs
    x, weight, bias, dy = norm_inputs(11, 1, 1, (530000,), 127, F32)
    op = layers.GroupNorm(1, 1, 127, 1, "silu", dtype=F32)
    check_norm(op, x, weight, bias, dy, 1, "silu", chain=256)
    assert op.launches == 3 + 4


@pytest.mark.parametrize("size", [(1, 1, 100, 1024, 1, BF), (1, 2, 104, 600, 2, HF), (1, 1, 101, 512, 1, F32)], ids=str)
def test_few_samples_of_wide_groups(size):
    """Gradients whose blocks' shared memory is nearly used up."""
    from test_layers import check_norm, norm_inputs
    n, b, pixels, c, groups, dtype = size
    x, weight, bias, dy = norm_inputs(12, n, b, (pixels,), c, dtype)
    check_norm(layers.GroupNorm(n, b, c, groups, "silu", dtype=dtype), x, weight, bias, dy, groups, "silu")


@pytest.mark.parametrize("dtype", [BF, F32], ids=str)
@pytest.mark.parametrize("size", [(1, 1, 2 ** 20 + 1), (8, 1, 1001), (2, 5, 4099), (3, 7, 1001), (3, 8, 1001), (1, 100, 10001)], ids=str)
def test_few_rows_of_columns_that_no_vector_divides(size, dtype):
    """Against the formula; a call with fewer rows than the handle is for sums as many."""
    from test_layers import SEED, check_drop, gen_of, mask, normal
    n, rows, cols = size
    gen = gen_of(13)
    x, r, dy = (normal(gen, *size).to(dtype) for _ in range(3))
    bias = normal(gen, n, cols)
    for most in (rows, 9 * rows):
        check_drop(layers.Dropout(n, most, cols, 0.3, SEED, 3, dtype), x, bias, r, dy, 0.3, mask(n, rows * cols, 0.3))


def test_a_handle_for_one_wide_row_takes_no_memory():
    layers.Dropout(1, 1, 8, 0.1, 0, 1).close()          # what the library takes once
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    op = layers.Dropout(1, 1, 2 ** 25 + 1, 0.1, 0, 1)
    assert before - torch.cuda.mem_get_info()[0] < 2 ** 23          # (another process's share of the card may move a little)
    op.close()


def test_arrays_that_share_memory_are_refused():
    """But a result in an input's place; columns of one wider array lie beside each other and share nothing."""
    from paper_2007_13221_b200.binding import CSERError
    n, rows, cols = 2, 12, 16
    room = torch.zeros(4 * n * rows * cols, device="cuda", dtype=F32)
    count = n * rows * cols
    drop, norm = layers.Dropout(n, rows, cols, 0.5, 0, 1, F32), layers.GroupNorm(n, 3, cols, 4, dtype=F32)

    def array(at, shape=(n, rows, cols)):
        return room[at:at + count].view(shape)

    def image(at):
        return array(at, (n, 3, 4, cols))

    params, far = torch.zeros((n, cols), device="cuda"), array(2 * count)
    y, stats = norm.apply(image(0))
    inside = room[5 * cols:5 * cols + n * cols].view(n, cols)
    wide = torch.zeros((n, rows, 3 * cols), device="cuda")
    halves = wide[..., :cols], wide[..., cols:2 * cols], wide[..., cols - 4:2 * cols - 4]
    calls = [lambda: drop.apply(array(0), 1, out=array(4)), lambda: drop.apply(array(cols), 1, out=array(0)),
             lambda: drop.apply(far, 1, residual=array(0), out=array(8)), lambda: drop.apply(far, 1, bias=inside, out=array(0)),
             lambda: drop.grad(array(0), 1, dx=array(count - 4)), lambda: drop.grad(array(0), 1, need_dx=False, dbias=inside),
             lambda: drop.grad(far, 1, dx=array(0), dbias=inside), lambda: drop.apply(halves[0], 1, out=halves[2]),
             lambda: norm.apply(image(0), out=image(4)), lambda: norm.apply(image(2 * count), weight=inside, out=image(0)),
             lambda: norm.grad(image(0), image(2 * count), stats, dx=image(4)), lambda: norm.grad(image(2 * count), image(0), stats, dx=image(4)),
             lambda: norm.grad(image(0), image(count), stats, dweight=inside), lambda: norm.grad(image(0), image(count), stats, dweight=params, dbias=params),
             lambda: norm.grad(image(0), image(count), stats, weight=params, dweight=params),
             lambda: norm.grad(image(0), image(count), stats, dx=image(2 * count), dbias=far.view(-1)[:n * cols].view(n, cols))]
    for call in calls:
        with pytest.raises(CSERError, match="share memory"):
            call()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    halves[0].copy_(torch.randn((n, rows, cols), generator=gen, device="cuda"))
    want = drop.apply(halves[0].contiguous(), 1)
    assert torch.equal(drop.apply(halves[0], 1, out=halves[1]), want)
    assert torch.equal(drop.apply(halves[0], 1, out=halves[0]), want)
    assert torch.equal(drop.apply(array(0), 1, out=array(count)), drop.apply(array(0), 1))


def test_an_error_that_was_reported_stays_behind():
    """A handle too large for the GPU is refused, and the next call of any kind does not hear of it."""
    from paper_2007_13221_b200 import binding, train
    from paper_2007_13221_b200.binding import CSERError
    opt = binding.CSER(1000, 2, 16, R1=4, R2=2, H=4, eta=0.1, beta=0.9, flags=binding.FLAG_THREE_KERNELS)
    opt.set_x0(torch.zeros(1000, device="cuda"))
    grad = torch.ones((2, 1000), device="cuda")
    for make in (lambda: layers.GroupNorm(4096, 4096, 65536, 1), lambda: layers.Dropout(4096, 2 ** 20, 2 ** 14, 0.1, 0, 1),
                 lambda: train.LinearCrossEntropy(1, 2 ** 24, 2 ** 22, 64, piece=2 ** 22)):
        with pytest.raises(CSERError):
            make()
        opt.step(grad)
    opt.close()
