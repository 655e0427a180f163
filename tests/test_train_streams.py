"""The operators' `stream` argument: the call runs on a stream that is not torch's current one.

Results are made on that stream, and the allocator is told who uses what: memory of inputs, given results and made results is not given out
again while either stream may still use it.
"""
import pytest
import torch

from paper_2007_13221_b200 import binding, train

pytestmark = pytest.mark.gpu
LONG = 200_000_000                                    # cycles, about a tenth of a second: what is queued behind it runs late


def orth():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    g = torch.randn((2, 4096), generator=gen, device="cuda")
    op = train.Orthogonalizer([(0, 40, 70), (3000, 30, 30)], 2, 4096)
    return op, g, op.apply(g)


def xent():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    h = torch.randn((2, 64, 256), generator=gen, device="cuda").bfloat16()
    w = (torch.randn((2, 500, 256), generator=gen, device="cuda") / 16).bfloat16()
    y = torch.randint(0, 500, (2, 64), generator=gen, device="cuda")
    dloss = torch.rand((2, 64), generator=gen, device="cuda")
    op = train.LinearCrossEntropy(2, 64, 500, 256)
    loss, lse = op.loss(h, w, y)
    return op, (h, w, y), dloss, (loss, lse), op.grad(h, w, y, lse, dloss)


def stale(*like):
    """Memory that the current stream writes late and that its pool gives out again at once."""
    old = [torch.empty_like(a) for a in like]
    torch.cuda._sleep(LONG)
    for a in old:
        a.fill_(7)


def test_orth_result_is_made_on_the_stream():
    op, g, want = orth()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    torch.cuda._sleep(LONG)
    got = op.apply(g, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_xent_results_are_made_on_the_stream():
    op, x, dloss, (loss, lse), grads = xent()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    stale(loss, lse)
    got = op.loss(*x, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got[0], loss) and torch.equal(got[1], lse)
    stale(*grads)
    got = op.grad(*x, lse, dloss, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, grads))


def test_inputs_may_be_dropped_after_the_call():
    op, (h, w, y), dloss, (loss, lse), grads = xent()
    side = torch.cuda.Stream()
    for k in range(3):
        args = [a.clone() for a in (h, w, y)]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(LONG)
        got = op.loss(*args, stream=side)
        like = args[k]
        del args
        junk = [torch.full_like(like, 3) for _ in range(4)]
        torch.cuda.synchronize()
        del junk
        assert torch.equal(got[0], loss) and torch.equal(got[1], lse)
    args, dw = [a.clone() for a in (lse, dloss)], torch.empty_like(w)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(LONG)
    got = op.grad(h, w, y, *args, dweight=dw, stream=side)
    del args
    junk = [torch.full_like(lse, 3) for _ in range(4)]
    torch.cuda.synchronize()
    del junk
    assert torch.equal(got[0], grads[0]) and torch.equal(dw, grads[1])
    op, g, want = orth()
    arg = g.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(LONG)
    got = op.apply(arg, stream=side)
    del arg
    junk = [torch.full_like(g, 3) for _ in range(4)]
    torch.cuda.synchronize()
    del junk
    assert torch.equal(got, want)


def test_results_may_be_dropped_while_the_current_stream_reads_them():
    op, x, dloss, (loss, lse), grads = xent()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = [*op.loss(*x, stream=side), *op.grad(*x, lse, dloss, stream=side)]
    torch.cuda.synchronize()
    torch.cuda._sleep(LONG)
    read = [a.clone() for a in got]
    del got
    with torch.cuda.stream(side):
        junk = [torch.full_like(a, 3) for a in read for _ in range(3)]
    torch.cuda.synchronize()
    del junk
    assert all(torch.equal(a, b) for a, b in zip(read, (loss, lse, *grads)))


def test_streams_of_other_packages():
    """Anything with a cuda_stream, as the optimizer's calls take."""
    class Stream:
        def __init__(self, raw):
            self.cuda_stream = raw

    op, g, want = orth()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for s in (Stream(side.cuda_stream), torch.cuda.ExternalStream(side.cuda_stream)):
        torch.cuda._sleep(LONG)
        got = op.apply(g, stream=s)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_the_current_stream_by_name():
    """The stream that is current anyway, given or not."""
    op, g, want = orth()
    assert torch.equal(op.apply(g, stream=torch.cuda.current_stream()), want)
    op, x, dloss, (loss, lse), grads = xent()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = op.loss(*x, stream=side)
        b = op.grad(*x, a[1], dloss, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(a[0], loss) and all(torch.equal(p, q) for p, q in zip(b, grads))


def test_a_handle_may_go_while_a_graph_is_captured():
    """Closed or collected; it is destroyed with the next one that goes."""
    op, g, want = orth()
    closed, dropped = (train.Orthogonalizer([(0, 40, 70), (3000, 30, 30)], 2, 4096) for _ in range(2))
    head, step, after = train.LinearCrossEntropy(2, 8, 30, 16), binding.CSER(1000, 2, 100, 2, 2, 2, 0.1, 0.9), train.LinearCrossEntropy(1, 8, 30, 16)
    out = torch.zeros_like(g)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        closed.close()
        op.apply(g, out)
        del dropped, head
        step.close()
    graph.replay()
    assert torch.equal(out, want) and closed.h is None and step.h is None and len(binding._waiting) >= 4
    after.close()
    assert binding._waiting == []
