"""The layers together with the optimizer step, as a training step uses them: against a 64-bit model differentiated by torch."""
import os
import sys

import numpy as np
import pytest
import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
pytestmark = pytest.mark.gpu


def exact(flat, x, label, keep):
    """Losses and the flat gradient in 64 bits."""
    import wide_residual_step as ex
    n = ex.WORKERS
    p = flat.double().requires_grad_()
    loss = []

    def norm(v, w, b):                                  # [images, channels, side, side]
        return F.silu(F.group_norm(v, ex.GROUPS, w, b, 1e-5))

    for i in range(n):
        q = {k: ex.view(p, k)[i] for k in ex.shapes()[0]}
        v = x[i].double().permute(0, 3, 1, 2)
        c = F.conv2d(norm(v, q["weight1"], q["bias1"]), q["conv1"], padding=1)
        m = keep[i].view(ex.IMAGES, ex.SIDE, ex.SIDE, ex.CHANNELS).permute(0, 3, 1, 2)
        b = norm(c * m / (1 - ex.P), q["weight2"], q["bias2"])
        h = v + F.conv2d(b, q["conv2"], padding=1)
        loss.append(F.cross_entropy(h.mean((2, 3)) @ q["head"].t(), label[i]))
    loss = torch.stack(loss)
    loss.sum().backward()
    return loss.detach(), p.grad


def test_gradients_against_64_bits():
    """The whole step's gradient.  Each of its about twenty products and layers rounds sums of up to 1024 terms in 32 bits, 2^-24 sqrt(1024)
    of their size at most where roundings are independent: 20 * 2^-19 of each parameter's gradient in the 2-norm, and ten times that
    for what a layer passes on of the errors before it."""
    import wide_residual_step as ex
    from oracle.philox import philox4x32_10
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    d = ex.shapes()[1]
    flat = ex.start(gen) + 0.05 * torch.randn((ex.WORKERS, d), generator=gen, device="cuda")
    x = torch.randn((ex.WORKERS, ex.IMAGES, ex.SIDE, ex.SIDE, ex.CHANNELS), generator=gen, device="cuda")
    label = torch.randint(0, ex.CLASSES, (ex.WORKERS, ex.IMAGES), generator=gen, device="cuda")
    count, step, seed = x[0].numel(), 17, 3
    keep = torch.from_numpy(np.stack([np.stack(philox4x32_10(seed, 0, np.arange(count // 4, dtype=np.uint64), step, 0, 4096 * ex.SITE + i), 1)
                                      .reshape(-1) >= int(ex.P * 2 ** 32) for i in range(ex.WORKERS)])).cuda().double()
    before = torch.backends.cudnn.allow_tf32
    torch.backends.cudnn.allow_tf32 = False
    try:
        grad = torch.full((ex.WORKERS, d), 7.0, device="cuda")
        loss = ex.Block(seed).gradient(flat, x, label, step, grad)
    finally:
        torch.backends.cudnn.allow_tf32 = before
    want_loss, want = exact(flat, x, label, keep)
    assert bool(((loss.double() - want_loss).abs() <= 200 * 2.0 ** -19 * (1 + want_loss)).all())
    for name in ex.shapes()[0]:
        got, w = ex.view(grad, name).double(), ex.view(want, name)
        assert float((got - w).norm() / w.norm()) < 200 * 2.0 ** -19, name


def test_steps_run_and_repeat():
    import wide_residual_step as ex
    a = ex.run(6)
    assert len(a) == 6 and all(v == v for v in a)
