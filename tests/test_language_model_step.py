"""The operators together, as a training step uses them: loss and gradient, orthogonalised update, optimizer step."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.gpu
def test_training_steps_learn_and_repeat():
    import language_model_step as example
    a = example.run(40)
    assert a[0] > 6.0 and all(v == v for v in a)
    assert a[-1] < a[0] - 1.5, a
    assert example.run(8) == a[:8]


@pytest.mark.gpu
def test_the_update_reaches_every_worker_as_the_step_defines_it():
    """One step with everything selected and no reset: x = x0 - eta * mean over workers of what was put into the gradient."""
    from paper_2007_13221_b200 import binding, train
    n, r, c, rest = 3, 96, 160, 40
    d = r * c + rest
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    grad = torch.randn((n, d), generator=gen, device="cuda")
    x0 = torch.randn(d, generator=gen, device="cuda")
    update = train.Orthogonalizer([(0, r, c)], n, d).apply(grad, grad.clone())
    assert torch.equal(update[:, r * c:], grad[:, r * c:])
    opt = binding.CSER(d, n, 64, R1=1, R2=1, H=100, eta=0.1, beta=0.0)
    opt.set_x0(x0)
    opt.step(update)
    want = x0 - (0.1 * update).double().mean(0)
    assert torch.allclose(opt.state(binding.STATE_X).double(), want.expand(n, -1), rtol=1e-6, atol=1e-7)
    opt.close()
