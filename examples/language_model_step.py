"""Training steps of a small language model on n simulated workers, through the three parts that the library has for it.

Each worker holds its own model x_i = (hidden matrix W [D, D], head H [V, D]) in the optimizer's [n, d] state and sees its
own tokens.  A step is
    loss, dhidden, dH   linear cross entropy of the head, per worker          (train.LinearCrossEntropy)
    dW                  = inputs^T dhidden
    update of W         orthogonalised, with momentum                         (train.Orthogonalizer, straight into the flat gradient)
    x <- x - eta * ...  partial synchronisation and error reset              (binding.CSER)
The text is synthetic: each token is followed by one fixed successor, or, one time in ten, by any token.

    python examples/language_model_step.py [steps]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2007_13221_b200 import binding, train  # noqa: E402

WORKERS, TOKENS, VOCAB, DIM = 4, 512, 2000, 256


def run(steps=60, seed=0, report=None):
    """Mean loss over the workers at each step."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    embed = torch.randn((VOCAB, DIM), generator=gen, device="cuda").bfloat16()
    successor = torch.randperm(VOCAB, generator=gen, device="cuda")
    split, d = DIM * DIM, DIM * DIM + VOCAB * DIM
    x0 = torch.cat([torch.eye(DIM, device="cuda").reshape(-1),
                    torch.randn(VOCAB * DIM, generator=gen, device="cuda") * 0.02])

    opt = binding.CSER(d, WORKERS, 1024, R1=4, R2=2, H=4, eta=0.02, beta=0.0, seed=seed)
    opt.set_x0(x0)
    head_loss = train.LinearCrossEntropy(WORKERS, TOKENS, VOCAB, DIM)
    # The orthogonalised matrix has singular values near 1 whatever its gradient's size; 0.2 sqrt(D) gives its entries 0.2.
    orth = train.Orthogonalizer([(0, DIM, DIM)], WORKERS, d, scales=[0.2 * DIM ** 0.5])
    grad = torch.zeros((WORKERS, d), device="cuda")
    momentum = torch.zeros_like(grad)
    mean = torch.full((WORKERS, TOKENS), 1.0 / TOKENS, device="cuda")

    losses = []
    for step in range(steps):
        token = torch.randint(0, VOCAB, (WORKERS, TOKENS), generator=gen, device="cuda")
        target = successor[token]
        any_token = torch.randint(0, VOCAB, target.shape, generator=gen, device="cuda")
        target = torch.where(torch.rand(target.shape, generator=gen, device="cuda") < 0.1, any_token, target)

        x = opt.state(binding.STATE_X)
        w = x[:, :split].view(WORKERS, DIM, DIM).bfloat16()
        head = x[:, split:].view(WORKERS, VOCAB, DIM).bfloat16()
        inputs = embed[token]
        hidden = inputs @ w
        loss, lse = head_loss.loss(hidden, head, target)
        dhidden, dhead = head_loss.grad(hidden, head, target, lse, mean)

        grad[:, :split] = (inputs.transpose(1, 2) @ dhidden).float().view(WORKERS, split)
        orth.apply(grad, grad, momentum=momentum, mu=0.9)             # the matrix only; the head's part is not touched
        grad[:, split:] = dhead.float().view(WORKERS, -1) * 200.0     # the head's own step size, relative to eta
        opt.step(grad)
        losses.append(float(loss.mean()))
        if report:
            report(step, losses[-1])
    opt.close()
    return losses


if __name__ == "__main__":
    n = int(sys.argv[1]) if len(sys.argv) > 1 else 60
    run(n, report=lambda s, v: print(f"step {s:4d}  loss {v:.4f}") if s % 10 == 0 or s + 1 == n else None)
