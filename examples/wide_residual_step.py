"""Training steps of a wide residual block on n simulated workers, with the layers that the library has for what stands between the products.

Each worker holds its own model in the optimizer's [n, d] state, channels last:
    a = silu(norm(x)) ;  c = conv1(a) ;  b = silu(norm(dropout(c))) ;  h = x + conv2(b) ;  loss = cross entropy of head(mean of h over the pixels)
The second norm reads the dropout's result without a pass of its own (layers.GroupNorm with a dropout); norms take their weights and biases
from the flat state and leave their gradients in the flat gradient, which binding.CSER.step communicates and applies.  The convolutions
are torch's.  The images are synthetic: a pattern for each class, and noise.

    python examples/wide_residual_step.py [steps]
"""
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2007_13221_b200 import binding, layers  # noqa: E402

WORKERS, IMAGES, SIDE, CHANNELS, GROUPS, CLASSES, P, SITE = 4, 16, 8, 64, 16, 10, 0.3, 1


def shapes():
    """Name, place and shape of each parameter in a worker's vector, and the vector's length."""
    c, at, got = CHANNELS, 0, {}
    for name, shape in (("conv1", (c, c, 3, 3)), ("conv2", (c, c, 3, 3)), ("head", (CLASSES, c)), ("weight1", (c,)), ("bias1", (c,)),
                        ("weight2", (c,)), ("bias2", (c,))):
        size = 1
        for s in shape:
            size *= s
        got[name] = (at, size, shape)
        at += size
    return got, at


def view(flat, name):
    """A parameter of all workers, inside their vectors."""
    at, size, shape = shapes()[0][name]
    part = flat[:, at:at + size]
    return part if len(shape) == 1 else part.unflatten(1, shape)


class Block:
    """The block's layers; gradient() computes one step's gradient into a flat [n, d] array."""

    def __init__(self, seed=0, dtype=torch.float32):
        self.dtype = dtype
        self.drop = layers.Dropout(WORKERS, IMAGES * SIDE * SIDE, CHANNELS, P, seed, SITE, dtype)
        self.norm1 = layers.GroupNorm(WORKERS, IMAGES, CHANNELS, GROUPS, "silu", dtype=dtype)
        self.norm2 = layers.GroupNorm(WORKERS, IMAGES, CHANNELS, GROUPS, "silu", dtype=dtype, dropout=self.drop)

    def conv(self, a, w):
        """3 x 3, channels last, with each worker's own weights."""
        return torch.stack([F.conv2d(a[i].permute(0, 3, 1, 2), w[i].to(self.dtype), padding=1).permute(0, 2, 3, 1) for i in range(WORKERS)])

    def conv_grad(self, a, w, d):
        """Gradients for a and w, the second in 32 bits."""
        da, dw = [], []
        for i in range(WORKERS):
            x, g, k = a[i].permute(0, 3, 1, 2), d[i].permute(0, 3, 1, 2), w[i].to(self.dtype)
            one = torch.ops.aten.convolution_backward(g, x, k, None, [1, 1], [1, 1], [1, 1], False, [0, 0], 1, [True, True, False])
            da.append(one[0].permute(0, 2, 3, 1))
            dw.append(one[1].float())
        return torch.stack(da), torch.stack(dw)

    def gradient(self, flat, x, label, step, grad):
        """Mean loss of each worker; the gradient goes into grad."""
        p = {k: view(flat, k) for k in shapes()[0]}
        g = {k: view(grad, k) for k in shapes()[0]}
        a, stats1 = self.norm1.apply(x, p["weight1"], p["bias1"])
        c = self.conv(a, p["conv1"])
        b, stats2 = self.norm2.apply(c, p["weight2"], p["bias2"], step=step)
        h = x + self.conv(b, p["conv2"])
        pooled = h.float().mean((2, 3))
        logits = pooled @ p["head"].transpose(1, 2)
        loss = F.cross_entropy(logits.transpose(1, 2), label, reduction="none").mean(1)

        dlogits = (logits.softmax(2) - F.one_hot(label, CLASSES)) / IMAGES
        g["head"].copy_(dlogits.transpose(1, 2) @ pooled)
        dh = (dlogits @ p["head"] / SIDE ** 2)[:, :, None, None, :].expand(h.shape).to(self.dtype)
        db, dw = self.conv_grad(b, p["conv2"], dh)
        g["conv2"].copy_(dw)
        dc = self.norm2.grad(c, db, stats2, p["weight2"], p["bias2"], step=step, dweight=g["weight2"], dbias=g["bias2"])[0]
        da, dw = self.conv_grad(a, p["conv1"], dc)
        g["conv1"].copy_(dw)
        self.norm1.grad(x, da, stats1, p["weight1"], p["bias1"], dweight=g["weight1"], dbias=g["bias1"], need_dx=False)
        return loss


def start(gen):
    """A worker's first vector."""
    names, d = shapes()
    x0 = torch.zeros(d, device="cuda")
    for name, (at, size, shape) in names.items():
        if name.startswith("weight"):
            x0[at:at + size] = 1.0
        elif not name.startswith("bias"):
            fan = size // shape[0]
            x0[at:at + size] = torch.randn(size, generator=gen, device="cuda") * (1.0 / fan) ** 0.5
    return x0


def run(steps=30, seed=0, report=None):
    """Mean loss over the workers at each step."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    patterns = torch.randn((CLASSES, SIDE, SIDE, CHANNELS), generator=gen, device="cuda")
    d = shapes()[1]
    opt = binding.CSER(d, WORKERS, 256, R1=4, R2=2, H=4, eta=0.05, beta=0.9, seed=seed)
    opt.set_x0(start(gen))
    block, grad = Block(seed), torch.zeros((WORKERS, d), device="cuda")
    losses = []
    for step in range(steps):
        label = torch.randint(0, CLASSES, (WORKERS, IMAGES), generator=gen, device="cuda")
        x = patterns[label] + torch.randn((WORKERS, IMAGES, SIDE, SIDE, CHANNELS), generator=gen, device="cuda")
        loss = block.gradient(opt.state(binding.STATE_X), x, label, step, grad)
        opt.step(grad)
        losses.append(float(loss.mean()))
        if report:
            report(step, losses[-1])
    opt.close()
    return losses


if __name__ == "__main__":
    n = int(sys.argv[1]) if len(sys.argv) > 1 else 30
    run(n, report=lambda s, v: print(f"step {s:4d}  loss {v:.4f}") if s % 5 == 0 or s + 1 == n else None)
