"""Cases of the operators of a training step around the optimizer (include/cser_train.h), with their plain forms.

Two operators:

* ``orth``: the matrices inside the flat [n, d] gradient of n workers are replaced by their orthogonalised form.
  u = g, or with momentum m <- mu*m + g, u = mu*m + g;  X = u / (|u|_F + 1e-7), taken as its transpose where it is
  tall;  five times  A = X X^T,  X <- a X + (b A + c A A) X;  out = scale * X.
* ``xent``: softmax cross entropy of hidden @ weight^T against one target per token, for n workers with weights of
  their own, and its gradient for the hidden states and the weights.  Tokens whose target is IGNORE have loss 0.

``run`` computes them with elementary torch operations in 32 bits where ``own`` is false, and with the framework's
operators where it is true.
"""
import math

import torch

own = False

IGNORE = -100
ABC = (3.4445, -4.7750, 2.0315)
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
BYTES = {"float32": 4, "bfloat16": 2, "float16": 2}


def _orth(name, n, shapes, grad, out, mu=0.0):
    return {"name": name, "op": "orth", "n": n, "shapes": shapes, "grad": grad, "out": out, "mu": mu}


def _xent(name, n, tokens, vocab, dim, type, grad, ignored=0.0):
    return {"name": name, "op": "xent", "n": n, "tokens": tokens, "vocab": vocab, "dim": dim, "type": type,
            "grad": grad, "ignored": ignored}


def listed():
    return [
        # One small square matrix, as a test or a toy model has it: the call's latency.
        _orth("orth one small", 1, "64x64", "bfloat16", "bfloat16"),
        # Low-rank adapters of two dozen layers, per worker two factors each: many small matrices in one call.
        _orth("orth adapters", 8, ",".join(["16x1024", "1024x16"] * 24), "bfloat16", "bfloat16"),
        # Ragged shapes at unaligned offsets, full-precision gradients in and out, as the optimizer step takes them.
        _orth("orth ragged f32", 3, "100x333,257x129,33x1000,1x77,640x511", "float32", "float32"),
        # One hidden matrix of a mid-sized model with fp32 momentum, fp32 out: the update goes straight into the step.
        _orth("orth hidden f32 momentum", 2, "1024x2048", "float32", "float32", 0.95),
        # The matrices of one BERT-large-sized block for 8 workers, with momentum: the ordinary training step.
        _orth("orth block", 8, "1024x1024,1024x1024,1024x1024,1024x1024,4096x1024,1024x4096", "bfloat16", "bfloat16",
              0.95),
        # One large feed-forward matrix of a single worker.
        _orth("orth large", 1, "4096x16384", "bfloat16", "bfloat16"),
        # Scoring one token against a BERT-sized vocabulary: one read of the weights.
        _xent("xent one token", 1, 1, 30522, 1024, "bfloat16", False),
        # Evaluation of a held-out text: the loss alone, at a length and a vocabulary that no tile divides.
        _xent("xent evaluation", 1, 1999, 50001, 768, "float16", False),
        # Small odd sizes, rows that no 16-byte load can start at.
        _xent("xent ragged", 3, 77, 1003, 201, "float16", True, 0.1),
        # A short sequence for every one of 8 workers: the weights and their gradient are most of the work.
        _xent("xent short", 8, 16, 30522, 1024, "bfloat16", True),
        # Masked-language-model training of the BERT-large-sized model: 8 workers, an eighth of the tokens not counted.
        _xent("xent workers", 8, 512, 30522, 1024, "bfloat16", True, 0.125),
        # A long sequence and a large vocabulary: the largest ordinary training step.
        _xent("xent large", 1, 4096, 131072, 4096, "bfloat16", True),
    ]


def _log_size(rng, low, high):
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    return v if rng.random() < 0.5 else max(low, v // 8 * 8)     # half of them multiples of eight


def draw(rng):
    if rng.random() < 0.5:
        kind = rng.random()
        while True:
            n = rng.choice([1, 2, 3, 4, 8])
            count = _log_size(rng, 1, 12)
            top = 4096 if kind < 0.6 else 256
            shapes = ["%dx%d" % (_log_size(rng, 1, top), _log_size(rng, 1, 4 * top)) for _ in range(count)]
            if rng.random() < 0.5:                               # a stack of equal layers
                shapes = [shapes[0]] * count
            grad = rng.choice(["bfloat16", "float32"])
            case = _orth("", n, ",".join(shapes), grad, grad if rng.random() < 0.7 else "float32",
                         rng.choice([0.0, 0.9, 0.95]))
            w = work(case)
            # The 32-bit results take three products each.
            if w["flops"] * (3 if case["out"] == "float32" else 1) <= 2e12 and w["bytes"] <= 2e9:
                break
    else:
        while True:
            case = _xent("", rng.choice([1, 2, 4, 8]), _log_size(rng, 1, 8192), _log_size(rng, 2, 131072),
                         _log_size(rng, 16, 4096), rng.choice(["bfloat16", "float16"]), rng.random() < 0.7,
                         rng.choice([0.0, 0.1, 0.85]))
            w = work(case)
            if w["flops"] <= 4e12 and w["bytes"] <= 4e9 and case["n"] * case["tokens"] * case["vocab"] <= 2 ** 30:
                break
    del case["name"]
    return case


def _matrices(case):
    """(offset, rows, cols) of each matrix in the flat vector, and the vector's length."""
    at, got = 0, []
    for s in case["shapes"].split(","):
        r, c = (int(v) for v in s.split("x"))
        got.append((at, r, c))
        at += r * c
    return got, at


def _alike(case):
    """The matrices of each shape: {(rows, cols): [offset, ...]}."""
    by = {}
    for at, r, c in _matrices(case)[0]:
        by.setdefault((r, c), []).append(at)
    return by


def _random(seed, *size):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randn(size, generator=gen, device="cuda"), gen


def _orth_inputs(case, seed):
    """Gradients of matrices: a part of low rank that the workers share, and noise of each worker's own."""
    mats, d = _matrices(case)
    n = case["n"]
    noise, gen = _random(seed, n, d)
    grad = noise.mul_(0.3)
    for (r, c), ats in _alike(case).items():
        rank = min(8, r, c)
        u = torch.randn((len(ats), r, rank), generator=gen, device="cuda")
        v = torch.randn((len(ats), rank, c), generator=gen, device="cuda")
        shared = (u @ v).mul_(1 / math.sqrt(rank)).reshape(len(ats), r * c)
        for k, at in enumerate(ats):
            grad[:, at:at + r * c] += shared[k]
    grad = grad.mul_(0.02).to(TYPES[case["grad"]])
    m = None
    if case["mu"]:
        m = torch.randn((n, d), generator=gen, device="cuda").mul_(0.01).add_(grad.float(), alpha=2.0)
    return {"grad": grad, "m": m, "out": torch.zeros((n, d), dtype=TYPES[case["out"]], device="cuda")}


def _xent_inputs(case, seed):
    """Hidden states of unit scale that lean towards their target's row of the weights, as a trained model's do."""
    n, t, v, dim, dt = case["n"], case["tokens"], case["vocab"], case["dim"], TYPES[case["type"]]
    weight = torch.empty((n, v, dim), dtype=dt, device="cuda")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    for i in range(n):
        weight[i] = torch.randn((v, dim), generator=gen, device="cuda").mul_(2.0 / math.sqrt(dim))
    target = (torch.rand((n, t), generator=gen, device="cuda").square_() * v).long().clamp_(max=v - 1)
    hidden = torch.randn((n, t, dim), generator=gen, device="cuda")
    lean = torch.rand((n, t, 1), generator=gen, device="cuda") * 3.0
    hidden += lean * torch.stack([weight[i][target[i]].float() for i in range(n)])
    counted = torch.rand((n, t), generator=gen, device="cuda") >= case["ignored"]
    target = torch.where(counted, target, IGNORE)
    dloss = (1.0 / counted.sum(1, keepdim=True).clamp(min=1)).expand(n, t).contiguous()
    return {"hidden": hidden.to(dt), "weight": weight, "target": target, "dloss": dloss}


def prepare(case, seed):
    state = _orth_inputs(case, seed) if case["op"] == "orth" else _xent_inputs(case, seed)
    state["case"] = case
    if own:
        from paper_2007_13221_b200 import train
        if case["op"] == "orth":
            mats, d = _matrices(case)
            state["plan"] = train.Orthogonalizer(mats, case["n"], d, state["grad"].dtype, state["out"].dtype)
        else:
            state["plan"] = train.LinearCrossEntropy(case["n"], case["tokens"], case["vocab"], case["dim"],
                                                     state["weight"].dtype)
    return state


def run(state):
    if state["case"]["op"] == "orth":
        if own:
            state["plan"].apply(state["grad"], state["out"], momentum=state["m"], mu=state["case"]["mu"])
        else:
            _plain_orth(state)
        return [state["out"]] if state["m"] is None else [state["out"], state["m"]]
    if not own:
        return _plain_xent(state)
    p = state["plan"]
    loss, lse = p.loss(state["hidden"], state["weight"], state["target"], ignore_index=IGNORE)
    if not state["case"]["grad"]:
        return [loss]
    dhidden, dweight = p.grad(state["hidden"], state["weight"], state["target"], lse, state["dloss"],
                              ignore_index=IGNORE)
    return [loss, dhidden, dweight]


def _plain_orth(state):
    case, out = state["case"], state["out"]
    u = state["grad"].float()
    if state["m"] is not None:
        state["m"].mul_(case["mu"]).add_(u)
        u = u + case["mu"] * state["m"]
    a, b, c = ABC
    for (r, cols), ats in _alike(case).items():
        x = torch.stack([u[:, at:at + r * cols] for at in ats]).view(-1, r, cols)
        if r > cols:
            x = x.transpose(1, 2)
        x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + 1e-7)
        for _ in range(5):
            g = x @ x.transpose(1, 2)
            x = a * x + (b * g + c * (g @ g)) @ x
        if r > cols:
            x = x.transpose(1, 2)
        x = x.reshape(len(ats), -1, r * cols).to(out.dtype)
        for k, at in enumerate(ats):
            out[:, at:at + r * cols] = x[k]


def _plain_xent(state):
    h, w, target = state["hidden"].float(), state["weight"].float(), state["target"]
    logits = h @ w.transpose(1, 2)
    top = logits.amax(2, keepdim=True)
    e = logits.sub_(top).exp()
    total = e.sum(2, keepdim=True)
    counted = target != IGNORE
    at = target.clamp(min=0).unsqueeze(2)
    loss = (total.log() - logits.gather(2, at)).squeeze(2) * counted
    if not state["case"]["grad"]:
        return [loss]
    p = e.div_(total)
    p.scatter_add_(2, at, torch.full_like(total, -1.0))
    p.mul_((state["dloss"] * counted).unsqueeze(2))
    dt = state["hidden"].dtype
    return [loss, (p @ w).to(dt), (p.transpose(1, 2) @ h).to(dt)]


def work(case):
    """Each input read and each output written once.  The products of a symmetric result are counted for one half of
    it; the cross entropy's gradient with the logits computed once."""
    n = case["n"]
    if case["op"] == "orth":
        mats, d = _matrices(case)
        flops = 0
        for _, r, c in mats:
            s, l = min(r, c), max(r, c)
            flops += 5 * (s * (s + 1) * l + s * s * (s + 1) + 2 * s * s * l)
        moved = BYTES[case["grad"]] + BYTES[case["out"]] + (8 if case["mu"] else 0)
        return {"bytes": n * d * moved, "flops": n * flops}
    t, v, dim, size = case["tokens"], case["vocab"], case["dim"], BYTES[case["type"]]
    times = 2 if case["grad"] else 1
    moved = times * (t * dim + v * dim) * size + t * (8 + 4 + (4 if case["grad"] else 0))
    return {"bytes": n * moved, "flops": n * t * v * dim * 2 * (3 if case["grad"] else 1)}


def exact(case, seed):
    if case["op"] == "orth":
        return _exact_orth(case, _orth_inputs(case, seed))
    return _exact_xent(case, _xent_inputs(case, seed))


def _exact_orth(case, s):
    """Matrix by matrix, through the polynomial of the singular values' squares: X p(X^T X) with the short side last."""
    n = case["n"]
    g = s["grad"].double()
    out = torch.zeros_like(g)
    if s["m"] is not None:
        new_m = case["mu"] * s["m"].double() + g
        g = g + case["mu"] * new_m
    for at, r, c in _matrices(case)[0]:
        for i in range(n):
            y = g[i, at:at + r * c].view(r, c)
            y = y if r >= c else y.t()
            y = y / (torch.linalg.vector_norm(y) + 1e-7)
            for _ in range(5):
                k = y.t() @ y
                y = y @ (ABC[0] * torch.eye(len(k), dtype=k.dtype, device=k.device) + ABC[1] * k + ABC[2] * (k @ k))
            out[i, at:at + r * c] = (y if r >= c else y.t()).reshape(-1)
    return [out] if s["m"] is None else [out, new_m]


def _exact_xent(case, s):
    n, t, v = case["n"], case["tokens"], case["vocab"]
    if 6.0 * n * t * v * case["dim"] > 3e13:
        return None
    loss = torch.zeros((n, t), dtype=torch.float64, device="cuda")
    dh = torch.zeros(s["hidden"].shape, dtype=torch.float64, device="cuda")
    dw = torch.zeros(s["weight"].shape, dtype=torch.float64, device="cuda") if case["grad"] else None
    for i in range(n):
        w = s["weight"][i].double()
        for k in range(0, t, 1024):
            h, y = s["hidden"][i, k:k + 1024].double(), s["target"][i, k:k + 1024]
            z = h @ w.t()
            lse = torch.logsumexp(z, 1)
            rows = torch.arange(len(y), device="cuda")
            valid = y != IGNORE
            label = torch.where(valid, y, torch.zeros_like(y))
            loss[i, k:k + 1024] = torch.where(valid, lse - z[rows, label], torch.zeros_like(lse))
            if case["grad"]:
                q = torch.exp(z - lse[:, None])
                q[rows, label] -= 1.0
                q *= torch.where(valid, s["dloss"][i, k:k + 1024].double(), torch.zeros_like(lse))[:, None]
                dh[i, k:k + 1024] = q @ w
                dw[i] += q.t() @ h
    return [loss, dh, dw] if case["grad"] else [loss]
