"""Cases of the layers between the products of the workers' models (include/cser_layers.h), with their plain forms.

Two operators, each for n workers with parameters and random draws of their own:

* ``drop``: dropout whose mask comes from a counter-based generator and is never stored.  Element e of worker i's
  array is dropped where word e & 3 of Philox4x32-10, with the seed as its key and the counter
  (e >> 2, step's low half, step's high half, 4096 * site + i), is below p * 2^32; others are divided by 1 - p.
  y = residual + dropout(x + bias), with both, one or neither; its gradient: dx = dropout(dy), dbias = dx summed over rows.
* ``norm``: group norm with an activation, channels last.  Mean and variance over the pixels and channels of a group of
  one sample; y = act((x - mean) / sqrt(var + eps) * weight + bias).  Where p > 0 it reads dropout(x) in the place of x.
  Its gradient: dx, and for each worker dweight and dbias.

``run`` computes them with elementary torch operations in 32 bits where ``own`` is false, and with the framework's
operators where it is true.
"""
import math

import torch

own = False

EPS = 1e-5
SITE = 5
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
BYTES = {"float32": 4, "bfloat16": 2, "float16": 2}
LOW = 0xFFFFFFFF


def _drop(name, n, rows, cols, type, p, bias, residual, grad):
    return {"name": name, "op": "drop", "n": n, "rows": rows, "cols": cols, "type": type, "p": p, "bias": bias,
            "residual": residual, "grad": grad}


def _norm(name, n, samples, high, wide, channels, groups, type, act, grad, p=0.0):
    return {"name": name, "op": "norm", "n": n, "samples": samples, "high": high, "wide": wide, "channels": channels,
            "groups": groups, "type": type, "act": act, "grad": grad, "p": p}


def listed():
    return [
        # One token's row at the end of a sublayer: the call's latency.
        _drop("drop one row", 1, 1, 1024, "bfloat16", 0.1, True, True, False),
        # Odd sizes: workers' arrays that begin anywhere, rows that no vector divides, both directions.
        _drop("drop ragged", 3, 77, 201, "float16", 0.1, True, True, True),
        # Embeddings of a word-level model in full precision, an odd number of columns.
        _drop("drop f32 odd", 2, 9999, 1111, "float32", 0.5, False, False, True),
        # A sublayer's end in training: 8 workers of 8 sequences of 512 tokens of the BERT-large-sized model.
        _drop("drop sublayer", 8, 4096, 1024, "bfloat16", 0.1, True, True, True),
        # The hidden layer of a feed-forward block for many tokens: the largest array.
        _drop("drop feed-forward", 8, 8192, 4096, "bfloat16", 0.1, False, False, False),
        # One small image at the end of a net: the call's latency.
        _norm("norm one image", 1, 1, 8, 8, 64, 32, "bfloat16", "silu", False),
        # Odd images and channels, no power of two anywhere, full precision, both directions.
        _norm("norm ragged f32", 3, 5, 13, 9, 60, 12, "float32", "silu", True),
        # First stage of a wide residual net of width 8: 8 workers of 16 images each, training.
        _norm("norm wide stage", 8, 16, 32, 32, 128, 32, "bfloat16", "silu", True),
        # Its second stage's second norm, which stands behind a dropout.
        _norm("norm wide dropout", 8, 16, 16, 16, 256, 32, "bfloat16", "silu", True, 0.3),
        # Evaluation of a stem's output: large images, few channels, two to a group.
        _norm("norm stem", 2, 16, 112, 112, 64, 32, "float16", "relu", False),
        # First stage of a 50-layer residual net, 8 workers of 16 images: the largest training step.
        _norm("norm residual stage", 8, 16, 56, 56, 256, 32, "bfloat16", "silu", True),
        # One large image of one worker: few samples, each of them many pixels.
        _norm("norm large image", 1, 1, 512, 512, 128, 32, "bfloat16", "silu", True),
    ]


def _log_size(rng, low, high):
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    return v if rng.random() < 0.5 else max(low, v // 8 * 8)     # half of them multiples of eight


def draw(rng):
    type = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
    if rng.random() < 0.5:
        while True:
            case = _drop("", rng.choice([1, 2, 3, 4, 8]), _log_size(rng, 1, 65536), _log_size(rng, 1, 16384), type,
                         rng.choice([0.1, 0.25, 0.3, 0.5]), rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.7)
            if case["n"] * case["rows"] * case["cols"] <= 2 ** 26:
                break
    else:
        while True:
            groups = rng.choice([1, 4, 8, 16, 32])
            high = _log_size(rng, 1, 224)
            # ReLU's gradient jumps where a value is next to 0, whatever the arithmetic: it is drawn for the forward pass.
            grad = rng.random() < 0.7
            case = _norm("", rng.choice([1, 2, 3, 4, 8]), _log_size(rng, 1, 64), high,
                         high if rng.random() < 0.5 else _log_size(rng, 1, 224), groups * _log_size(rng, 1, 64), groups,
                         type, rng.choice(["none", "silu"] if grad else ["none", "relu", "silu"]), grad,
                         rng.choice([0.0, 0.0, 0.0, 0.3]))
            elements = case["n"] * case["samples"] * high * case["wide"] * case["channels"]
            if elements <= 2 ** 26 and high * case["wide"] * case["channels"] >= 32 * groups:
                break
    del case["name"]
    return case


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*size):
        return torch.randn(size, generator=gen, device="cuda")

    dt, n = TYPES[case["type"]], case["n"]
    s = {"seed": seed * 0x9E3779B97F4A7C15 % 2 ** 64, "step": 2 ** 32 + 1000 + seed % 1000}
    if case["op"] == "drop":
        shape = (n, case["rows"], case["cols"])
        s["x"] = normal(*shape).to(dt)
        s["bias"] = normal(n, case["cols"]).mul_(0.1) if case["bias"] else None
        s["residual"] = normal(*shape).to(dt) if case["residual"] else None
        s["dy"] = normal(*shape).mul_(0.1).to(dt) if case["grad"] else None
        return s
    # A convolution's outputs: each channel has a mean and a scale of its own.
    c = case["channels"]
    shape = (n, case["samples"], case["high"], case["wide"], c)
    scale, mean = torch.rand((n, 1, 1, 1, c), generator=gen, device="cuda").add_(0.5), normal(n, 1, 1, 1, c)
    s["x"] = normal(*shape).mul_(scale).add_(mean).to(dt)
    s["weight"] = normal(n, c).mul_(0.2).add_(1.0)
    s["bias"] = normal(n, c).mul_(0.2)
    s["dy"] = normal(*shape).mul_(0.1).to(dt) if case["grad"] else None
    return s


def prepare(case, seed):
    state = _inputs(case, seed)
    state["case"] = case
    if own:
        from paper_2007_13221_b200 import layers
        n = case["n"]
        if case["op"] == "drop":
            state["plan"] = layers.Dropout(n, case["rows"], case["cols"], case["p"], state["seed"], SITE, TYPES[case["type"]])
        else:
            pixels = case["samples"] * case["high"] * case["wide"]
            drop = layers.Dropout(n, pixels, case["channels"], case["p"], state["seed"], SITE,
                                  TYPES[case["type"]]) if case["p"] else None
            state["plan"] = layers.GroupNorm(n, case["samples"], case["channels"], case["groups"], case["act"], EPS,
                                             TYPES[case["type"]], dropout=drop)
    return state


def run(state):
    case = state["case"]
    if not own:
        return _plain_drop(state) if case["op"] == "drop" else _plain_norm(state)
    plan, x, step = state["plan"], state["x"], state["step"]
    if case["op"] == "drop":
        y = plan.apply(x, step, bias=state["bias"], residual=state["residual"])
        if not case["grad"]:
            return [y]
        dx, dbias = plan.grad(state["dy"], step, need_dbias=case["bias"])
        return [y, dx, dbias] if case["bias"] else [y, dx]
    y, stats = plan.apply(x, state["weight"], state["bias"], step=step)
    if not case["grad"]:
        return [y]
    return [y, *plan.grad(x, state["dy"], stats, state["weight"], state["bias"], step=step)]


def _keep(case, seed, step, n, count):
    """[n, count] truth values: what dropout keeps."""
    c0 = torch.arange((count + 3) // 4, device="cuda").expand(n, -1)
    c1 = torch.full_like(c0, step & LOW)
    c2 = torch.full_like(c0, step >> 32)
    c3 = (4096 * SITE + torch.arange(n, device="cuda")).unsqueeze(1).expand_as(c0)
    k0, k1 = seed & LOW, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57                   # modulo 2^64
        c0, c1, c2, c3 = (b >> 32 & LOW) ^ c1 ^ k0, b & LOW, (a >> 32 & LOW) ^ c3 ^ k1, a & LOW
        k0, k1 = k0 + 0x9E3779B9 & LOW, k1 + 0xBB67AE85 & LOW
    return torch.stack([c0, c1, c2, c3], 2).view(n, -1)[:, :count] >= math.floor(case["p"] * 2 ** 32)


def _plain_drop(state):
    case, x = state["case"], state["x"]
    keep = _keep(case, state["seed"], state["step"], case["n"], case["rows"] * case["cols"]).view(x.shape)
    factor = 1.0 / (1.0 - case["p"])
    y = x.float()
    if case["bias"]:
        y = y + state["bias"].unsqueeze(1)
    y = torch.where(keep, y * factor, 0.0)
    if case["residual"]:
        y = y + state["residual"].float()
    if not case["grad"]:
        return [y.to(x.dtype)]
    dx = torch.where(keep, state["dy"].float() * factor, 0.0)
    out = [y.to(x.dtype), dx.to(x.dtype)]
    return out + [dx.sum(1)] if case["bias"] else out


def _plain_norm(state):
    case, dt = state["case"], state["x"].dtype
    n, b, c, g = case["n"], case["samples"], case["channels"], case["groups"]
    size = (n, b, -1, g, c // g)
    x = state["x"].float().view(size)
    if case["p"]:
        keep = _keep(case, state["seed"], state["step"], n, x[0].numel()).view(x.shape)
        factor = 1.0 / (1.0 - case["p"])
        x = torch.where(keep, x * factor, 0.0)
    mean = x.mean((2, 4), keepdim=True)
    x = x - mean
    rstd = (x.square().mean((2, 4), keepdim=True) + EPS).rsqrt()
    x = x * rstd
    weight, bias = state["weight"].view(n, 1, 1, g, -1), state["bias"].view(n, 1, 1, g, -1)
    z = x * weight + bias
    gate = None
    if case["act"] == "relu":
        y = z.clamp(min=0.0)
    elif case["act"] == "silu":
        gate = 1.0 / (1.0 + (-z).exp())
        y = z * gate
    else:
        y = z
    y = y.to(dt).view(state["x"].shape)
    if not case["grad"]:
        return [y]
    dz = state["dy"].float().view(x.shape)
    if gate is not None:
        dz = dz * (gate * (1.0 + z * (1.0 - gate)))
    dbias, dweight = dz.sum((1, 2)).view(n, c), (dz * x).sum((1, 2)).view(n, c)
    dz = dz * weight
    dx = rstd * (dz - dz.mean((2, 4), keepdim=True) - x * (dz * x).mean((2, 4), keepdim=True))
    if case["p"]:
        dx = torch.where(keep, dx * factor, 0.0)
    return [y, dx.to(dt).view(state["x"].shape), dweight, dbias]


def work(case):
    """Each input read and each output written once, for each of the two directions."""
    n, size = case["n"], BYTES[case["type"]]
    if case["op"] == "drop":
        e, small = n * case["rows"] * case["cols"], 4 * n * case["cols"] * case["bias"]
        moved = e * size * (2 + case["residual"]) + small
        if case["grad"]:
            moved += e * size * 2 + small
        return {"bytes": moved, "flops": e * (1 + case["bias"] + case["residual"] + case["grad"] * (1 + case["bias"]))}
    e = n * case["samples"] * case["high"] * case["wide"] * case["channels"]
    moved = e * size * (5 if case["grad"] else 2) + 8 * n * case["channels"] * (3 if case["grad"] else 1)
    per = 6 + (5 if case["act"] == "silu" else 0)                 # forward: mean, variance, normalised, weight, bias, activation
    if case["grad"]:
        per += 5 + (10 if case["act"] == "silu" else 0) + 9       # value again, activation's slope, sums, result
    return {"bytes": moved, "flops": e * per}


def exact(case, seed):
    s = _inputs(case, seed)
    return _exact_drop(case, s) if case["op"] == "drop" else _exact_norm(case, s)


def _times(a, b):
    """High and low 32 bits of the product of 32-bit numbers, from 16-bit halves."""
    a1, a0, b1, b0 = a >> 16, a & 0xFFFF, b >> 16, b & 0xFFFF
    low = a0 * b0
    mid = a1 * b0 + (low >> 16)
    cross = a0 * b1 + (mid & 0xFFFF)
    return a1 * b1 + (mid >> 16) + (cross >> 16), (cross & 0xFFFF) << 16 | low & 0xFFFF


def _kept(p, seed, step, worker, count):
    """Truth values for one worker's `count` elements."""
    ctr = [torch.arange(-(-count // 4), device="cuda"), step % 2 ** 32, step // 2 ** 32, 4096 * SITE + worker]
    key = [seed % 2 ** 32, seed // 2 ** 32]
    for r in range(10):
        h0, l0 = _times(ctr[0], 0xD2511F53)
        h1, l1 = _times(ctr[2], 0xCD9E8D57)
        ctr = [h1 ^ ctr[1] ^ (key[0] + r * 0x9E3779B9) % 2 ** 32, l1, h0 ^ ctr[3] ^ (key[1] + r * 0xBB67AE85) % 2 ** 32, l0]
    words = torch.empty((len(ctr[0]), 4), dtype=torch.int64, device="cuda")
    for j in range(4):
        words[:, j] = ctr[j]
    return words.reshape(-1)[:count].double() / 2 ** 32 >= math.floor(p * 2 ** 32) / 2 ** 32


def _exact_drop(case, s):
    n, p = case["n"], case["p"]
    y = torch.empty(s["x"].shape, dtype=torch.float64, device="cuda")
    dx = torch.empty_like(y) if case["grad"] else None
    for i in range(n):
        mask = _kept(p, s["seed"], s["step"], i, y[i].numel()).view(y[i].shape).double() / (1.0 - p)
        v = s["x"][i].double()
        if case["bias"]:
            v += s["bias"][i].double()
        y[i] = v * mask
        if case["residual"]:
            y[i] += s["residual"][i].double()
        if case["grad"]:
            dx[i] = s["dy"][i].double() * mask
    if not case["grad"]:
        return [y]
    return [y, dx, dx.sum(1)] if case["bias"] else [y, dx]


def _exact_norm(case, s):
    """Sample by sample; the gradient as the derivative of the normalised values, projected off their mean and themselves."""
    n, c, g = case["n"], case["channels"], case["groups"]
    y = torch.empty(s["x"].shape, dtype=torch.float64, device="cuda")
    dx = torch.empty_like(y) if case["grad"] else None
    dw = torch.zeros((n, c), dtype=torch.float64, device="cuda")
    db = torch.zeros_like(dw)
    for i in range(n):
        mask = None
        if case["p"]:
            mask = _kept(case["p"], s["seed"], s["step"], i, y[i].numel()).view(y[i].shape).double() / (1.0 - case["p"])
        w, b = s["weight"][i].double(), s["bias"][i].double()
        for k in range(case["samples"]):
            v = s["x"][i, k].double()
            if mask is not None:
                v = v * mask[k]
            # one row per group: [groups, pixels * channels of a group]
            rows = v.view(-1, g, c // g).transpose(0, 1).reshape(g, -1)
            var, mu = torch.var_mean(rows, 1, correction=0, keepdim=True)
            std = (var + EPS).sqrt()
            hat = (rows - mu) / std
            xhat = hat.view(g, -1, c // g).transpose(0, 1).reshape(-1, c)
            z = xhat * w + b
            gate = torch.sigmoid(z)
            y[i, k] = {"none": z, "relu": torch.relu(z), "silu": z * gate}[case["act"]].view(v.shape)
            if not case["grad"]:
                continue
            dz = s["dy"][i, k].double().view(-1, c)
            if case["act"] == "silu":
                dz = dz * (gate + z * gate * (1.0 - gate))
            dw[i] += (dz * xhat).sum(0)
            db[i] += dz.sum(0)
            u = (dz * w).view(-1, g, c // g).transpose(0, 1).reshape(g, -1)
            u = u - u.mean(1, keepdim=True)
            u = (u - hat * (u * hat).mean(1, keepdim=True)) / std
            d = u.view(g, -1, c // g).transpose(0, 1).reshape(v.shape)
            dx[i, k] = d if mask is None else d * mask[k]
    return [y, dx, dw, db] if case["grad"] else [y]
