"""Performance cases of the operators around the lmKAN layer: those that train and answer with the dense
matrices that a preconditioned layer ``y = gamma * lmKAN(x) + Linear(ReLU(x))`` and its tables are made of.

  ortho   ``lmkan_orthogonalize``: each matrix of a batch brought near the closest one with orthonormal rows
          (or columns) by steps of X <- a X + (b A + c A^2) X with A = X X^T, from X / (|X| + eps)
  muon    ``lmkan_muon_step``: an optimiser's step with it: momentum, orthogonalised update, weights in place.
          A table in the layout of Alg. 1, [G+1][G+1][pairs][outputs], is a batch of (G+1)^2 matrices of
          pairs x outputs: the layer is one linear map of the pairs' basis functions for each table node
  linear  ``lmkan_linear_i8``: the linear term when it answers: rows scaled to 8 bits one by one, weights
          held in 8 bits with a scale for each output, sums in whole numbers, added to what the layer gave

Sizes are those of ``workloads.py`` and of ``perf/cases.py``, or generic ones between them.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# the usual quintic: singular values from a few thousandths up come near one in five steps
QUINTIC = (3.4445, -4.7750, 2.0315)
STEPS, EPS = 5, 1e-7
LR, MOMENTUM, DECAY = 0.02, 0.95, 0.01


def _ortho(name, batch, rows, cols, dtype="f32"):
    c = {"kind": "ortho", "batch": batch, "rows": rows, "cols": cols, "dtype": dtype}
    return {"name": name, **c} if name else c


def _muon(name, batch, rows, cols, dtype="f32", nesterov=True):
    c = {"kind": "muon", "batch": batch, "rows": rows, "cols": cols, "dtype": dtype, "nesterov": nesterov}
    return {"name": name, **c} if name else c


def _linear(name, batch, n_in, n_out, x="f32", y="f32", relu=True, bias=True, beta=0.0):
    c = {"kind": "linear", "batch": batch, "n_in": n_in, "n_out": n_out, "x": x, "y": y, "relu": relu,
         "bias": bias, "beta": beta}
    return {"name": name, **c} if name else c


def listed():
    return [
        # the table of the smallest layer (16 -> 16, G = 8), node by node: latency
        _ortho("ortho_81x8x16", 81, 8, 16),
        # the linear term of the headline layer
        _ortho("ortho_1024", 1, 1024, 1024),
        # a table nothing of which is a multiple of a tile (500 -> 333, G = 20)
        _ortho("ortho_441x250x333", 441, 250, 333),
        # the linear term of the widest layer, its gradient held in 16 bits
        _ortho("ortho_4096_bf16", 1, 4096, 4096, "bf16"),
        # the table of a convolution stage (3 x 3 windows of 32 channels -> 64, G = 12)
        _muon("muon_169x144x64", 169, 144, 64),
        # the table of a stage on lifted pixels (128 -> 128, G = 12) as one matrix: all basis functions -> outputs
        _muon("muon_flat_10816x128", 1, 10816, 128, nesterov=False),
        # the table of the headline layer (1024 -> 1024, G = 16)
        _muon("muon_289x512x1024", 289, 512, 1024),
        # one request to the widest layer
        _linear("linear_1x4096", 1, 4096, 4096),
        # a few requests in 16 bits
        _linear("linear_48x1024_bf16", 48, 1024, 1024, "bf16", "bf16"),
        # the headline batch, added to the layer's own output
        _linear("linear_8192x1024", 8192, 1024, 1024, beta=0.3),
        # ragged everywhere
        _linear("linear_5000x500x333_f16", 5000, 500, 333, "f16", "f32"),
        # the widest layer
        _linear("linear_4096_bf16", 4096, 4096, 4096, "bf16", "bf16", relu=False, bias=False),
    ]


def _log(rng, low, high):
    """A whole number between low and high, uniform in its logarithm."""
    return min(high, max(low, round(low * (high / low) ** rng.random())))


# the largest listed cases
MOST_ELEMENTS = 289 * 512 * 1024
MOST_PRODUCTS = {"matrices": 289 * 512 * 512 * 1024, "linear": 4096 ** 3}


def draw(rng):
    while True:
        kind = rng.choice(["ortho", "muon", "linear"])
        if kind == "linear":
            c = _linear("", _log(rng, 1, rng.choice([64, 16384, 65536])), _log(rng, 8, 4096), _log(rng, 1, 4096),
                        rng.choice(["f32", "f32", "f16", "bf16"]), rng.choice(["f32", "f32", "f16", "bf16"]),
                        rng.random() < 0.7, rng.random() < 0.5, rng.choice([0.0, 0.3, 1.0]))
            size = max(c["batch"] * c["n_in"], c["batch"] * c["n_out"], c["n_in"] * c["n_out"])
            products = c["batch"] * c["n_in"] * c["n_out"]
            most = MOST_PRODUCTS["linear"]
        else:
            form = rng.choice(["table", "table", "weight", "flat"])
            if form == "table":
                batch, rows, cols = rng.randint(4, 41) ** 2, _log(rng, 2, 1024), _log(rng, 1, 1024)
            elif form == "weight":
                batch, rows, cols = rng.choice([1, 1, 2, 4]), _log(rng, 8, 4096), _log(rng, 8, 4096)
            else:
                batch, rows, cols = 1, _log(rng, 1024, 65536), _log(rng, 1, 512)
            dtype = rng.choice(["f32", "f32", "f16", "bf16"])
            c = (_ortho("", batch, rows, cols, dtype) if kind == "ortho"
                 else _muon("", batch, rows, cols, dtype, rng.random() < 0.7))
            size = batch * rows * cols
            products = size * min(rows, cols)
            most = MOST_PRODUCTS["matrices"]
        if size <= MOST_ELEMENTS and products <= most:
            return c


def _gradients(c, gen):
    """Gradients of a batch of matrices: noise and a few strong directions; the nodes of a table see anything
    from many samples to none, so that whole matrices are zero."""
    batch, rows, cols = c["batch"], c["rows"], c["cols"]
    g = torch.randn((batch, rows, cols), device=DEVICE, generator=gen)
    u = torch.randn((batch, rows, 4), device=DEVICE, generator=gen)
    v = torch.randn((batch, 4, cols), device=DEVICE, generator=gen)
    g += 0.5 * (u @ v)
    if batch > 1:
        seen = torch.rand((batch, 1, 1), device=DEVICE, generator=gen)
        g *= torch.where(seen < 0.05, torch.zeros_like(seen), torch.exp(4.0 * seen - 4.0))
    return (1e-3 * g).to(DTYPE[c["dtype"]])


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    state = {"case": c}
    if c["kind"] == "linear":
        batch, n_in, n_out = c["batch"], c["n_in"], c["n_out"]
        # rows after a normalisation, each with a scale of its own
        x = torch.randn((batch, n_in), device=DEVICE, generator=gen)
        x *= 0.5 + torch.rand((batch, 1), device=DEVICE, generator=gen)
        state["x"] = x.to(DTYPE[c["x"]])
        # the weights as they are kept: whole numbers in [-127, 127] and a scale for each output
        state["w"] = torch.randint(-127, 128, (n_out, n_in), device=DEVICE, generator=gen, dtype=torch.int8)
        state["w_scale"] = (0.5 + torch.rand((n_out,), device=DEVICE, generator=gen)) / (73.0 * math.sqrt(n_in))
        state["bias"] = torch.randn((n_out,), device=DEVICE, generator=gen) if c["bias"] else None
        y = torch.randn((batch, n_out), device=DEVICE, generator=gen).to(DTYPE[c["y"]])
        state["y"] = y if c["beta"] else torch.empty_like(y)
        return state
    state["grad"] = _gradients(c, gen)
    if c["kind"] == "muon":
        shape = state["grad"].shape
        state["momentum"] = 1e-3 * torch.randn(shape, device=DEVICE, generator=gen)
        state["weight"] = torch.randn(shape, device=DEVICE, generator=gen) / math.sqrt(c["rows"])
    return state


def _scale(c):
    """Length of an update's rows: that of the rows of a matrix with orthonormal columns, or one."""
    return math.sqrt(max(1.0, c["rows"] / c["cols"]))


def _orthogonal(x):
    """The plain form, float32: x [batch][rows][cols], the shorter side first."""
    a, b, c = QUINTIC
    wide = x.shape[1] <= x.shape[2]
    x = x if wide else x.mT.contiguous()
    x = x / (x.square().sum(dim=(1, 2), keepdim=True).sqrt() + EPS)
    for _ in range(STEPS):
        gram = x @ x.mT.contiguous()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x if wide else x.mT.contiguous()


def _plain(state):
    c = state["case"]
    if c["kind"] == "ortho":
        return _orthogonal(state["grad"].float()).to(state["grad"].dtype)
    if c["kind"] == "muon":
        m, w, g = state["momentum"], state["weight"], state["grad"].float()
        m.copy_(MOMENTUM * m + (1.0 - MOMENTUM) * g)
        u = MOMENTUM * m + (1.0 - MOMENTUM) * g if c["nesterov"] else m
        w.copy_((1.0 - LR * DECAY) * w - LR * _scale(c) * _orthogonal(u))
        return {"momentum": m, "weight": w}
    x, y = state["x"].float(), state["y"]
    if c["relu"]:
        x = x.clamp(min=0.0)
    most = x.abs().amax(dim=1, keepdim=True)
    full = torch.full_like(most, 127.0)
    steps = torch.where(most > 0, full / most, torch.zeros_like(most))    # one rounding each: the codes are exact
    codes = torch.round(x * steps)
    out = (codes @ state["w"].float().t().contiguous()) * (most / full) * state["w_scale"]
    if state["bias"] is not None:
        out = out + state["bias"]
    if c["beta"]:
        out = c["beta"] * y.float() + out
    y.copy_(out)
    return y


def _kernels(state):
    import paper_2509_07103_amd as pkg
    kinds = {torch.float32: pkg.LMKAN_F32, torch.float16: pkg.LMKAN_F16, torch.bfloat16: pkg.LMKAN_BF16}
    c = state["case"]
    if c["kind"] == "linear":
        desc = pkg.LinearDesc(c["n_in"], c["n_out"], x_dtype=kinds[state["x"].dtype], y_dtype=kinds[state["y"].dtype],
                              relu=c["relu"])
        return pkg.lmkan_linear_i8(desc, state["x"], state["w"], state["w_scale"], bias=state["bias"], beta=c["beta"],
                                   y=state["y"])
    desc = pkg.MatrixDesc(c["batch"], c["rows"], c["cols"], dtype=kinds[state["grad"].dtype], eps=EPS)
    schedule = [QUINTIC] * STEPS
    if c["kind"] == "ortho":
        return pkg.lmkan_orthogonalize(desc, state["grad"], schedule=schedule)
    muon = pkg.MuonParams(lr=LR, momentum=MOMENTUM, nesterov=c["nesterov"], weight_decay=DECAY, scale=_scale(c))
    pkg.lmkan_muon_step(desc, muon, state["grad"], state["momentum"], state["weight"], schedule=schedule)
    return {"momentum": state["momentum"], "weight": state["weight"]}


def run(state):
    return _kernels(state) if own else _plain(state)


def work(case):
    """Each input read once, each output written once.  Products of matrices: a symmetric one counts half; the
    steps either as they are written, or as one polynomial of the Gram matrix that is applied once."""
    c = case
    size = {"f32": 4, "f16": 2, "bf16": 2}
    if c["kind"] == "linear":
        x, w, y = c["batch"] * c["n_in"], c["n_in"] * c["n_out"], c["batch"] * c["n_out"]
        return {"bytes": size[c["x"]] * x + w + 4 * c["n_out"] * (1 + c["bias"]) + size[c["y"]] * y * (1 + bool(c["beta"])),
                "flops": 2 * x * c["n_out"]}
    elements = c["batch"] * c["rows"] * c["cols"]
    m, n = sorted((c["rows"], c["cols"]))
    flops = c["batch"] * min(STEPS * (3 * m * m * n + m ** 3), 3 * m * m * n + (5 + 2 * (STEPS - 1) + STEPS - 1) * m ** 3)
    if c["kind"] == "ortho":
        return {"bytes": 2 * size[c["dtype"]] * elements, "flops": flops}
    return {"bytes": (size[c["dtype"]] + 16) * elements, "flops": flops}


def exact(case, seed):
    """The definitions in float64.  The codes of the rows are whole numbers that the definition fixes in
    float32: the nearest to x times the float32 next to 127 / max |x|."""
    c, s = case, prepare(case, seed)
    if c["kind"] == "linear":
        x = s["x"].double()
        if c["relu"]:
            x = torch.maximum(x, torch.zeros_like(x))
        top = x.abs().max(dim=1, keepdim=True).values
        inverse = torch.where(top > 0, 127.0 / top, torch.zeros_like(top)).float().double()
        product = torch.matmul((x * inverse).float().double().round(), s["w"].double().t().contiguous())
        value = product * (top / 127.0) * s["w_scale"].double()[None, :]
        if s["bias"] is not None:
            value = value + s["bias"].double()[None, :]
        return value + c["beta"] * s["y"].double() if c["beta"] else value
    g = s["grad"].double()
    if c["kind"] == "muon":
        beta = MOMENTUM
        moved = beta * s["momentum"].double() + (1 - beta) * g
        direction = beta * moved + (1 - beta) * g if c["nesterov"] else moved
    else:
        direction = g
    flip = c["rows"] > c["cols"]
    z = direction.transpose(1, 2).contiguous() if flip else direction
    z = z / (torch.linalg.vector_norm(z, dim=(1, 2), keepdim=True) + EPS)
    p, q, r = QUINTIC
    eye = torch.eye(z.shape[1], dtype=z.dtype, device=z.device)
    for _ in range(STEPS):
        s2 = torch.bmm(z, z.transpose(1, 2).contiguous())
        z = torch.bmm(p * eye + q * s2 + r * torch.bmm(s2, s2), z)
    z = z.transpose(1, 2).contiguous() if flip else z
    if c["kind"] == "ortho":
        return z
    return {"momentum": moved, "weight": s["weight"].double() * (1 - LR * DECAY) - LR * _scale(c) * z}
