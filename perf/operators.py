"""Operators around the features and their gradients, measured against their plain form in elementary torch operations.

A case is a dict of plain values.  `kind` names the operator:

  norm       layer norm of every plane of every example's features (rocket_layer_norm)
  norm_grad  its backward pass: gradients of the features, and of weight and bias summed over the examples
             (rocket_layer_norm_backward)
  clip       global norm over many gradient tensors, and the gradients scaled by min(1, max / norm) (rocket_grad_clip)
  step       the same norm, and the parameters moved by -lr times the scaled gradients (rocket_grad_norm,
             rocket_sgd_tensors)

`rows` are examples, `planes` the feature planes of an example, `n` the values of a plane: the layer norm is over n, and
weight and bias are (planes, n).  `tensors` gradient tensors have `elements` values together, split unevenly with odd sizes
(`sizes` names them instead); the `clipped` ones have a norm above the limit.  `dtype` is f32, bf16, f16 or, for clip and
step, `mixed` (f32, bf16 and f16 in turn).  Parameters are f32.
"""
import math
import random

import torch

own = False

EPS = 1e-5
LEARNING_RATE = 1e-2
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}

# values of the largest listed case of each direction: draw() asks for no more
MOST_VALUES = {"norm": 60001 * 3 * 1537, "norm_grad": 65536 * 2048, "clip": 200_000_000, "step": 100_000_000}


def listed():
    return [
        # serving: the max and PPV planes of one reading, 10,000 kernels; launches and latency count
        dict(name="norm-reading", kind="norm", rows=1, planes=2, n=10000, dtype="f32"),
        # the three planes of a univariate archive data set through the standard 10,000 kernels
        dict(name="norm-univariate", kind="norm", rows=256, planes=3, n=10000, dtype="f32"),
        # a large training set's features kept in 16 bits, odd rows that start at any even address
        dict(name="norm-ragged-bf16", kind="norm", rows=60001, planes=3, n=1537, dtype="bf16"),
        # a few examples of a very wide transform: rows longer than one workgroup's registers hold
        dict(name="norm-wide-f16", kind="norm", rows=7, planes=1, n=200001, dtype="f16"),
        # training of a few hundred kernels on a handful of short series: launches count
        dict(name="grad-tiny", kind="norm_grad", rows=16, planes=2, n=500, dtype="f32"),
        # the paper's training set in one batch: 677 examples, 20,000 features
        dict(name="grad-paper", kind="norm_grad", rows=677, planes=2, n=10000, dtype="f32"),
        # many rows of an ordinary width in 16 bits
        dict(name="grad-rows-bf16", kind="norm_grad", rows=65536, planes=1, n=2048, dtype="bf16"),
        # what one training step of 10,000 kernels and a layer norm over two planes has: weights, biases, norm's weight, bias
        dict(name="clip-kernels", kind="clip", tensors=4, sizes="314159,10000,20000,20000", dtype="f32", clipped=True),
        # a network of some hundred tensors of every size, gradients of three types
        dict(name="clip-many", kind="clip", tensors=300, elements=25_000_000, dtype="mixed", clipped=True),
        # a large model's gradients
        dict(name="clip-large", kind="clip", tensors=48, elements=200_000_000, dtype="f32", clipped=True),
        # update of the kernels and the layer norm of one training step, no clipping needed this time
        dict(name="step-kernels", kind="step", tensors=4, sizes="314159,10000,20000,20000", dtype="f32", clipped=False),
        # update of a large model from 16-bit gradients
        dict(name="step-large-bf16", kind="step", tensors=150, elements=100_000_000, dtype="bf16", clipped=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "norm_grad", "clip", "clip", "step"])
    if kind in ("norm", "norm_grad"):
        n = _log_int(rng, 8, 200_000)
        planes = rng.randint(1, 3)
        rows = min(_log_int(rng, 1, 65536), max(1, MOST_VALUES[kind] // (planes * n)))
        return dict(kind=kind, rows=rows, planes=planes, n=n, dtype=rng.choice(["f32", "f32", "bf16", "f16"]))
    elements = _log_int(rng, 2000, MOST_VALUES[kind])
    tensors = min(_log_int(rng, 1, 400), elements // 4)
    return dict(kind=kind, tensors=tensors, elements=elements, dtype=rng.choice(["f32", "bf16", "f16", "mixed"]),
                clipped=rng.random() < 0.6)


# ------------------------------------------------------------------ inputs

def _sizes(case):
    """Sizes of the tensors: a few large ones and many small ones, the same for every seed."""
    if "sizes" in case:
        return [int(v) for v in case["sizes"].split(",")]
    rng = random.Random("%d of %d" % (case["tensors"], case["elements"]))
    share = [math.exp(rng.uniform(0.0, 6.0)) for _ in range(case["tensors"])]
    scale = case["elements"] / sum(share)
    return [max(1, int(v * scale)) for v in share]


def _types(case):
    names = ["f32", "bf16", "f16"] if case["dtype"] == "mixed" else [case["dtype"]]
    return [names[i % len(names)] for i in range(len(_sizes(case)))]


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _features(rows, planes, n, g):
    """Rows as the transform gives them: a plane of maxima around 8, one of shares of positives, one of sigmoid means, each
    example with a level and a spread of its own."""
    x = torch.randn((rows, planes, n), generator=g, device="cuda")
    level = torch.randn((rows, planes, 1), generator=g, device="cuda")
    x = x.mul_(torch.exp(0.3 * level)).add_(level)
    x[:, 0] += 8.0
    if planes > 1:
        x[:, 1:] = torch.sigmoid(0.5 * x[:, 1:])
    return x


def _views(sizes, types, only):
    """One buffer of a type, and the tensors of that type as consecutive pieces of it, which start at any element."""
    total = sum(n for n, t in zip(sizes, types) if t == only)
    flat = torch.empty(total, dtype=TYPES[only], device="cuda")
    return flat, iter(flat.split([n for n, t in zip(sizes, types) if t == only]))


def prepare(case, seed):
    kind, g = case["kind"], _generator(seed)
    s = dict(kind=kind)
    if kind in ("norm", "norm_grad"):
        rows, planes, n, dtype = case["rows"], case["planes"], case["n"], TYPES[case["dtype"]]
        s.update(planes=planes, x=_features(rows, planes, n, g).to(dtype).view(rows, planes * n),
                 weight=1.0 + 0.2 * torch.randn(planes * n, generator=g, device="cuda"),
                 bias=0.1 * torch.randn(planes * n, generator=g, device="cuda"))
        s["y"] = torch.empty_like(s["x"])
        if kind == "norm":
            return s
        s["grad_y"] = torch.randn((rows, planes * n), generator=g, device="cuda").to(dtype)
        s["mean"] = torch.empty((rows, planes), device="cuda")
        s["rstd"] = torch.empty((rows, planes), device="cuda")
        at = max(1, 50_000_000 // (planes * n))
        for i in range(0, rows, at):        # the statistics that the forward pass left
            x = s["x"][i:i + at].double().view(-1, planes, n)
            s["mean"][i:i + at] = x.mean(-1)
            s["rstd"][i:i + at] = torch.rsqrt(x.var(-1, unbiased=False) + EPS)
        s["grad_weight"], s["grad_bias"] = torch.empty_like(s["weight"]), torch.empty_like(s["bias"])
        if own:     # scratch memory that a training program keeps
            from paper_2301_08527_amd import rocket
            s["workspace"] = torch.empty(rocket.rocket_layer_norm_workspace_bytes(rows, planes, n), dtype=torch.uint8,
                                         device="cuda")
        return s
    sizes, types = _sizes(case), _types(case)
    scale = {"f32": 1e-3, "bf16": 1e-3, "f16": 1e-1}      # losses are scaled up where gradients are f16
    # heavy-tailed values: randn * exp(randn) has a mean square of e^2
    s["grads"] = [(torch.randn(n, generator=g, device="cuda") * torch.exp(torch.randn(n, generator=g, device="cuda")) * scale[t])
                  .to(TYPES[t]) for n, t in zip(sizes, types)]
    norm = math.e * math.sqrt(sum(n * scale[t] ** 2 for n, t in zip(sizes, types)))
    s["max_norm"] = (0.25 if case["clipped"] else 8.0) * norm
    if kind == "clip":
        s["flat"] = {}
        pieces = {}
        for t in sorted(set(types)):
            s["flat"][t], pieces[t] = _views(sizes, types, t)
        out = [next(pieces[t]) for t in types]
    else:
        s["params"] = [torch.randn(n, generator=g, device="cuda") for n in sizes]
        flat, pieces = _views(sizes, ["f32"] * len(sizes), "f32")
        s["flat"] = {"f32": flat}
        out = list(pieces)
    s["types"], s["out"] = types, out
    s["norm"] = torch.empty(2, dtype=torch.float64, device="cuda")
    if own:     # the lists of tensors and the scratch memory that a training program keeps
        from paper_2301_08527_amd import rocket
        s["grads"], s["out"] = rocket.rocket_tensors(s["grads"]), rocket.rocket_tensors(s["out"])
        if kind == "step":
            s["params"] = rocket.rocket_tensors(s["params"])
        s["workspace"] = torch.empty(rocket.rocket_grad_workspace_bytes(s["grads"]), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------ the operators' calls

def _run_own(s):
    from paper_2301_08527_amd import rocket
    kind = s["kind"]
    if kind == "norm":
        return rocket.rocket_layer_norm(s["x"], s["weight"], s["bias"], eps=EPS, planes=s["planes"], y=s["y"])
    if kind == "norm_grad":
        return rocket.rocket_layer_norm_backward(s["x"], s["grad_y"], s["mean"], s["rstd"], s["weight"], planes=s["planes"],
                                                 grad_x=s["y"], grad_weight=s["grad_weight"], grad_bias=s["grad_bias"],
                                                 workspace=s["workspace"])
    if kind == "clip":
        rocket.rocket_grad_clip(s["grads"], s["max_norm"], out=s["out"], norm=s["norm"], workspace=s["workspace"])
    else:
        rocket.rocket_grad_norm(s["grads"], s["max_norm"], norm=s["norm"], workspace=s["workspace"])
        rocket.rocket_sgd_tensors(s["params"], s["grads"], LEARNING_RATE, norm=s["norm"], out=s["out"])
    return dict(s["flat"]), s["norm"]


def _plain_norm(x, weight, bias, planes):
    x3 = x.float().view(x.shape[0], planes, -1)
    d = x3 - x3.mean(-1, keepdim=True)
    rstd = torch.rsqrt((d * d).mean(-1, keepdim=True) + EPS)
    y = d * rstd * weight.view(planes, -1) + bias.view(planes, -1)
    return y.to(x.dtype).view(x.shape)


def _plain_norm_grad(x, grad_y, mean, rstd, weight, planes):
    shape = (x.shape[0], planes, -1)
    dy = grad_y.float().view(shape)
    h = (x.float().view(shape) - mean[..., None]) * rstd[..., None]
    g = dy * weight.view(planes, -1)
    dx = (g - g.mean(-1, keepdim=True) - h * (g * h).mean(-1, keepdim=True)) * rstd[..., None]
    return dx.to(x.dtype).view(x.shape), (dy * h).sum(0).view(-1), dy.sum(0).view(-1)


def _plain_coefficient(flats, max_norm):
    """[norm, coefficient], summed in 64 bits: hundreds of millions of squares"""
    squares = [f.double().square().sum() for f in flats]
    norm = torch.sqrt(torch.stack(squares).sum())
    return torch.stack([norm, torch.where(norm <= max_norm, torch.ones_like(norm), max_norm / norm)])


def run(s):
    if own:
        return _run_own(s)
    kind = s["kind"]
    if kind == "norm":
        return _plain_norm(s["x"], s["weight"], s["bias"], s["planes"])
    if kind == "norm_grad":
        return _plain_norm_grad(s["x"], s["grad_y"], s["mean"], s["rstd"], s["weight"], s["planes"])
    if kind == "clip":
        flats = {t: torch.cat([g for g, u in zip(s["grads"], s["types"]) if u == t]) for t in s["flat"]}
        norm = _plain_coefficient(flats.values(), s["max_norm"])
        c = norm[1].float()
        return {t: (f.float() * c).to(f.dtype) for t, f in flats.items()}, norm
    flat = torch.cat([g.float() for g in s["grads"]])
    norm = _plain_coefficient([flat], s["max_norm"])
    return {"f32": torch.cat(s["params"]) - flat * (LEARNING_RATE * norm[1]).float()}, norm


# ------------------------------------------------------------------ work and exact values

def work(case):
    if case["kind"] in ("norm", "norm_grad"):
        rows, planes, n, size = case["rows"], case["planes"], case["n"], BYTES[case["dtype"]]
        values, wide = rows * planes * n, planes * n
        if case["kind"] == "norm":
            return {"bytes": 2.0 * values * size + 8.0 * wide, "flops": 8.0 * values}
        return {"bytes": 3.0 * values * size + 12.0 * wide + 8.0 * rows * planes, "flops": 14.0 * values}
    sizes, types = _sizes(case), _types(case)
    grads = float(sum(n * BYTES[t] for n, t in zip(sizes, types)))
    values = float(sum(sizes))
    if case["kind"] == "clip":
        return {"bytes": 2.0 * grads, "flops": 3.0 * values}
    return {"bytes": grads + 8.0 * values, "flops": 4.0 * values}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("norm", "norm_grad"):
        rows, planes, n = case["rows"], case["planes"], case["n"]
        w, b = s["weight"].to(torch.float64).reshape(planes, n), s["bias"].to(torch.float64).reshape(planes, n)
        whole = torch.empty((rows, planes, n), dtype=torch.float64, device="cuda")
        dw, db = torch.zeros_like(w), torch.zeros_like(w)
        at = max(1, 50_000_000 // (planes * n))
        for i in range(0, rows, at):
            x = s["x"][i:i + at].to(torch.float64).reshape(-1, planes, n)
            x = x - x.sum(2, keepdim=True) / n
            sd = torch.sqrt(x.pow(2).sum(2, keepdim=True) / n + EPS)
            if kind == "norm":
                whole[i:i + at] = x / sd * w + b
                continue
            dy = s["grad_y"][i:i + at].to(torch.float64).reshape(-1, planes, n)
            # the Jacobian of (x - m) / sd, applied to dy * w
            v = dy * w
            whole[i:i + at] = (v - v.sum(2, keepdim=True) / n) / sd - x * ((v * x).sum(2, keepdim=True) / (n * sd.pow(3)))
            dw += (dy * (x / sd)).sum(0)
            db += dy.sum(0)
        whole = whole.reshape(rows, planes * n)
        return whole if kind == "norm" else (whole, dw.reshape(-1), db.reshape(-1))
    grads = s["grads"].tensors if own else s["grads"]
    norm = math.sqrt(math.fsum(float(g.to(torch.float64).pow(2).sum()) for g in grads))
    c = 1.0 if norm <= s["max_norm"] else s["max_norm"] / norm
    told = torch.tensor([norm, c], dtype=torch.float64)
    if kind == "clip":
        return {t: torch.cat([g.to(torch.float64) * c for g, u in zip(grads, s["types"]) if u == t]) for t in s["flat"]}, told
    params = s["params"].tensors if own else s["params"]
    return {"f32": torch.cat([p.to(torch.float64) - LEARNING_RATE * c * g.to(torch.float64) for p, g in zip(params, grads)])}, told
