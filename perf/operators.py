"""What the operators that learn a normalised layer are timed on: layer normalisation over the channels of every pixel and
its gradient, the orthogonalised update of filters by Newton-Schulz products, and the descent step built on it.

Formulas (per pixel of a feature map, sums over its c channels):

* norm: y = gamma (x - mean) rstd + beta, mean = sum x / c, rstd = 1 / sqrt(sum (x - mean)^2 / c + eps); then max(y, 0) where
  the case says relu.  "stats": mean and rstd are outputs too, for the gradient.
* norm_grad: with g = dy gamma and z = (x - mean) rstd: dx = rstd (g - sum g / c - z sum (g z) / c), dgamma = sum over pixels of
  dy z, dbeta = sum over pixels of dy.
* orth: X = G / (|G|_F + eps); five times A = X X^T, X = a X + (b A + c A A) X; on the transpose where G has more rows than columns.
* muon: for every layer's filters as a matrix of k rows: m = mu m + g, u = g + mu m,
  w = (1 - lr decay) w - lr sqrt(max(1, rows / columns)) orth(u).

Plain forms are computed in 32 bits with elementary torch operations and rounded once at the end.
"""
from __future__ import annotations

import math
import struct

import torch

own = False

EPS = 1e-5                                       # of a norm
ORTH_EPS = 1e-7
STEPS = 5
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
LR, MOMENTUM, DECAY = 0.02, 0.95, 0.01

# GoogLeNet's inception modules: channels in, 1x1, 3x3 reduce, 3x3, 5x5 reduce, 5x5, pool projection
MODULES = {
    "3a": (192, 64, 96, 128, 16, 32, 32), "3b": (256, 128, 128, 192, 32, 96, 64), "4a": (480, 192, 96, 208, 16, 48, 64),
    "4b": (512, 160, 112, 224, 24, 64, 64), "4c": (512, 128, 128, 256, 24, 64, 64), "4d": (512, 112, 144, 288, 32, 64, 64),
    "4e": (528, 256, 160, 320, 32, 128, 128), "5a": (832, 256, 160, 320, 32, 128, 128), "5b": (832, 384, 192, 384, 48, 128, 128),
}


def listed():
    return [
        # the classifier's feature vector of a single image: one pixel of 1024 channels
        dict(name="norm_one_vector_bf16", op="norm", dtype="bf16", order="nhwc", n=1, c=1024, h=1, w=1, relu=False, stats=False),
        # training forward of a layer in front of a module, channel planes as the fp32 convolutions leave them
        dict(name="norm_map_f32_planes_b32", op="norm", dtype="f32", order="nchw", n=32, c=192, h=28, w=28, relu=True, stats=True),
        # an odd batch, a ragged map and a channel count that nothing divides
        dict(name="norm_ragged_bf16", op="norm", dtype="bf16", order="nhwc", n=37, c=509, h=15, w=13, relu=True, stats=False),
        # inference on the second convolution's map of a full batch
        dict(name="norm_map_bf16_b128", op="norm", dtype="bf16", order="nhwc", n=128, c=192, h=56, w=56, relu=True, stats=False),
        # the gradient that learns the layer of norm_map_f32_planes_b32
        dict(name="norm_grad_f32_planes_b32", op="norm_grad", dtype="f32", order="nchw", n=32, c=192, h=28, w=28),
        # ... of a ragged channels-last map
        dict(name="norm_grad_ragged_f32", op="norm_grad", dtype="f32", order="nhwc", n=19, c=333, h=14, w=14),
        # ... of wide rows, a batch of 8192 feature vectors
        dict(name="norm_grad_rows_bf16", op="norm_grad", dtype="bf16", order="nhwc", n=8192, c=4096, h=1, w=1),
        # filters of the first layer, 64 of 3 x 7 x 7
        dict(name="orth_first_layer_f32", op="orth", dtype="f32", rows=64, cols=147),
        # more rows than columns, neither a multiple of anything, in bf16
        dict(name="orth_tall_bf16", op="orth", dtype="bf16", rows=1201, cols=500),
        # a large square matrix
        dict(name="orth_square_f32", op="orth", dtype="f32", rows=4096, cols=4096),
        # the descent step of one slim layer, 192 filters of 64 x 3 x 3
        dict(name="muon_slim_layer", op="muon", layers="192x64x3"),
        # ... of all filters of GoogLeNet and its classifier
        dict(name="muon_googlenet", op="muon", layers="googlenet"),
    ]


def _log(rng, lo, hi):
    """A whole number whose logarithm is spread evenly over [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("norm", "norm", "norm_grad", "norm_grad", "orth", "orth", "muon"))
    if op == "orth":
        return dict(op=op, dtype=rng.choice(("f32", "bf16")), rows=_log(rng, 16, 4096), cols=_log(rng, 16, 4096))
    if op == "muon":
        if rng.random() < 0.5:
            return dict(op=op, layers="%dx%dx%d" % (_log(rng, 8, 512), _log(rng, 3, 512), rng.choice((1, 3, 5, 7))))
        return dict(op=op, layers=",".join(sorted(rng.sample(sorted(MODULES), rng.randint(1, 8)))))
    case = dict(op=op, dtype=rng.choice(("f32", "bf16")), order=rng.choice(("nchw", "nhwc", "nhwc")), n=_log(rng, 1, 256), c=_log(rng, 3, 4096), h=_log(rng, 1, 64), w=_log(rng, 1, 64))
    while case["n"] * case["c"] * case["h"] * case["w"] > (1 << 25):
        big = max(("n", "h", "w"), key=lambda k: case[k])
        case[big] = max(1, case[big] // 2)
    return dict(case, relu=rng.random() < 0.5, stats=rng.random() < 0.5) if op == "norm" else case


# ---- inputs ------------------------------------------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _layers(case):
    """(k, c, r) of every layer of a muon case."""
    if "x" in case["layers"]:
        return [tuple(int(v) for v in case["layers"].split("x"))]
    whole = case["layers"] == "googlenet"
    out = [(64, 3, 7), (64, 64, 1), (192, 64, 3)] if whole else []
    for m in sorted(MODULES) if whole else case["layers"].split(","):
        ci, c1, c3r, c3, c5r, c5, cp = MODULES[m]
        out += [(c1, ci, 1), (c3r, ci, 1), (c3, c3r, 3), (c5r, ci, 1), (c5, c5r, 5), (cp, ci, 1)]
    return out + ([(1000, 1024, 1)] if whole else [])


def _gradient(gen, rows, cols):
    """A parameter gradient: sum over pixels of (gradient of an output behind a ReLU) x (features behind a ReLU)."""
    pixels = 2 * min(rows, cols) + 64
    dz = torch.randn((rows, pixels), device="cuda", generator=gen) * (torch.rand((rows, pixels), device="cuda", generator=gen) < 0.6)
    x = torch.randn((pixels, cols), device="cuda", generator=gen).abs()
    return dz @ x


def _shape(case):
    n, c, h, w = (case[d] for d in ("n", "c", "h", "w"))
    return (n, c, h, w) if case["order"] == "nchw" else (n, h, w, c)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case=case)
    if case["op"] == "orth":
        s["g"] = _gradient(gen, case["rows"], case["cols"]).to(_dtype(case))
    elif case["op"] == "muon":
        s["shapes"] = _layers(case)
        sizes = [k * c * r * r for k, c, r in s["shapes"]]
        for name in ("w", "g", "m"):                  # every layer's piece of one buffer each
            s[name] = torch.empty(sum(sizes), device="cuda")
            s[name + "s"] = [t.view(k, c, r, r) for t, (k, c, r) in zip(s[name].split(sizes), s["shapes"])]
        for (k, c, r), w, g, m in zip(s["shapes"], s["ws"], s["gs"], s["ms"]):
            w.copy_(torch.randn(w.shape, device="cuda", generator=gen) * math.sqrt(2.0 / (c * r * r)))
            g.copy_(_gradient(gen, k, c * r * r).view(g.shape))
            m.copy_(_gradient(gen, k, c * r * r).view(m.shape) * 4)
    else:
        channel = 1 if case["order"] == "nchw" else 3
        dims = [1] * 4
        dims[channel] = case["c"]
        # a convolution's outputs: every channel with a spread and an offset of its own
        s["x"] = (torch.randn(_shape(case), device="cuda", generator=gen) * (0.5 + torch.rand(dims, device="cuda", generator=gen))
                  + 0.5 * torch.randn(dims, device="cuda", generator=gen)).to(_dtype(case))
        s["gamma"] = 1 + 0.2 * torch.randn(case["c"], device="cuda", generator=gen)
        s["beta"] = 0.2 * torch.randn(case["c"], device="cuda", generator=gen)
        if case["op"] == "norm_grad":
            s["dy"] = (torch.randn(_shape(case), device="cuda", generator=gen) * (torch.rand(_shape(case), device="cuda", generator=gen) < 0.6)).to(_dtype(case))
            x = s["x"].float()
            s["mean"] = x.mean(channel)
            s["rstd"] = 1 / ((x - s["mean"].unsqueeze(channel)).square().mean(channel) + EPS).sqrt()
    if own:
        _buffers(s)
    return s


def _buffers(s):
    """The outputs, the scratch memory and the list of layers that a program keeps from call to call."""
    from paper_1708_04728_amd import binding as B
    case = s["case"]
    scratch = lambda n: torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
    if case["op"] == "orth":
        s["out"] = torch.empty_like(s["g"])
        s["scratch"] = scratch(B.orthogonalise_workspace_bytes([s["g"]]))
    elif case["op"] == "muon":
        s["params"] = B.muon_params(list(zip(s["ws"], s["gs"], s["ms"])))
        s["scratch"] = scratch(B.muon_step_workspace_bytes(s["params"]))
    else:
        tensor = B.NHWC if case["order"] == "nhwc" else lambda t: t
        s["out"] = torch.empty_like(s["x"])
        s["tx"], s["ty"] = tensor(s["x"]), tensor(s["out"])
        if case["op"] == "norm":
            pixels = (case["n"], case["h"], case["w"])
            s["mean"], s["rstd"] = (torch.empty(pixels, device="cuda") if case["stats"] else None for _ in range(2))
        else:
            s["tdy"], s["dgamma"], s["dbeta"] = tensor(s["dy"]), torch.empty_like(s["gamma"]), torch.empty_like(s["beta"])
            s["scratch"] = scratch(B.layernorm_bwd_workspace_bytes(s["tx"]))


# ---- one pass ------------------------------------------------------------------------------------------------------------
def run(s):
    return (_run_own if own else {"norm": _norm, "norm_grad": _norm_grad, "orth": _orth, "muon": _muon}[s["case"]["op"]])(s)


def _run_own(s):
    from paper_1708_04728_amd import binding as B
    case = s["case"]
    if case["op"] == "orth":
        B.orthogonalise([s["g"]], [s["out"]], s["scratch"], steps=STEPS, coefficients=COEFFICIENTS, eps=ORTH_EPS)
        return s["out"]
    if case["op"] == "muon":
        B.muon_step(s["params"], s["scratch"], LR, momentum=MOMENTUM, weight_decay=DECAY, steps=STEPS, coefficients=COEFFICIENTS, eps=ORTH_EPS)
        return {"w": s["w"], "m": s["m"]}
    if case["op"] == "norm":
        B.layernorm_fwd(s["tx"], s["gamma"], s["beta"], EPS, case["relu"], s["ty"], s["mean"], s["rstd"])
        return {"y": s["out"], "mean": s["mean"], "rstd": s["rstd"]} if case["stats"] else s["out"]
    B.layernorm_bwd(s["tdy"], s["tx"], s["gamma"], s["mean"], s["rstd"], s["ty"], s["dgamma"], s["dbeta"], s["scratch"])
    return {"dx": s["out"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}


def _over(case, v):
    """A vector over the channels, along the channel axis."""
    return v.view(1, -1, 1, 1) if case["order"] == "nchw" else v


def _norm(s):
    case = s["case"]
    axis = 1 if case["order"] == "nchw" else 3
    x = s["x"].float()
    mean = x.mean(axis, keepdim=True)
    d = x - mean
    rstd = 1 / ((d * d).mean(axis, keepdim=True) + EPS).sqrt()
    y = d * rstd * _over(case, s["gamma"]) + _over(case, s["beta"])
    if case["relu"]:
        y = y.clamp(min=0)
    y = y.to(s["x"].dtype)
    return {"y": y, "mean": mean.squeeze(axis), "rstd": rstd.squeeze(axis)} if case["stats"] else y


def _norm_grad(s):
    case = s["case"]
    axis = 1 if case["order"] == "nchw" else 3
    pixels = [d for d in range(4) if d != axis]
    rstd, dy = s["rstd"].unsqueeze(axis), s["dy"].float()
    z = (s["x"].float() - s["mean"].unsqueeze(axis)) * rstd
    g = dy * _over(case, s["gamma"])
    dx = rstd * (g - g.mean(axis, keepdim=True) - z * (g * z).mean(axis, keepdim=True))
    return {"dx": dx.to(s["x"].dtype), "dgamma": (dy * z).sum(pixels), "dbeta": dy.sum(pixels)}


def _orthogonal(u):
    a, b, c = COEFFICIENTS
    x = u.t() if u.shape[0] > u.shape[1] else u
    x = x / (x.norm() + ORTH_EPS)
    for _ in range(STEPS):
        p = x @ x.t()
        x = a * x + (b * p + c * (p @ p)) @ x
    return x.t() if u.shape[0] > u.shape[1] else x


def _orth(s):
    return _orthogonal(s["g"].float()).contiguous().to(s["g"].dtype)


def _muon(s):
    for (k, _, _), w, g, m in zip(s["shapes"], s["ws"], s["gs"], s["ms"]):
        m.mul_(MOMENTUM).add_(g)
        u = (g + MOMENTUM * m).view(k, -1)
        w.mul_(1 - LR * DECAY).sub_(_orthogonal(u).view(w.shape), alpha=LR * math.sqrt(max(1.0, k / u.shape[1])))
    return {"w": s["w"], "m": s["m"]}


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------
def _orth_flops(rows, cols):
    m, n = min(rows, cols), max(rows, cols)
    return STEPS * (m * (m + 1.0) * n + m * (m + 1.0) * m + 2.0 * m * m * n)      # the first two products are symmetric


def work(case):
    if case["op"] == "orth":
        return {"bytes": 2.0 * case["rows"] * case["cols"] * _dtype(case).itemsize, "flops": _orth_flops(case["rows"], case["cols"])}
    if case["op"] == "muon":
        shapes = [(k, c * r * r) for k, c, r in _layers(case)]
        return {"bytes": 5 * 4.0 * sum(k * n for k, n in shapes), "flops": sum(_orth_flops(k, n) + 8.0 * k * n for k, n in shapes)}
    pixels, size = case["n"] * case["h"] * case["w"], _dtype(case).itemsize
    elements = pixels * case["c"]
    if case["op"] == "norm":
        return {"bytes": 2.0 * elements * size + 8 * case["c"] + (8 * pixels if case["stats"] else 0), "flops": 8.0 * elements}
    return {"bytes": 3.0 * elements * size + 12 * case["c"] + 8 * pixels, "flops": 14.0 * elements}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------
def _single(v):
    """A number as the 32-bit argument that it is passed as."""
    return struct.unpack("f", struct.pack("f", v))[0]


def _exact_orthogonal(u):
    """On Y = X^T (long axis first): Y <- Y (a + b S + c S^2), S = Y^T Y."""
    a, b, c = (_single(v) for v in COEFFICIENTS)
    long_first = u.shape[0] >= u.shape[1]
    y = u if long_first else u.transpose(0, 1).contiguous()
    y = y / (torch.sqrt((y * y).sum()) + _single(ORTH_EPS))
    one = torch.eye(y.shape[1], dtype=torch.float64, device=y.device)
    for _ in range(STEPS):
        s = y.transpose(0, 1) @ y
        y = y @ (a * one + s @ (b * one + c * s))
    return y if long_first else y.transpose(0, 1).contiguous()


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "orth":
        return _exact_orthogonal(s["g"].double())
    if case["op"] == "muon":
        mu, lr, decay = _single(MOMENTUM), _single(LR), _single(DECAY)
        ws, ms = [], []
        for (k, _, _), w, g, m in zip(s["shapes"], s["ws"], s["gs"], s["ms"]):
            w, g, m = (t.double().reshape(k, -1) for t in (w, g, m))
            m = mu * m + g
            ms.append(m.reshape(-1))
            ws.append((w - lr * (decay * w + math.sqrt(max(1.0, k / w.shape[1])) * _exact_orthogonal(g + mu * m))).reshape(-1))
        return {"w": torch.cat(ws), "m": torch.cat(ms)}
    last = (lambda t: t.permute(0, 2, 3, 1)) if case["order"] == "nchw" else (lambda t: t)
    back = (lambda t: t.permute(0, 3, 1, 2)) if case["order"] == "nchw" else (lambda t: t)
    x, gamma = last(s["x"].double()).reshape(-1, case["c"]), s["gamma"].double()
    shape = (case["n"], case["h"], case["w"])
    if case["op"] == "norm":
        mean = x.sum(1) / case["c"]
        var = (x - mean[:, None]).pow(2).sum(1) / case["c"]
        rstd = (var + _single(EPS)).pow(-0.5)
        y = (x - mean[:, None]) * rstd[:, None] * gamma + s["beta"].double()
        y = back((torch.where(y > 0, y, torch.zeros_like(y)) if case["relu"] else y).reshape(*shape, -1)).contiguous()
        return {"y": y, "mean": mean.reshape(shape), "rstd": rstd.reshape(shape)} if case["stats"] else y
    dy = last(s["dy"].double()).reshape(-1, case["c"])
    mean, rstd = (s[k].double().reshape(-1, 1) for k in ("mean", "rstd"))
    z = (x - mean) * rstd
    dz = dy * gamma
    dx = rstd * (dz - dz.sum(1, keepdim=True) / case["c"] - z * ((dz * z).sum(1, keepdim=True) / case["c"]))
    return {"dx": back(dx.reshape(*shape, -1)).contiguous(), "dgamma": (dy * z).sum(0), "dbeta": dy.sum(0)}
