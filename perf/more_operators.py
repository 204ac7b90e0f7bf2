"""What the operators that adapt a slimmed network's classifier are timed on: dropout, low-rank adapters of many requests beside one
shared projection with their gradient, and the softmax loss with its gradient.

Formulas:

* dropout: T = round(65536 p); element i, in memory order, has the 16-bit number d = half i % 8 of Philox4x32-10 (Salmon et al. 2011) of
  counter (i / 8, offset) under the key `seed`; y = x 65536 / (65536 - T) where d >= T, else 0.
* adapter: for every pixel i of an image with adapter a: t = s_a A_a drop(x_i), y_i = W x_i + b + B_a t; images with a = -1 have no
  adapter (t = 0).  "keep": t is an output too, for the gradient.
* adapter_grad: u = s_a B_a^T dy_i, dx_i = W^T dy_i + drop'(A_a^T u) with the forward pass's mask and scale,
  dA_a = sum u drop(x_i)^T, dB_a = sum dy_i t^T over the pixels of adapter a.  W and b are shared and fixed.
* loss: with the label j* of a row of c logits: l = log sum exp z - (1 - e) z_j* - e / c sum z, dz = (softmax(z) - (1 - e) [j = j*] - e / c) / n,
  over the n rows that have a label (0 <= j* < c); rows without one have l = 0 and dz = 0.  The loss is the mean of l.

Plain forms are computed in 32 bits with elementary torch operations and rounded once at the end.
"""
from __future__ import annotations

import math
import struct

import numpy as np
import torch

own = False

SMOOTHING = 0.1


def listed():
    return [
        # dropout in front of the classifier, one batch of feature vectors
        dict(name="dropout_features_bf16", op="dropout", dtype="bf16", order="nhwc", n=32, c=1024, h=1, w=1, p=0.4),
        # dropout on an odd map in channel planes
        dict(name="dropout_ragged_f32", op="dropout", dtype="f32", order="nchw", n=13, c=509, h=31, w=45, p=0.1),
        # ... on the second convolution's map of a full batch
        dict(name="dropout_map_bf16_b128", op="dropout", dtype="bf16", order="nhwc", n=128, c=192, h=56, w=56, p=0.5),
        # the loss of one batch of the classifier
        dict(name="loss_classifier_bf16", op="loss", dtype="bf16", rows=128, classes=1000, smoothing=False),
        # an odd number of classes, labels missing in places
        dict(name="loss_ragged_f32", op="loss", dtype="f32", rows=515, classes=32003, smoothing=True),
        # a large batch over many classes
        dict(name="loss_large_bf16", op="loss", dtype="bf16", rows=8192, classes=32768, smoothing=False),
        # one feature vector through the classifier and its adapter
        dict(name="adapter_one_vector_bf16", op="adapter", dtype="bf16", n=1, h=1, w=1, cin=1024, cout=1000, rank=8, adapters=1, runs=False, p=0.0),
        # one vector each of 64 requests, each with an adapter of its own
        dict(name="adapter_requests_bf16", op="adapter", dtype="bf16", n=64, h=1, w=1, cin=4096, cout=4096, rank=16, adapters=64, runs=False, p=0.0),
        # the first step of a module on an odd batch of ragged maps, five tasks in turn
        dict(name="adapter_maps_f32", op="adapter", dtype="f32", n=19, h=15, w=13, cin=528, cout=256, rank=12, adapters=5, runs=False, p=0.0),
        # many vectors of eight tasks, as a training step runs them
        dict(name="adapter_many_bf16", op="adapter", dtype="bf16", n=8192, h=1, w=1, cin=4096, cout=4096, rank=16, adapters=8, runs=False, p=0.1),
        # the gradient of one batch of the classifier, one adapter
        dict(name="adapter_grad_classifier_f32", op="adapter_grad", dtype="f32", n=128, h=1, w=1, cin=1024, cout=1000, rank=8, adapters=1, runs=False, p=0.4),
        # the gradient of adapter_many_bf16
        dict(name="adapter_grad_many_bf16", op="adapter_grad", dtype="bf16", n=8192, h=1, w=1, cin=4096, cout=4096, rank=16, adapters=8, runs=False, p=0.1),
    ]


def _log(rng, lo, hi):
    """A whole number whose logarithm is spread evenly over [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("dropout", "loss", "adapter", "adapter", "adapter_grad", "adapter_grad"))
    dtype = rng.choice(("f32", "bf16", "bf16"))
    if op == "loss":
        case = dict(op=op, dtype=dtype, rows=_log(rng, 1, 16384), classes=_log(rng, 2, 65536), smoothing=rng.random() < 0.5)
        while case["rows"] * case["classes"] > (1 << 27):
            case["rows"] //= 2
        return case
    if op == "dropout":
        case = dict(op=op, dtype=dtype, order=rng.choice(("nchw", "nhwc")), n=_log(rng, 1, 256), c=_log(rng, 1, 4096), h=_log(rng, 1, 64), w=_log(rng, 1, 64), p=rng.choice((0.05, 0.1, 0.4, 0.5, 0.9)))
        while case["n"] * case["c"] * case["h"] * case["w"] > (1 << 26):
            big = max(("n", "h", "w", "c"), key=lambda k: case[k])
            case[big] = max(1, case[big] // 2)
        return case
    maps = rng.random() < 0.4
    case = dict(op=op, dtype=dtype, n=_log(rng, 1, 64 if maps else 8192), h=_log(rng, 2, 56) if maps else 1, w=_log(rng, 2, 56) if maps else 1,
                cin=_log(rng, 8, 4096), cout=_log(rng, 8, 4096), rank=_log(rng, 1, 64), adapters=_log(rng, 1, 64), runs=rng.random() < 0.5, p=rng.choice((0.0, 0.0, 0.1, 0.4)))
    while work(case)["flops"] > (2e11 if dtype == "bf16" else 2e10) or case["n"] * case["h"] * case["w"] * case["adapters"] * case["rank"] > (1 << 26):
        big = max(("n", "h", "w"), key=lambda k: case[k])
        case[big] = max(1, case[big] // 2)
    return case


# ---- inputs ------------------------------------------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _map_shape(case):
    n, c, h, w = (case[d] for d in ("n", "c", "h", "w"))
    return (n, c, h, w) if case["order"] == "nchw" else (n, h, w, c)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case=case)
    dt = _dtype(case)
    normal = lambda *shape: torch.randn(shape, device="cuda", generator=gen)
    # what a program passes as the generator's key and place: a seed of its run, and where this layer's draws begin
    s["seed"], s["offset"] = 0x9E3700000000 + seed, (seed % 1000) * 0x100000001 + 7
    if case["op"] == "dropout":
        s["x"] = normal(*_map_shape(case)).to(dt)
    elif case["op"] == "loss":
        rows, classes = case["rows"], case["classes"]
        # logits of a network that knows something: the labelled class lies higher
        s["labels"] = torch.randint(0, classes, (rows,), device="cuda", generator=gen, dtype=torch.int32)
        z = 2 * normal(rows, classes)
        z[torch.arange(rows, device="cuda"), s["labels"].long()] += 4
        s["z"] = z.to(dt)
        del z
        if rows > 8:                                             # rows without a label
            s["labels"][torch.rand(rows, device="cuda", generator=gen) < 0.1] = -1
    else:
        n, h, w, cin, cout, rank, count = (case[k] for k in ("n", "h", "w", "cin", "cout", "rank", "adapters"))
        # features behind a ReLU, averaged or not
        s["x"] = normal(n, h, w, cin).abs_().to(dt)
        s["w"] = (normal(cout, cin) * math.sqrt(2.0 / cin)).to(dt)
        s["bias"] = 0.01 * normal(cout)
        s["a"] = (normal(count, rank, cin) * math.sqrt(1.0 / cin)).to(dt)
        s["b"] = (normal(count, cout, rank) * (0.5 / math.sqrt(rank))).to(dt)
        s["scales"] = 0.5 + torch.rand(count, device="cuda", generator=gen)
        ids = torch.randint(0, count, (n,), device="cuda", generator=gen, dtype=torch.int32)
        if n == count:                                           # each request has an adapter of its own
            ids = torch.randperm(n, device="cuda", generator=gen).to(torch.int32)
        elif n > 8:                                              # requests without an adapter
            ids[torch.rand(n, device="cuda", generator=gen) < 0.1] = -1
        s["ids"] = torch.sort(ids)[0].contiguous() if case["runs"] else ids
        if case["op"] == "adapter_grad":
            s["dy"] = (normal(n, h, w, cout) * 0.01).to(dt)
            s["inner"] = _inner(s)
    if own:
        _buffers(s)
    return s


def _buffers(s):
    """The outputs and the scratch memory that a program keeps from call to call."""
    from paper_1708_04728_amd import binding as B
    case = s["case"]
    scratch = lambda n: torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
    s["drop"] = B.dropout_desc(case["p"], s["seed"], s["offset"]) if case.get("p") else None
    if case["op"] == "dropout":
        tensor = B.NHWC if case["order"] == "nhwc" else lambda t: t
        s["out"] = torch.empty_like(s["x"])
        s["tx"], s["ty"] = tensor(s["x"]), tensor(s["out"])
    elif case["op"] == "loss":
        s["dz"], s["row_loss"], s["loss"] = torch.empty_like(s["z"]), torch.empty(case["rows"], device="cuda"), torch.empty(1, device="cuda")
        s["scratch"] = scratch(B.softmax_loss_workspace_bytes(s["z"]))
    else:
        n, h, w = (case[k] for k in ("n", "h", "w"))
        s["tx"] = B.NHWC(s["x"])
        if case["op"] == "adapter":
            s["y"] = torch.empty((n, h, w, case["cout"]), dtype=s["x"].dtype, device="cuda")
            s["t"] = torch.empty((n, h, w, case["rank"]), device="cuda") if case["p"] else None
            s["scratch"] = scratch(B.adapter_fwd_workspace_bytes(s["tx"], s["a"], s["b"]))
            s["ty"] = B.NHWC(s["y"])
        else:
            s["dx"] = torch.empty_like(s["x"])
            s["da"], s["db"] = (torch.empty(s[k].shape, device="cuda") for k in ("a", "b"))
            s["scratch"] = scratch(B.adapter_bwd_workspace_bytes(s["tx"], s["a"], s["b"]))
            s["tdy"], s["tdx"] = B.NHWC(s["dy"]), B.NHWC(s["dx"])


# ---- one pass ------------------------------------------------------------------------------------------------------------
def run(s):
    return (_run_own if own else {"dropout": _dropout, "loss": _loss, "adapter": _adapter, "adapter_grad": _adapter_grad}[s["case"]["op"]])(s)


def _run_own(s):
    from paper_1708_04728_amd import binding as B
    case = s["case"]
    if case["op"] == "dropout":
        B.dropout_fwd(s["tx"], s["drop"], s["ty"])
        return s["out"]
    if case["op"] == "loss":
        B.softmax_loss_grad(s["z"], s["labels"], s["dz"], s["loss"], s["scratch"], smoothing=SMOOTHING if case["smoothing"] else 0.0, row_loss=s["row_loss"])
        return {"dz": s["dz"], "row_loss": s["row_loss"], "loss": s["loss"]}
    if case["op"] == "adapter":
        B.adapter_fwd(s["tx"], s["w"], s["bias"], s["a"], s["b"], s["ids"], s["ty"], s["scratch"], scales=s["scales"], drop=s["drop"], inner=s["t"])
        return {"y": s["y"], "inner": s["t"]} if case["p"] else s["y"]
    B.adapter_bwd(s["tdy"], s["tx"], s["w"], s["a"], s["b"], s["ids"], s["inner"], s["tdx"], s["da"], s["db"], s["scratch"], scales=s["scales"], drop=s["drop"])
    return {"dx": s["dx"], "da": s["da"], "db": s["db"]}


def _times(m, v):
    """High and low 32 bits of the products of m and the 32-bit numbers v (both held in 64 bits)."""
    low = m * (v & 0xFFFF)
    mid = m * (v >> 16) + (low >> 16)
    return mid >> 16, ((mid & 0xFFFF) << 16) | (low & 0xFFFF)


def _scaled_mask(shape, p, seed, offset):
    """What dropout multiplies by: 65536 / (65536 - T) where an element is kept, else 0."""
    count, border = math.prod(shape), int(math.floor(p * 65536 + 0.5))
    c0 = torch.arange((count + 7) // 8, device="cuda")
    c1, c2, c3 = c0 >> 32, torch.full_like(c0, offset & 0xFFFFFFFF), torch.full_like(c0, offset >> 32)
    c0 = c0 & 0xFFFFFFFF
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        (h0, l0), (h1, l1) = _times(0xD2511F53, c0), _times(0xCD9E8D57, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    draws = torch.stack([half for c in (c0, c1, c2, c3) for half in (c & 0xFFFF, c >> 16)], 1).view(-1)[:count]
    return ((draws >= border).float() * (65536 / (65536 - border))).view(shape)


def _dropped(s, x):
    p = s["case"]["p"]
    return x * _scaled_mask(x.shape, p, s["seed"], s["offset"]) if p else x


def _dropout(s):
    return _dropped(s, s["x"].float()).to(s["x"].dtype)


def _loss(s):
    z, classes, e = s["z"].float(), s["case"]["classes"], SMOOTHING if s["case"]["smoothing"] else 0.0
    has = s["labels"] >= 0
    label = s["labels"].clamp(min=0).long()[:, None]
    top = z.max(1, keepdim=True)[0]
    d = z - top
    ex = d.exp()
    total = ex.sum(1, keepdim=True)
    row = total.log() - (1 - e) * d.gather(1, label)
    if e:
        row = row - e * d.mean(1, keepdim=True)
    row = torch.where(has, row[:, 0], 0.0)
    n = has.sum().clamp(min=1).float()
    dz = ex.div_(total).sub_(e / classes)
    dz[torch.arange(len(z), device="cuda"), label[:, 0]] -= 1 - e
    dz = torch.where(has[:, None], dz / n, 0.0)
    return {"dz": dz.to(s["z"].dtype), "row_loss": row, "loss": (row.double().sum() / n).float().view(1)}


def _chosen(s):
    """(pixels, adapters): the scale of each pixel's adapter, 0 for the others."""
    case = s["case"]
    ids = s["ids"][:, None].expand(-1, case["h"] * case["w"]).reshape(-1, 1)
    return (ids == torch.arange(case["adapters"], device="cuda", dtype=torch.int32)).float()


def _inner_of_all(s):
    """(pixels, adapters, rank): t in its adapter's place, 0 elsewhere."""
    case = s["case"]
    x = _dropped(s, s["x"].float()).view(-1, case["cin"])
    t = (x @ s["a"].float().view(-1, case["cin"]).t()).view(-1, case["adapters"], case["rank"])
    return t * (_chosen(s) * s["scales"])[:, :, None]


def _inner(s):
    case = s["case"]
    return _inner_of_all(s).sum(1).view(case["n"], case["h"], case["w"], case["rank"])


def _adapter(s):
    case = s["case"]
    t = _inner_of_all(s)
    y = s["x"].float().view(-1, case["cin"]) @ s["w"].float().t() + s["bias"]
    y = y + t.view(len(t), -1) @ s["b"].float().permute(0, 2, 1).reshape(-1, case["cout"])
    y = y.view(case["n"], case["h"], case["w"], -1).to(s["x"].dtype)
    return {"y": y, "inner": t.sum(1).view(case["n"], case["h"], case["w"], -1)} if case["p"] else y


def _adapter_grad(s):
    case = s["case"]
    dy = s["dy"].float().view(-1, case["cout"])
    chosen = _chosen(s)
    u = (dy @ s["b"].float().permute(1, 0, 2).reshape(case["cout"], -1)).view(-1, case["adapters"], case["rank"])
    u = (u * (chosen * s["scales"])[:, :, None]).view(len(dy), -1)
    t = (chosen[:, :, None] * s["inner"].view(-1, 1, case["rank"])).view(len(dy), -1)
    through = (u @ s["a"].float().view(-1, case["cin"])).view(s["x"].shape)
    x = s["x"].float()
    if case["p"]:
        mask = _scaled_mask(x.shape, case["p"], s["seed"], s["offset"])
        through, x = through * mask, x * mask
    dx = (dy @ s["w"].float()).view(x.shape) + through
    da = (u.t() @ x.view(-1, case["cin"])).view(s["a"].shape)
    db = (dy.t() @ t).view(case["cout"], case["adapters"], case["rank"]).permute(1, 0, 2).contiguous()
    return {"dx": dx.to(s["x"].dtype), "da": da, "db": db}


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------
def work(case):
    size = _dtype(case).itemsize
    if case["op"] == "dropout":
        count = case["n"] * case["c"] * case["h"] * case["w"]
        return {"bytes": 2.0 * count * size, "flops": 1.0 * count}
    if case["op"] == "loss":
        count = case["rows"] * case["classes"]
        return {"bytes": 2.0 * count * size + 8.0 * case["rows"], "flops": 6.0 * count}
    rows, cin, cout, rank = case["n"] * case["h"] * case["w"], case["cin"], case["cout"], case["rank"]
    present = min(case["adapters"], case["n"])
    shared = size * (cin * cout + present * rank * (cin + cout)) + 4.0 * case["n"]
    if case["op"] == "adapter":
        return {"bytes": shared + size * rows * (cin + cout) + (4.0 * rows * rank if case["p"] else 0), "flops": 2.0 * rows * (cin * cout + rank * (cin + cout))}
    return {"bytes": shared + size * rows * (2 * cin + cout) + 4.0 * rows * rank + 4.0 * case["adapters"] * rank * (cin + cout),
            "flops": 2.0 * rows * (cin * cout + 2 * rank * (cin + cout))}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------
def _single(v):
    """A number as the 32-bit argument that it is passed as."""
    return struct.unpack("f", struct.pack("f", v))[0]


def _exact_keep(shape, p, seed, offset):
    """The kept elements, by the generator's definition on the host's 64-bit products."""
    count = int(np.prod(shape))
    block = np.arange(-(-count // 8), dtype=np.uint64)
    low32, by32 = np.uint64(0xFFFFFFFF), np.uint64(32)
    word = [block & low32, block >> by32, np.uint64(offset & 0xFFFFFFFF), np.uint64(offset >> 32)]
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        first, second = np.uint64(0xD2511F53) * word[0], np.uint64(0xCD9E8D57) * word[2]
        word = [(second >> by32) ^ word[1] ^ np.uint64(key[0]), second & low32, (first >> by32) ^ word[3] ^ np.uint64(key[1]), first & low32]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    halves = np.empty((len(block), 4), dtype="<u4")
    for i, v in enumerate(word):
        halves[:, i] = v
    draws = halves.view("<u2").reshape(-1)[:count]
    return torch.from_numpy(draws >= round(p * 65536)).to("cuda").view(shape)


def exact(case, seed):
    s = prepare(case, seed)
    x = s["x"].double() if "x" in s else None
    mask = None
    if case.get("p"):
        mask = _exact_keep(tuple(x.shape), case["p"], s["seed"], s["offset"]).double() * (65536.0 / (65536 - round(case["p"] * 65536)))
    if case["op"] == "dropout":
        return x * mask
    if case["op"] == "loss":
        e = _single(SMOOTHING) if case["smoothing"] else 0.0
        rows, classes = s["z"].shape
        target = torch.zeros(rows, classes, dtype=torch.float64, device="cuda") + e / classes
        has = (s["labels"] >= 0).double()
        target.scatter_add_(1, s["labels"].clamp(min=0).long().view(-1, 1), torch.full((rows, 1), 1 - e, dtype=torch.float64, device="cuda"))
        z = s["z"].double()
        lse = torch.logsumexp(z, 1)
        row = has * (lse - (target * z).sum(1))
        n = max(1.0, float(has.sum()))
        z.sub_(lse.view(-1, 1)).exp_().sub_(target).mul_((has / n).view(-1, 1))
        return {"dz": z, "row_loss": row, "loss": (row.sum() / n).view(1)}
    pixels = case["h"] * case["w"]
    dropped = (x * mask if mask is not None else x).view(-1, case["cin"])
    w, scales = s["w"].double(), s["scales"].double()
    ids = s["ids"].repeat_interleave(pixels)
    members = [(a, (ids == a).nonzero().view(-1)) for a in range(case["adapters"])]
    if case["op"] == "adapter":
        y = torch.addmm(s["bias"].double(), x.view(-1, case["cin"]), w.t())
        t = torch.zeros(len(y), case["rank"], dtype=torch.float64, device="cuda")
        for a, i in members:
            if len(i):
                t[i] = scales[a] * (dropped[i] @ s["a"][a].double().t())
                y[i] += t[i] @ s["b"][a].double().t()
        y = y.view(*x.shape[:3], -1)
        return {"y": y, "inner": t.view(*x.shape[:3], -1)} if case["p"] else y
    dy, t = s["dy"].double().view(-1, case["cout"]), s["inner"].double().view(-1, case["rank"])
    dx = dy @ w
    da, db = torch.zeros(s["a"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["b"].shape, dtype=torch.float64, device="cuda")
    for a, i in members:
        if len(i):
            u = scales[a] * (dy[i] @ s["b"][a].double())
            back = u @ s["a"][a].double()
            dx[i] += back if mask is None else back * mask.view(-1, case["cin"])[i]
            da[a] = u.t() @ dropped[i]
            db[a] = dy[i].t() @ t[i]
    return {"dx": dx.view(x.shape), "da": da, "db": db}
