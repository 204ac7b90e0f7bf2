"""A slim layer with a normalisation of its own, learned on the GPU: the steps against the same steps in 64 bits, and the layer in a network."""
import numpy as np
import pytest

import oracle
from paper_1708_04728_amd import binding as B, graph as G
from paper_1708_04728_amd.fit import NormalisedSlimLayer
from test_gpu_orthogonal import newton_schulz
from util import TOL_BF16, TOL_F32, close, gpu, host, note

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def layernorm(z, gamma, beta, eps):
    mean = z.mean(1, keepdims=True)
    rstd = 1 / np.sqrt(((z - mean) ** 2).mean(1, keepdims=True) + eps)
    return (z - mean) * rstd * gamma[:, None, None] + beta[:, None, None], mean, rstd


def step64(s, x, y, stride, pad, lr, lr_vectors, mu, eps):
    """One step of NormalisedSlimLayer on the state dict s, in 64 bits; returns the loss before it."""
    z = oracle.conv2d(x, s["w"], s["b"], stride, pad)
    n, mean, rstd = layernorm(z, s["gamma"], s["beta"], eps)
    f = np.maximum(n, 0)
    dn = np.where(f > 0, 2 * (f - y), 0)
    xhat, g = (z - mean) * rstd, dn * s["gamma"][:, None, None]
    dz = rstd * (g - g.mean(1, keepdims=True) - xhat * (g * xhat).mean(1, keepdims=True))
    dw, db = oracle.conv2d_bwd_params(x, dz, s["w"].shape[2], s["w"].shape[3], stride, pad)
    k = s["w"].shape[0]
    s["m"] = mu * s["m"] + dw
    u = (dw + mu * s["m"]).reshape(k, -1)
    s["w"] = s["w"] - lr * np.sqrt(max(1.0, k / u.shape[1])) * newton_schulz(u).reshape(s["w"].shape)
    s["b"], s["gamma"], s["beta"] = s["b"] - lr_vectors * db, s["gamma"] - lr_vectors * (dn * xhat).sum((0, 2, 3)), s["beta"] - lr_vectors * dn.sum((0, 2, 3))
    return ((f - y) ** 2).sum()


@pytest.mark.parametrize("case", ((3, 16, 20, 24, 3, 2, 1), (2, 5, 13, 40, 5, 1, 2), (1, 3, 31, 9, 7, 4, 0)))
def test_steps_follow_64_bits(case):
    n, c, size, k, r, stride, pad = case
    rng = np.random.default_rng(k)
    x = np.abs(rng.standard_normal((n, c, size, size))).astype(np.float32)
    xg = gpu(x)
    layer = NormalisedSlimLayer(xg, k, r, stride, pad)
    w0 = (rng.standard_normal((k, c, r, r)) * np.sqrt(2.0 / (c * r * r))).astype(np.float32)
    layer.w.copy_(gpu(w0))
    teacher = (rng.standard_normal((k, c, r, r)) * np.sqrt(2.0 / (c * r * r))).astype(np.float32)
    y = np.maximum(layernorm(oracle.conv2d(x, teacher, np.zeros(k), stride, pad), np.ones(k), np.zeros(k), 1e-5)[0], 0).astype(np.float32)
    s = dict(w=w0.astype(np.float64), b=np.zeros(k), gamma=np.ones(k), beta=np.zeros(k), m=np.zeros(w0.shape))
    lr, mu = 0.02, float(np.float32(0.95))
    lr_vectors = float(np.float32(0.05 / (n * y.shape[2] * y.shape[3])))
    yg, got, ref = gpu(y), [], []
    for _ in range(6):
        layer.step(xg, yg, float(np.float32(lr)), lr_vectors)
        got.append(float(layer.loss.item()))
        ref.append(step64(s, x, y, stride, pad, float(np.float32(lr)), lr_vectors, mu, float(np.float32(1e-5))))
    assert got[-1] < got[0]
    # a step's direction is off by (steps + 1) a^steps 2^-23 = 3.5e-4 of a matrix of norm about sqrt(min(k, c r r)) at worst (see test_gpu_orthogonal.py); the
    # loss's slope along it, over six steps, stays within the loss itself
    np.testing.assert_allclose(got, ref, rtol=6 * 3.5e-4)
    # six moves of lr, each off by that much in all; an element's share of it beside the weights' rms
    off = np.linalg.norm(host(layer.w) - s["w"])
    assert note("weights", off, 6 * lr * np.sqrt(max(1, k / (c * r * r))) * 3.5e-4 * np.sqrt(min(k, c * r * r)))
    for v, name in ((layer.gamma, "gamma"), (layer.beta, "beta")):
        assert close(host(v), s[name], 10 * TOL_F32, name)


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("fuse", (False, True))
def test_layer_in_a_network(dtype, fuse):
    """conv - layernorm - ReLU, twice, as a layer list: every order and data type, layer by layer and with the ReLU in the normalisation's store."""
    rng = np.random.default_rng(6)
    n, c, size = 3, 16, 18
    layers = [("conv", {"k": 24, "r": 3, "s": 3, "stride": 2, "pad": 1}), ("layernorm", {"eps": 1e-5}), ("relu", {}),
              ("conv", {"k": 40, "r": 1, "s": 1, "stride": 1, "pad": 0}), ("layernorm", {"eps": 1e-5}), ("relu", {})]
    x = rng.standard_normal((n, c, size, size)).astype(np.float32)
    rnd = oracle.round_bf16 if dtype == "bf16" else (lambda a: np.asarray(a, dtype=np.float64))
    x = rnd(x)
    params, cur, cin = [], x, c
    for kind, p in layers:
        if kind == "conv":
            w, b = rnd(rng.standard_normal((p["k"], cin, p["r"], p["r"])) * np.sqrt(2.0 / (cin * p["r"] ** 2))), 0.01 * rng.standard_normal(p["k"]).astype(np.float32)
            w = w.astype(np.float32)
            params.append({"w": w, "b": b})
            cur, cin = rnd(oracle.conv2d(cur, w, b, p["stride"], p["pad"])), p["k"]
        elif kind == "layernorm":
            g, b = (1 + 0.2 * rng.standard_normal(cin)).astype(np.float32), (0.2 * rng.standard_normal(cin)).astype(np.float32)
            params.append({"gamma": g, "beta": b})
            cur = rnd(layernorm(cur, g.astype(np.float64), b.astype(np.float64), p["eps"])[0])
        else:
            cur = np.maximum(cur, 0)
    net = B.Net(G.net_descs(layers, c, fuse_relu=fuse, pack=dtype))
    assert net.num_params() == 8
    xd = G.to_device(x, dtype, nhwc=dtype == "bf16")
    y = G.empty_like_desc(net.output_desc(B.desc(xd)))
    ws = torch.empty(max(net.workspace_bytes(B.desc(xd)), 256), dtype=torch.uint8, device="cuda")
    flat = G.flat_params(params, dtype, pack=True)
    net.fwd(xd, flat, y, ws)
    torch.cuda.synchronize()
    got = G.to_host(y)
    # two convolutions and two normalisations: four roundings to bf16 on the deepest path
    assert close(got, cur, TOL_F32 if dtype == "f32" else 2 * TOL_BF16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = net.capture(xd, flat, y, ws, side)
    first = (y.t if isinstance(y, B.NHWC) else y).clone()
    for _ in range(3):
        (y.t if isinstance(y, B.NHWC) else y).fill_(float("nan"))
        graph.launch()
        torch.cuda.synchronize()
        assert torch.equal(y.t if isinstance(y, B.NHWC) else y, first)
