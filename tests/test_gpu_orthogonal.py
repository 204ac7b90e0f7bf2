"""Newton-Schulz orthogonalisation and the descent step on it against the formulas in 64 bits.

Tolerance.  X, A, Q and their products are kept to a relative u: 2^-23 for fp32 (rounding of the value and of a sum), 2^-17 for bf16 (two pieces of 8 bits and the product
that is left out).  A step multiplies an error in X by at most a (the polynomial's slope at zero, its largest), and |X|_F by at most a from 1 on: after s steps the errors of
the s + 1 matrices X come to at most (s + 1) a^s u, in the Frobenius norm.  A bf16 result is then rounded: up to 2^-8 of each element."""
import numpy as np
import pytest

from paper_1708_04728_amd import binding as B
from util import case_seed, note

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

COEFFICIENTS = tuple(float(np.float32(v)) for v in B.NEWTON_SCHULZ)
EPS = float(np.float32(1e-7))
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def newton_schulz(u, steps=5, coefficients=COEFFICIENTS, eps=EPS):
    a, b, c = coefficients
    x = u.T if u.shape[0] > u.shape[1] else u
    x = x / (np.sqrt((x * x).sum()) + eps)
    for _ in range(steps):
        p = x @ x.T
        x = a * x + (b * p + c * (p @ p)) @ x
    return x.T if u.shape[0] > u.shape[1] else x


def bound(ref, dtype, steps=5, a=COEFFICIENTS[0]):
    """Of |got - ref|_F."""
    u = 2.0 ** -17 if dtype == "bf16" else 2.0 ** -23
    return (steps + 1) * max(abs(a), 1) ** steps * u + (2.0 ** -8 * np.linalg.norm(ref) if dtype == "bf16" else 0)


def gradient(rng, rows, cols):
    """A filter gradient: gradients behind a ReLU times features behind a ReLU, summed over pixels."""
    pixels = 2 * min(rows, cols) + 64
    return ((rng.standard_normal((rows, pixels)) * (rng.random((rows, pixels)) < 0.6)) @ np.abs(rng.standard_normal((pixels, cols)))).astype(np.float32)


def scratch(n, fill=255):
    return torch.full((max(n, 256),), fill, dtype=torch.uint8, device="cuda")


def run(gs, **kw):
    out = [torch.full_like(g, float("nan")) for g in gs]
    B.orthogonalise(gs, out, scratch(B.orthogonalise_workspace_bytes(gs)), **kw)
    torch.cuda.synchronize()
    return out


def on_gpu(a, dtype="f32", offset=0):
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DTYPES[dtype]).cuda()
    flat = torch.empty(t.numel() + offset, dtype=t.dtype, device="cuda")
    out = flat[offset:].view(t.shape)
    out.copy_(t)
    return out


def array(t):
    return t.double().cpu().numpy()


def check(got, g, dtype, what="", **kw):
    ref = newton_schulz(array(g).reshape(g.shape[0], -1), **kw)
    tol = bound(ref, dtype, **{k: v for k, v in kw.items() if k == "steps"}, a=kw.get("coefficients", COEFFICIENTS)[0])
    return note("|error| " + what, np.linalg.norm(array(got).reshape(ref.shape) - ref) / tol, 1.0)


SHAPES = [(1, 1), (1, 7), (7, 1), (2, 3), (16, 16), (31, 33), (32, 32), (33, 31), (64, 147), (147, 64), (64, 64), (65, 200), (3, 1000), (1000, 3), (96, 363), (192, 576), (16, 4000), (4000, 16),
          (129, 129), (500, 301), (256, 2400), (384, 864), (700, 1300), (1300, 700), (1000, 1024), (64, 20000), (1500, 1501)]


# shared contractions and the largest tiles, the reference in 64 bits on the GPU (products of torch)
LARGE = [(500, 6000), (33000, 250), (1024, 4000), (2049, 2500), (2700, 2600), (3300, 3700), (4160, 4100), (4300, 4500)]


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("shape", LARGE)
def test_orthogonalise_large(shape, dtype):
    gen = torch.Generator(device="cuda").manual_seed(case_seed(shape))
    pixels = min(shape) + 500
    g = ((torch.randn((shape[0], pixels), device="cuda", generator=gen) @ torch.randn((pixels, shape[1]), device="cuda", generator=gen).abs())).to(DTYPES[dtype])
    got, = run([g])
    a, b, c = COEFFICIENTS
    x = g.double().t() if shape[0] > shape[1] else g.double()
    x = x / (x.norm() + EPS)
    for _ in range(5):
        p = x @ x.t()
        x = a * x + (b * p + c * (p @ p)) @ x
    ref = x.t() if shape[0] > shape[1] else x
    tol = 6 * a ** 5 * (2.0 ** -17 if dtype == "bf16" else 2.0 ** -23) + (2.0 ** -8 * ref.norm().item() if dtype == "bf16" else 0)
    again, = run([g])
    assert torch.equal(got, again)


# a polynomial that takes singular values to 4.9: beyond what two fp16 pieces hold
FAR = (12.5, -12.0, 0.5)


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("shape", SHAPES + LARGE)
def test_values_beyond_fp16(shape, dtype):
    """Two steps.  Singular values are at most 1, then m = 4.95; the polynomial's slope is at most l(1) = 51, then l(m): an error u |X| of the first X, 51 u of the second and
    4.95 u of the result's factors come to at most 3 l(1) l(m) u in the Frobenius norm, times |X| = 1."""
    gen = torch.Generator(device="cuda").manual_seed(case_seed(shape, 5))
    g = torch.randn(shape, device="cuda", generator=gen).to(DTYPES[dtype])
    got, = run([g], steps=2, coefficients=FAR)
    a, b, c = FAR
    x = g.double().t() if shape[0] > shape[1] else g.double()
    x = x / (x.norm() + EPS)
    for _ in range(2):
        p = x @ x.t()
        x = a * x + (b * p + c * (p @ p)) @ x
    ref = x.t() if shape[0] > shape[1] else x
    slope = lambda s: a - 3 * b * s ** 2 + 5 * c * s ** 4
    tol = 3 * slope(1.0) * slope(4.95) * 2.0 ** -23 + (2.0 ** -8 * ref.norm().item() if dtype == "bf16" else 0)
    assert note("|error|", (got.double() - ref).norm().item() / tol, 1.0)


def test_muon_step_beyond_fp16():
    rng = np.random.default_rng(8)
    for rows, cols in ((20, 300), (70, 90), (100, 700)):
        w, g, m = (rng.standard_normal((rows, cols)).astype(np.float32) for _ in range(3))
        tw, tg, tm = on_gpu(w), on_gpu(g), on_gpu(m)
        params = B.muon_params([(tw, tg, tm)])
        B.muon_step(params, scratch(B.muon_step_workspace_bytes(params)), 0.5, momentum=0.5, weight_decay=0.0, steps=1, coefficients=FAR, eps=0.0)
        torch.cuda.synchronize()
        m64 = 0.5 * m.astype(np.float64) + g
        o = newton_schulz(g + 0.5 * m64, 1, FAR, 0.0)
        ref = w - 0.5 * np.sqrt(max(1.0, rows / cols)) * o
        # one step: 2 l(1) u |X|, and the weights' own rounding
        assert note("weights", np.linalg.norm(array(tw) - ref) / (0.5 * 2 * 51 * 2.0 ** -23 + 2.0 ** -23 * np.linalg.norm(ref)), 1.0)


@pytest.mark.parametrize("shape", ((40, 60), (64, 147), (192, 576), (500, 700)))
@pytest.mark.parametrize("kind", ("rows of all sizes", "elements of all sizes", "three directions", "one element"))
def test_values_far_apart(shape, kind):
    """Rows or elements eight decades apart, a matrix of rank three, a single element: what is small is kept well enough for the bound on the whole."""
    rng = np.random.default_rng(case_seed((shape, kind)))
    g = rng.standard_normal(shape)
    if kind == "rows of all sizes":
        g *= np.logspace(0, -8, shape[0])[:, None]
    elif kind == "elements of all sizes":
        g *= 10 ** (-8 * rng.random(shape))
    elif kind == "three directions":
        g = g[:, :3] @ rng.standard_normal((3, shape[1]))
    else:
        g[:] = 0
        g[shape[0] // 2, shape[1] // 3] = 7
    g = g.astype(np.float32)
    got, = run([on_gpu(g)])
    ref = newton_schulz(g.astype(np.float64))
    assert note("|error|", np.linalg.norm(array(got) - ref) / bound(ref, "f32"), 1.0)


@pytest.mark.parametrize("shape", ((20, 30), (64, 100), (70, 90), (100, 3000), (300, 900)))
@pytest.mark.parametrize("below", (1, 3, 6, 10, 14, 20, 40))
def test_norms_below_eps(shape, below):
    """|G| = 2^-below eps: X starts as small, and small values are kept to the same relative precision as others.  An error u |X| of a matrix X grows as X does, at most
    a-fold in a step: |error| <= 6 a^5 u |X|, |X| = 2^-below at the start."""
    g = gradient(np.random.default_rng(case_seed(shape, below)), *shape)
    g = (g / np.linalg.norm(g.astype(np.float64)) * 2.0 ** -10).astype(np.float32)
    got, = run([on_gpu(g)], eps=2.0 ** (below - 10))
    ref = newton_schulz(g.astype(np.float64), eps=2.0 ** (below - 10))
    assert note("|error|", np.linalg.norm(array(got) - ref) / (6 * COEFFICIENTS[0] ** 5 * 2.0 ** -23 * 2.0 ** -below), 1.0)


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("shape", SHAPES)
def test_orthogonalise(shape, dtype):
    rng = np.random.default_rng(case_seed((shape, dtype)))
    for offset in (0, 1):
        g = on_gpu(gradient(rng, *shape), dtype, offset)
        got, = run([g])
        assert check(got, g, dtype)
        # the same bits again, and in place
        again, = run([g])
        assert torch.equal(got, again)
        B.orthogonalise([g], [g], scratch(B.orthogonalise_workspace_bytes([g]), 0))
        torch.cuda.synchronize()
        assert torch.equal(got, g)


def test_orthogonalise_moves_singular_values_and_keeps_vectors():
    rng = np.random.default_rng(5)
    g = gradient(rng, 48, 100)
    got, = run([on_gpu(g)])
    u, _, v = np.linalg.svd(g.astype(np.float64), full_matrices=False)
    inside = u.T @ array(got) @ v.T
    values = np.diag(inside)
    assert 0.6 < values.min() and values.max() < 1.25
    assert note("off the diagonal", np.abs(inside - np.diag(values)).max(), 6 * COEFFICIENTS[0] ** 5 * 2.0 ** -23)


@pytest.mark.parametrize("steps,coefficients,eps", ((1, COEFFICIENTS, EPS), (2, COEFFICIENTS, EPS), (3, (1.875, -1.25, 0.375), EPS), (12, (1.875, -1.25, 0.375), 0.0), (5, COEFFICIENTS, 0.5)))
def test_other_polynomials(steps, coefficients, eps):
    rng = np.random.default_rng(steps)
    for shape in ((40, 90), (200, 130)):
        g = on_gpu(gradient(rng, *shape) * (0.01 if eps == 0.5 else 1))
        got, = run([g], steps=steps, coefficients=coefficients, eps=eps)
        assert check(got, g, "f32", steps=steps, coefficients=coefficients, eps=eps)


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
def test_lists(dtype):
    """Many matrices of one call: each as by itself, whatever lies beside it; empty ones among them; more than one table's worth."""
    rng = np.random.default_rng(9)
    shapes = [(64, 147), (0, 5), (33, 31), (5, 0), (192, 576), (1, 1), (300, 40)] + [(int(a), int(b)) for a, b in rng.integers(1, 120, (80, 2))]
    gs = [on_gpu(gradient(rng, *s) if min(s) else np.zeros(s), dtype) for s in shapes]
    got = run(gs)
    for i, (o, g) in enumerate(zip(got, gs)):
        if g.numel():
            assert check(o, g, dtype, "%dx%d" % shapes[i])
    # beside matrices of zeros, infinities and NaN
    gs[4].zero_()
    gs[0][3, 5] = float("inf")
    gs[2][1, 1] = float("nan")
    wild = run(gs)
    assert not wild[4].any() and not torch.isfinite(wild[0]).any() and not torch.isfinite(wild[2]).any()
    for i in range(len(gs)):
        if i not in (0, 2, 4):
            assert torch.equal(wild[i], got[i])
    assert run([]) == []


@pytest.mark.parametrize("exponent", (-100, -30, 30, 100))
def test_scales(exponent):
    """Gradients far from one: the result depends on their direction alone (above eps)."""
    rng = np.random.default_rng(1)
    g = gradient(rng, 70, 90)
    one, = run([on_gpu(g)], eps=0.0)
    far, = run([on_gpu(g * np.float32(2.0 ** exponent))], eps=0.0)
    assert torch.equal(one, far)
    if exponent == -100:                    # far below eps: divided by it
        tiny = on_gpu(g * np.float32(2.0 ** exponent))
        got, = run([tiny])
        ref = newton_schulz(array(tiny))
        assert note("tiny", np.linalg.norm(array(got) - ref) / np.linalg.norm(ref), 6 * 2.0 ** -23)


def test_low_rank():
    """Singular values of zero stay at what rounding leaves of them."""
    rng = np.random.default_rng(3)
    for shape in ((60, 200), (200, 60), (300, 300)):
        g = on_gpu(rng.standard_normal((shape[0], 3)) @ rng.standard_normal((3, shape[1])))
        got, = run([g])
        assert check(got, g, "f32")


def muon(w, g, m, lr, mu, decay, **kw):
    lr, mu, decay = (float(np.float32(v)) for v in (lr, mu, decay))
    m = mu * m + g
    rows, cols = w.shape
    return (1 - lr * decay) * w - lr * np.sqrt(max(1.0, rows / cols)) * newton_schulz(g + mu * m, **kw), m


@pytest.mark.parametrize("lr,mu,decay", ((0.02, 0.95, 0.0), (0.3, 0.9, 0.1), (0.02, 0.0, 0.01)))
def test_muon_step(lr, mu, decay):
    """Filter tensors of several shapes, two steps."""
    rng = np.random.default_rng(7)
    shapes = [(64, 3, 7, 7), (16, 8, 1, 1), (200, 10, 3, 3), (300, 12, 1, 1), (1, 1, 3, 3), (24, 16, 5, 5), (130, 40)]
    w = [on_gpu(rng.standard_normal(s) * np.sqrt(2.0 / np.prod(s[1:]))) for s in shapes]
    g = [on_gpu(gradient(rng, s[0], int(np.prod(s[1:]))).reshape(s)) for s in shapes]
    m = [on_gpu(gradient(rng, s[0], int(np.prod(s[1:]))).reshape(s)) for s in shapes]
    params = B.muon_params(list(zip(w, g, m)))
    ws = scratch(B.muon_step_workspace_bytes(params))
    for turn in range(2):
        before = [(array(a).reshape(a.shape[0], -1), array(b).reshape(a.shape[0], -1), array(c).reshape(a.shape[0], -1)) for a, b, c in zip(w, g, m)]
        B.muon_step(params, ws, lr, momentum=mu, weight_decay=decay)
        torch.cuda.synchronize()
        for i, (w0, g0, m0) in enumerate(before):
            w1, m1 = muon(w0, g0, m0, lr, mu, decay)
            got_w, got_m = array(w[i]).reshape(w1.shape), array(m[i]).reshape(w1.shape)
            # momentum: a product and a sum in fp32; U: the same again
            assert note("momentum", (np.abs(got_m - m1) / (2.0 ** -23 * (np.abs(mu * m0) + np.abs(g0)) + 1e-30)).max(), 1.0)
            move = float(np.float32(lr)) * np.sqrt(max(1.0, w1.shape[0] / w1.shape[1]))
            # weights: two products and a sum in fp32; the direction: as above, from a U that is off by 2^-22 of its terms
            slack = np.linalg.norm(2.0 ** -22 * (np.abs(w0) + np.abs(w1))) + move * (bound(w1, "f32") + COEFFICIENTS[0] ** 5 * 2.0 ** -22 * (np.linalg.norm(g0) + np.linalg.norm(mu * m0)) / np.linalg.norm(g0 + mu * m1))
            assert note("weights", np.linalg.norm(got_w - w1) / slack, 1.0)


def test_muon_step_recorded():
    """A recorded step, replayed, takes the steps that eager calls take."""
    rng = np.random.default_rng(8)
    shapes = [(64, 3, 7, 7), (96, 40, 3, 3), (130, 60)]
    make = lambda: [tuple(on_gpu(v.reshape(s)) for v in t) for s, t in zip(shapes, start)]
    start = [[gradient(rng, s[0], int(np.prod(s[1:]))) for _ in range(3)] for s in shapes]
    a, b = make(), make()
    pa, pb = B.muon_params(a), B.muon_params(b)
    wa, wb = (scratch(B.muon_step_workspace_bytes(p)) for p in (pa, pb))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with B.capture(side, keep=(pb, wb)) as rec:
        B.muon_step(pb, wb, 0.02, weight_decay=0.01, stream=side)
    for turn in range(3):
        for (_, g, _), (_, h, _) in zip(a, b):
            g.mul_(0.5).add_(g.roll(1, 0))
            h.copy_(g)
        B.muon_step(pa, wa, 0.02, weight_decay=0.01)
        torch.cuda.synchronize()
        rec.graph.launch()
        torch.cuda.synchronize()
        for x, y in zip(a, b):
            assert all(torch.equal(u, v) for u, v in zip(x, y))
