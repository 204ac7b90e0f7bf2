"""Layer normalisation and its gradient on the GPU against the formulas in 64 bits.

Tolerances are bounds, not fits.  A sum of fp32 terms is off by at most (additions on its longest chain) x 2^-24 x (sum of the terms' magnitudes); the
chains are at most 96 additions for the sums over channels up to 8192 (a lane's own elements, then a tree), and the mean's error, at most 96 x 2^-24 x max |x|,
reaches y multiplied by rstd gamma.  A bf16 result adds half a unit in its last place, 2^-8 of its size (8 significant bits)."""
import numpy as np
import pytest

from paper_1708_04728_amd import binding as B
from util import case_seed, note

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24
EPS = float(np.float32(1e-5))


def chain(c):
    return 96 + c / 256


def at_offset(t, offset):
    """A copy of t that starts `offset` elements behind an allocation's start."""
    flat = torch.empty(t.numel() + offset, dtype=t.dtype, device="cuda")
    out = flat[offset:].view(t.shape)
    out.copy_(t)
    return out


class Case:
    """Tensors of one shape in one order, and the same as (pixels, c) arrays in 64 bits."""

    def __init__(self, n, c, h, w, dtype, order, offset=0):
        self.shape = (n, c, h, w) if order == "nchw" else (n, h, w, c)
        self.n, self.c, self.h, self.w, self.order, self.offset = n, c, h, w, order, offset
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.u = 2.0 ** -8 if dtype == "bf16" else U

    def tensor(self, rows):
        """(pixels, c) array -> device tensor in the case's order."""
        a = torch.from_numpy(np.ascontiguousarray(rows, dtype=np.float32)).view(self.n, self.h, self.w, self.c)
        if self.order == "nchw":
            a = a.permute(0, 3, 1, 2).contiguous()
        return at_offset(a.to(self.dtype).cuda(), self.offset)

    def wrap(self, t):
        return B.NHWC(t) if self.order == "nhwc" else t

    def rows(self, t):
        a = t.double().cpu()
        if self.order == "nchw":
            a = a.permute(0, 2, 3, 1)
        return a.reshape(-1, self.c).numpy()

    def empty(self):
        return at_offset(torch.full(self.shape, float("nan"), dtype=self.dtype, device="cuda"), self.offset)


def vectors(c, rng):
    return (1 + 0.2 * rng.standard_normal(c)).astype(np.float32), (0.3 * rng.standard_normal(c)).astype(np.float32)


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()


def statistics(x):
    mean = x.mean(1)
    return mean, 1 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + EPS)


def forward(k, x, gamma, beta, relu, stats=True, out=None):
    pixels = k.n * k.h * k.w
    y = k.empty() if out is None else out
    mean, rstd = (torch.full((pixels,), float("nan"), device="cuda") if stats else None for _ in range(2))
    B.layernorm_fwd(k.wrap(x), None if gamma is None else cuda(gamma), None if beta is None else cuda(beta), EPS, relu, k.wrap(y), mean, rstd)
    torch.cuda.synchronize()
    return y, mean, rstd


def check_forward(k, x, gamma, beta, relu, got, mean_got, rstd_got):
    x = k.rows(x)
    mean, rstd = statistics(x)
    g, b = (np.ones(k.c) if gamma is None else gamma.astype(np.float64)), (np.zeros(k.c) if beta is None else beta.astype(np.float64))
    y = (x - mean[:, None]) * rstd[:, None] * g + b
    if relu:
        y = np.maximum(y, 0)
    most = np.abs(x).max(1)
    # mean: a chain of additions; rstd: relative to itself, through differences that are off by the mean's error (at worst in every element)
    d_mean = (chain(k.c) + 2) * U * most
    d_rstd = (chain(k.c) + 8) * U + np.minimum(d_mean * rstd, 1) ** 2 + 2 * U * most * rstd
    tol = (d_mean[:, None] * rstd[:, None] + np.abs(x - mean[:, None]) * rstd[:, None] * (d_rstd[:, None] + 4 * U)) * np.abs(g) + 4 * U * (np.abs(b) + np.abs(y)) + 1.01 * k.u * np.abs(y)
    # (where the result is rounded to bf16, the smallest step it can take is that of the value it is near)
    assert note("y", (np.abs(k.rows(got) - y) / (tol * (1 + k.u) + 1e-30)).max(), 1.0)
    if mean_got is not None:
        assert note("mean", (np.abs(mean_got.double().cpu().numpy() - mean) / (d_mean + 1e-30)).max(), 1.0)
        assert note("rstd", (np.abs(rstd_got.double().cpu().numpy() / rstd - 1) / d_rstd).max(), 1.0)


# n, c, h, w
SHAPES = [
    (1, 1, 1, 1), (5, 1, 3, 3), (1, 3, 7, 9), (2, 7, 5, 5), (3, 8, 1, 1), (130, 16, 1, 1), (1, 24, 63, 1), (2, 64, 13, 5), (3, 65, 8, 8), (1, 96, 1, 129),
    (2, 192, 14, 14), (7, 333, 3, 5), (3, 509, 5, 7), (1, 512, 8, 8), (1, 1000, 1, 1), (4, 1024, 3, 3), (300, 1024, 1, 1), (2, 1100, 7, 3), (3, 2048, 2, 2), (5, 2056, 1, 1),
    (2, 4096, 1, 3), (1, 5001, 2, 2), (2, 8192, 1, 2), (1, 20000, 1, 2), (1, 70001, 1, 1), (65, 192, 7, 7), (9, 12, 31, 33),
    (11, 700, 28, 28),
]


@pytest.mark.parametrize("order", ("nchw", "nhwc"))
@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape, dtype, order):
    for offset in (0, 1):
        k = Case(*shape, dtype, order, offset)
        rng = np.random.default_rng(case_seed((shape, dtype, order)))
        gamma, beta = vectors(k.c, rng)
        x = k.tensor(rng.standard_normal((k.n * k.h * k.w, k.c)) * (0.5 + rng.random(k.c)) + rng.standard_normal(k.c))
        for relu in (False, True):
            got, mean, rstd = forward(k, x, gamma, beta, relu)
            check_forward(k, x, gamma, beta, relu, got, mean, rstd)
        # without statistics and vectors; in place
        plain, _, _ = forward(k, x, None, None, False, stats=False)
        check_forward(k, x, None, None, False, plain, None, None)
        only, _, _ = forward(k, x, gamma, None, False, stats=False)
        check_forward(k, x, gamma, None, False, only, None, None)
        copy = at_offset(x, offset)
        inplace, mean2, _ = forward(k, copy, gamma, beta, True, out=copy)
        assert torch.equal(inplace, got) and torch.equal(mean, mean2)


def gradient(k, dy, x, gamma, mean, rstd, parts=("dx", "dgamma", "dbeta"), dx=None, fill=255):
    dx = (k.empty() if dx is None else dx) if "dx" in parts else None
    dgamma, dbeta = (torch.full((k.c,), float("nan"), device="cuda") if p in parts else None for p in ("dgamma", "dbeta"))
    ws = torch.full((max(B.layernorm_bwd_workspace_bytes(k.wrap(x)), 256),), fill, dtype=torch.uint8, device="cuda")
    B.layernorm_bwd(k.wrap(dy), k.wrap(x), None if gamma is None else cuda(gamma), mean, rstd, None if dx is None else k.wrap(dx), dgamma, dbeta, ws)
    torch.cuda.synchronize()
    return dx, dgamma, dbeta


def check_gradient(k, dy, x, gamma, mean, rstd, dx, dgamma, dbeta):
    x, dy = k.rows(x), k.rows(dy)
    mean, rstd = (t.double().cpu().numpy()[:, None] for t in (mean, rstd))
    g = dy * (np.ones(k.c) if gamma is None else gamma.astype(np.float64))
    z = (x - mean) * rstd
    ref = rstd * (g - g.mean(1, keepdims=True) - z * (g * z).mean(1, keepdims=True))
    if dx is not None:
        # z is off by 2 U |z| + U |x| rstd; the sums by their chains
        dz = 3 * U * np.abs(z) + U * np.abs(x) * rstd
        sums = (chain(k.c) + 6) * U * (np.abs(g).mean(1, keepdims=True) + np.abs(z) * np.abs(g * z).mean(1, keepdims=True))
        through = np.abs(z) * (np.abs(g) * dz).mean(1, keepdims=True) + dz * np.abs(g * z).mean(1, keepdims=True)
        tol = rstd * (sums + through + 4 * U * np.abs(g)) + (4 * U + 1.01 * k.u) * np.abs(ref)
        assert note("dx", (np.abs(k.rows(dx) - ref) / (tol * (1 + k.u) + 1e-30)).max(), 1.0)
    # a lane adds at most every 256th pixel, and at least 16 of them
    pixels = 32 + x.shape[0] / 256 + 16
    if dgamma is not None:
        tol = pixels * U * np.abs(dy * z).sum(0) + (np.abs(dy) * (3 * U * np.abs(z) + U * np.abs(x) * rstd)).sum(0)
        assert note("dgamma", (np.abs(dgamma.double().cpu().numpy() - (dy * z).sum(0)) / (tol + 1e-30)).max(), 1.0)
    if dbeta is not None:
        assert note("dbeta", (np.abs(dbeta.double().cpu().numpy() - dy.sum(0)) / (pixels * U * np.abs(dy).sum(0) + 1e-30)).max(), 1.0)


@pytest.mark.parametrize("order", ("nchw", "nhwc"))
@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("shape", SHAPES)
def test_gradient(shape, dtype, order):
    for offset in (0, 1):
        k = Case(*shape, dtype, order, offset)
        rng = np.random.default_rng(case_seed((shape, dtype, order), 1))
        gamma, _ = vectors(k.c, rng)
        pixels = k.n * k.h * k.w
        x = k.tensor(rng.standard_normal((pixels, k.c)) * (0.5 + rng.random(k.c)) + rng.standard_normal(k.c))
        dy = k.tensor(rng.standard_normal((pixels, k.c)) * (rng.random((pixels, k.c)) < 0.6))
        mean, rstd = (cuda(v) for v in statistics(k.rows(x)))
        dx, dgamma, dbeta = gradient(k, dy, x, gamma, mean, rstd)
        check_gradient(k, dy, x, gamma, mean, rstd, dx, dgamma, dbeta)
        # the same bits again, whatever the scratch held; in place; each part alone
        again = gradient(k, dy, x, gamma, mean, rstd, fill=0)
        assert all(torch.equal(a, b) for a, b in zip((dx, dgamma, dbeta), again))
        copy = at_offset(dy, offset)
        inplace = gradient(k, copy, x, gamma, mean, rstd, dx=copy)
        assert all(torch.equal(a, b) for a, b in zip((dx, dgamma, dbeta), inplace))
        for part, whole in (("dx", dx), ("dgamma", dgamma), ("dbeta", dbeta)):
            one = next(t for t in gradient(k, dy, x, gamma, mean, rstd, parts=(part,)) if t is not None)
            if part == "dx":
                check_gradient(k, dy, x, gamma, mean, rstd, one, None, None)
            else:
                assert torch.equal(one, whole)
        plain = gradient(k, dy, x, None, mean, rstd)
        check_gradient(k, dy, x, None, mean, rstd, *plain)


@pytest.mark.parametrize("order", ("nchw", "nhwc"))
def test_gradient_against_differences(order):
    """L = sum of t y(x, gamma, beta): central differences of L in 64 bits."""
    k = Case(2, 5, 2, 3, "f32", order)
    rng = np.random.default_rng(4)
    gamma, beta = vectors(k.c, rng)
    x64, t = rng.standard_normal((12, 5)).astype(np.float32).astype(np.float64), rng.standard_normal((12, 5)).astype(np.float32).astype(np.float64)

    def loss(x, g, b):
        mean, rstd = statistics(x)
        return (t * ((x - mean[:, None]) * rstd[:, None] * g + b)).sum()

    def difference(at):
        args = [x64.copy(), gamma.astype(np.float64), beta.astype(np.float64)]
        out, h = np.empty_like(args[at]), 1e-5
        for i in np.ndindex(out.shape):
            v = args[at][i]
            args[at][i] = v + h
            up = loss(*args)
            args[at][i] = v - h
            out[i] = (up - loss(*args)) / (2 * h)
            args[at][i] = v
        return out

    x, dy = k.tensor(x64), k.tensor(t)
    _, mean, rstd = forward(k, x, gamma, beta, False)
    dx, dgamma, dbeta = gradient(k, dy, x, gamma, mean, rstd)
    # differences: h^2 of the third derivative (of order 100 with rows as close as these) and 64-bit rounding over h; the kernel: 2^-24 a few times
    for got, at in ((k.rows(dx), 0), (dgamma.double().cpu().numpy(), 1), (dbeta.double().cpu().numpy(), 2)):
        ref = difference(at)
        assert note("difference", np.abs(got - ref).max() / np.abs(ref).max(), 1e-5)


@pytest.mark.parametrize("order", ("nchw", "nhwc"))
@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("c", (3, 64, 192, 509, 3000))
def test_rows_that_are_hard(dtype, order, c):
    """Equal values (no variance), values far from zero, the largest values, infinities and NaN: each pixel has its own result and touches no other."""
    k = Case(1, c, 4, 40, dtype, order)
    rng = np.random.default_rng(c)
    rows = rng.standard_normal((160, c)).astype(np.float32)
    rows[0] = 3.25
    rows[1] = 0
    rows[2] += 1024
    rows[3] *= 2.0 ** -60
    rows[5] *= 2.0 ** 60
    wild = rows.copy()
    wild[20, c // 2] = np.inf
    wild[21, 0] = -np.inf
    wild[22, c - 1] = np.nan
    gamma, beta = vectors(c, rng)
    x = k.tensor(rows)
    got, mean, rstd = forward(k, x, gamma, beta, False)
    keep = [i for i in range(160) if i not in (20, 21, 22)]
    # the pixel of equal values is beta, exactly
    b = torch.from_numpy(beta).to(k.dtype).double().numpy()
    assert np.array_equal(k.rows(got)[0], b) and np.array_equal(k.rows(got)[1], b)
    check_forward(k, x, gamma, beta, False, got, mean, rstd)
    got2, mean2, rstd2 = forward(k, k.tensor(wild), gamma, beta, False)
    assert np.array_equal(k.rows(got2)[keep], k.rows(got)[keep]) and torch.equal(mean2[keep], mean[keep]) and torch.equal(rstd2[keep], rstd[keep])
    assert np.isnan(k.rows(got2)[20:23]).any(1).all()
    dy = k.tensor(rng.standard_normal((160, c)))
    wild_dy = k.rows(dy)
    wild_dy[30, 0] = np.inf
    a, b = gradient(k, dy, x, gamma, mean, rstd), gradient(k, k.tensor(wild_dy), x, gamma, mean, rstd)
    keep = [i for i in range(160) if i != 30]
    assert np.array_equal(k.rows(a[0])[keep], k.rows(b[0])[keep])
    assert torch.equal(a[1][1:], b[1][1:]) and torch.equal(a[2][1:], b[2][1:]) and not torch.isfinite(b[2][0])


@pytest.mark.parametrize("n,c,hw,dtype,order", ((1, 1030, (2 ** 20 + 3, 1), "f32", "nhwc"), (1, 1030, (2 ** 20 + 5, 1), "bf16", "nhwc"), (2, 8192, (301, 300), "f32", "nchw"), (6000, 192, (31, 31), "f32", "nchw")))
def test_offsets_beyond_32_bits(n, c, hw, dtype, order):
    """More than 4 GiB (2 GiB in bf16), and planes whose 64 pixels reach that far: pixels from all over against the formulas, dgamma and dbeta against sums in 64 bits on the GPU."""
    k = Case(n, c, *hw, dtype, order)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.empty(k.shape, dtype=k.dtype, device="cuda").normal_(generator=gen) for _ in range(2))
    rng = np.random.default_rng(5)
    gamma, beta = vectors(c, rng)
    pixels = n * hw[0] * hw[1]
    at = torch.from_numpy(np.unique(np.concatenate([[0, 1, pixels - 2, pixels - 1], rng.integers(0, pixels, 400)]))).cuda()
    some = Case(len(at), c, 1, 1, dtype, "nhwc")

    def chosen(t):
        t = t.view(pixels, c)[at] if order == "nhwc" else t.view(n, c, -1)[at // (hw[0] * hw[1]), :, at % (hw[0] * hw[1])]
        return t.view(some.shape)

    y, mean, rstd = forward(k, x, gamma, beta, True)
    check_forward(some, chosen(x), gamma, beta, True, chosen(y), mean[at], rstd[at])
    del y
    dx, dgamma, dbeta = gradient(k, dy, x, gamma, mean, rstd)
    check_gradient(some, chosen(dy), chosen(x), gamma, mean[at], rstd[at], chosen(dx), None, None)
    del dx
    refs, mags = torch.zeros((2, c), dtype=torch.float64, device="cuda"), torch.zeros((3, c), dtype=torch.float64, device="cuda")
    flat = [t.view(1, pixels, c) if order == "nhwc" else t.view(n, c, -1) for t in (x, dy)]
    stats = [t.double().view(n, -1) for t in (mean, rstd)]
    step = 2 ** 15 if order == "nhwc" else 2 ** 13
    for i in range(flat[0].shape[0]):
        length = pixels // flat[0].shape[0]
        for p in range(0, length, step):
            if order == "nhwc":
                a, b = (t[0, p:p + step].double() for t in flat)
            else:
                a, b = (t[i, :, p:p + step].t().double() for t in flat)
            m, r = (t[i, p:p + step, None] for t in stats)
            z = (a - m) * r
            refs += torch.stack(((b * z).sum(0), b.sum(0)))
            mags += torch.stack(((b * z).abs().sum(0), b.abs().sum(0), (b.abs() * (3 * U * z.abs() + U * a.abs() * r)).sum(0)))
    chains = 32 + pixels / 256 + 16
    assert note("dgamma", ((dgamma.double() - refs[0]).abs() / (chains * U * mags[0] + mags[2])).max().item(), 1.0)
    assert note("dbeta", ((dbeta.double() - refs[1]).abs() / (chains * U * mags[1])).max().item(), 1.0)


def test_tensors_without_elements():
    for shape in ((0, 8, 3, 3), (2, 8, 0, 3), (0, 8, 1, 1)):
        for k in (Case(*shape, "f32", "nchw"), Case(*shape, "bf16", "nhwc")):
            x = torch.empty(k.shape, dtype=k.dtype, device="cuda")
            none = torch.empty(0, device="cuda")
            B.layernorm_fwd(k.wrap(x), None, None, EPS, False, k.wrap(x.clone()), none, none)
            _, dgamma, dbeta = gradient(k, x, x, None, none, none)
            assert not dgamma.any() and not dbeta.any()


@pytest.mark.parametrize("order,dtype,c", (("nchw", "f32", 192), ("nhwc", "bf16", 192), ("nhwc", "f32", 509)))
def test_recorded_and_on_another_stream(order, dtype, c):
    """A recorded forward and gradient, replayed with other inputs and the program's own work between, give the eager result."""
    k = Case(3, c, 9, 11, dtype, order)
    rng = np.random.default_rng(2)
    gamma, beta = (cuda(v) for v in vectors(c, rng))
    x, dy = (k.tensor(rng.standard_normal((297, c))) for _ in range(2))
    y, dx = k.empty(), k.empty()
    mean, rstd = torch.empty(297, device="cuda"), torch.empty(297, device="cuda")
    dgamma, dbeta = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    ws = torch.empty(max(B.layernorm_bwd_workspace_bytes(k.wrap(x)), 256), dtype=torch.uint8, device="cuda")

    def both(stream):
        B.layernorm_fwd(k.wrap(x), gamma, beta, EPS, True, k.wrap(y), mean, rstd, stream=stream)
        B.layernorm_bwd(k.wrap(dy), k.wrap(x), gamma, mean, rstd, k.wrap(dx), dgamma, dbeta, ws, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with B.capture(side, keep=(x, dy, y, dx, mean, rstd, dgamma, dbeta, ws, gamma, beta)) as rec:
        both(side)
    for turn in range(3):
        x.copy_(k.tensor(rng.standard_normal((297, c))))
        dy.copy_(k.tensor(rng.standard_normal((297, c))))
        side.wait_stream(torch.cuda.current_stream())
        both(side)
        side.synchronize()
        eager = [t.clone() for t in (y, dx, mean, rstd, dgamma, dbeta)]
        for t in (y, dx, mean, rstd, dgamma, dbeta):
            t.fill_(float("nan"))
        rec.graph.launch()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, (y, dx, mean, rstd, dgamma, dbeta)))
