"""Layer normalisation and its gradient in every kernel that the rules of csrc/layernorm.hip pick from the number of channels and pixels, each with more pixels than one turn of its
workgroups takes where it walks them, against the formulas in 64 bits on the GPU.

Tolerances are bounds, as in tests/test_gpu_layernorm.py: (additions on a sum's longest chain) x 2^-24 x (sum of the terms' magnitudes), and half a unit in the last place of a bf16
result, 2^-8 of it."""
import pytest

from paper_1708_04728_amd import binding as B
from util import case_seed, note

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24
EPS = 1e-5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
VECTOR = {"f32": 4, "bf16": 8}          # elements of 16 bytes


def near(got, ref, tol):
    """Largest ratio of |got - ref| to its bound."""
    return ((got.double() - ref).abs() / (tol + 1e-30)).max().item()


def compare(n, c, h, w, dtype, order, offset=0, relu=True):
    gen = torch.Generator(device="cuda").manual_seed(case_seed((n, c, h, w, dtype, order)))
    randn = lambda *s: torch.randn(s, device="cuda", generator=gen)
    u = 2.0 ** -8 if dtype == "bf16" else U

    def tensor(rows):               # (pixels, c) -> a tensor `offset` elements behind an allocation's start
        t = rows.view(n, h, w, c)
        t = (t.permute(0, 3, 1, 2) if order == "nchw" else t).to(DTYPES[dtype])
        out = torch.empty(t.numel() + offset, dtype=t.dtype, device="cuda")[offset:].view(t.shape)
        out.copy_(t)
        return out

    def rows(t):                    # ... and back, in 64 bits
        return (t.permute(0, 2, 3, 1) if order == "nchw" else t).reshape(-1, c).double()

    pixels = n * h * w
    wrap = B.NHWC if order == "nhwc" else lambda t: t
    x, dy = tensor(randn(pixels, c) * (0.5 + randn(c).abs()) + randn(c)), tensor(randn(pixels, c) * (randn(pixels, c) > -0.3))
    gamma, beta = 1 + 0.2 * randn(c), 0.3 * randn(c)
    nan = lambda t: torch.full_like(t, float("nan"))
    y, mean, rstd = nan(x), *(torch.full((pixels,), float("nan"), device="cuda") for _ in range(2))
    B.layernorm_fwd(wrap(x), gamma, beta, EPS, relu, wrap(y), mean, rstd)
    x64, d64, g64 = rows(x), rows(dy), gamma.double()
    mu = x64.mean(1, keepdim=True)
    r = 1 / ((x64 - mu).square().mean(1, keepdim=True) + EPS).sqrt()
    ref = (x64 - mu) * r * g64 + beta.double()
    ref = ref.clamp(min=0) if relu else ref
    chain, most = 96 + c / 256, x64.abs().amax(1, keepdim=True)
    d_mean = (chain + 2) * U * most
    d_rstd = (chain + 8) * U + (d_mean * r).clamp(max=1).square() + 2 * U * most * r
    tol = (d_mean * r + (x64 - mu).abs() * r * (d_rstd + 4 * U)) * g64.abs() + 4 * U * (beta.double().abs() + ref.abs()) + 1.01 * u * ref.abs()
    assert note("y", near(rows(y), ref, tol * (1 + u)), 1.0)
    assert note("mean", near(mean, mu[:, 0], d_mean[:, 0]), 1.0)
    assert note("rstd", near(rstd.double() / r[:, 0], torch.ones_like(r[:, 0]), d_rstd[:, 0]), 1.0)
    del ref, tol, y
    # the gradient, from the statistics that the forward pass left
    dx, dgamma, dbeta = nan(x), torch.full((c,), float("nan"), device="cuda"), torch.full((c,), float("nan"), device="cuda")
    ws = torch.full((max(B.layernorm_bwd_workspace_bytes(wrap(x)), 256),), 255, dtype=torch.uint8, device="cuda")
    B.layernorm_bwd(wrap(dy), wrap(x), gamma, mean, rstd, wrap(dx), dgamma, dbeta, ws)
    mu, r = mean.double()[:, None], rstd.double()[:, None]
    z = (x64 - mu) * r
    dz = 3 * U * z.abs() + U * x64.abs() * r
    chains = 32 + pixels / 256 + 16
    assert note("dgamma", near(dgamma, (d64 * z).sum(0), chains * U * (d64 * z).abs().sum(0) + (d64.abs() * dz).sum(0)), 1.0)
    assert note("dbeta", near(dbeta, d64.sum(0), chains * U * d64.abs().sum(0)), 1.0)
    g = d64 * g64
    ref = r * (g - g.mean(1, keepdim=True) - z * (g * z).mean(1, keepdim=True))
    sums = (chain + 6) * U * (g.abs().mean(1, keepdim=True) + z.abs() * (g * z).abs().mean(1, keepdim=True))
    through = z.abs() * (g.abs() * dz).mean(1, keepdim=True) + dz * (g * z).abs().mean(1, keepdim=True)
    tol = r * (sums + through + 4 * U * g.abs()) + (4 * U + 1.01 * u) * ref.abs()
    assert note("dx", near(rows(dx), ref, tol * (1 + u)), 1.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("ragged", (0, 3))
@pytest.mark.parametrize("vectors", (1, 2, 3, 4))
@pytest.mark.parametrize("lanes", (4, 8, 16, 32, 64))
def test_rows_in_groups_of_lanes(lanes, vectors, ragged, dtype):
    """`lanes` lanes a row, `vectors` 16-byte vectors each: as many rows as leave it at that, a wave for each of 256 compute units."""
    c = lanes * vectors * VECTOR[dtype] - ragged
    compare(1, c, 16384 // lanes + 5, 1, dtype, "nhwc", offset=1 if ragged else 0)


@pytest.mark.parametrize("rows,c,dtype", ((300000, 61, "f32"), (300000, 64, "f32"), (300000, 125, "bf16"), (70000, 192, "bf16"), (70000, 333, "f32"), (12000, 1021, "bf16"), (600, 8192, "f32"),
                                          (600, 16381, "f32"), (600, 4093, "f32"), (3000, 2045, "f32"), (600, 32765, "bf16"), (600, 8192, "bf16"), (600, 16376, "bf16"), (3000, 4091, "bf16"),
                                          (1100001, 3, "f32"), (1100001, 7, "bf16"), (1100001, 1, "f32"), (20000, 4100, "bf16")))
def test_more_rows_than_one_turn(rows, c, dtype):
    compare(rows, c, 1, 1, dtype, "nhwc", offset=1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("offset", (0, 1))
@pytest.mark.parametrize("n,h,w", ((11, 28, 28), (170, 7, 7), (1, 91, 91), (4200, 1, 2), (2, 28, 28)))
@pytest.mark.parametrize("c", (5, 40, 64, 65, 200, 256, 257, 400, 512, 700, 1024, 1100, 2100))
def test_planes(c, n, h, w, offset, dtype):
    """64 pixels a workgroup from 8192 pixels on, 16 below that and for some numbers of channels; 8, 16 or 32 channels in a lane's registers, or more than those hold; images of
    fewer pixels than a workgroup takes."""
    compare(n, c, h, w, dtype, "nchw", offset)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,c,h,w", ((90, 60, 28, 28), (100, 200, 28, 28), (90, 400, 28, 28), (1500, 300, 7, 7), (45, 700, 28, 28), (30, 1100, 28, 28), (400, 1100, 7, 7)))
def test_more_planes_than_one_turn(n, c, h, w, dtype):
    compare(n, c, h, w, dtype, "nchw", 1)
