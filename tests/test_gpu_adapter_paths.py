"""Every kernel that the adapters' rules pick, in both directions, against the formulas in 64 bits on the device: tiles of 64 x 64 fed straight into LDS (stages four deep: more than four
of them, and a last one that is no whole one), images longer than a tile, as they come; and sums over rows whose workgroups take more than 256 rows.

A sum of n products accumulated in fp32 in any order is off by at most 2 (n + 4) 2^-24 times the sum of the products' magnitudes; inner and u, held in fp32, carry that of their own sums; the result
is rounded to its type."""
import pytest

import adapt_oracle as O
from paper_1708_04728_amd import binding as B
from util import case_seed, note

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24


def chain(n):
    return 2 * (n + 4) * U


def compare(n, h, w, cin, cout, rank, count, p, dtype):
    dt, ut = (torch.bfloat16, 2.0 ** -8) if dtype == "bf16" else (torch.float32, U)
    gen = torch.Generator(device="cuda").manual_seed(case_seed((n, h, w, cin, cout, rank, count, p, dtype)))
    num = lambda *s: torch.randn(s, device="cuda", generator=gen).to(dt)
    rows = n * h * w
    x, wt, a, b, dy, bias = num(n, h, w, cin), num(cout, cin), num(count, rank, cin), num(count, cout, rank), num(n, h, w, cout), torch.randn(cout, device="cuda", generator=gen)
    scales = 0.5 + torch.rand(count, device="cuda", generator=gen)
    ids = torch.randint(-1, count, (n,), device="cuda", generator=gen, dtype=torch.int32)
    drop = B.dropout_desc(p, 77, 3) if p else None
    nan = float("nan")
    y, dx, inner = torch.full_like(dy, nan), torch.full_like(x, nan), torch.full((n, h, w, rank), nan, device="cuda")
    da, db = torch.full(a.shape, nan, device="cuda"), torch.full(b.shape, nan, device="cuda")
    N = B.NHWC
    ws = torch.full((max(B.adapter_fwd_workspace_bytes(N(x), a, b), B.adapter_bwd_workspace_bytes(N(x), a, b)),), 255, dtype=torch.uint8, device="cuda")
    B.adapter_fwd(N(x), wt, bias, a, b, ids, N(y), ws, scales=scales, drop=drop, inner=inner)
    B.adapter_bwd(N(dy), N(x), wt, a, b, ids, inner, N(dx), da, db, ws, scales=scales, drop=drop)
    only = torch.full_like(dx, nan)
    B.adapter_bwd(N(dy), N(x), wt, a, b, ids, None, N(only), None, None, ws, scales=scales, drop=drop)      # the mask drawn in the product itself
    assert torch.equal(only, dx)

    def check(what, got, ref, tol):
        got = got.double().view(ref.shape)
        assert torch.isfinite(got).all(), what
        assert note(what + " / bound", ((got - ref).abs() / (tol + 1e-37)).max().item(), 1.0)

    xd, dyd, wd = x.double().view(rows, cin), dy.double().view(rows, cout), wt.double()
    m = torch.from_numpy(O.mask((rows, cin), p, 77, 3)).cuda() if p else torch.ones((1, cin), dtype=torch.float64, device="cuda").expand(rows, cin)
    of = ids.repeat_interleave(h * w)
    y_ref, y_size = xd @ wd.t() + bias.double(), xd.abs() @ wd.abs().t() + bias.double().abs()
    dx_ref, dx_size = dyd @ wd, dyd.abs() @ wd.abs()
    y_off, dx_off = torch.zeros_like(y_ref), torch.zeros_like(dx_ref)
    t_ref, t_size = torch.zeros((rows, rank), dtype=torch.float64, device="cuda"), torch.zeros((rows, rank), dtype=torch.float64, device="cuda")
    for k in range(count):
        i = (of == k).nonzero().view(-1)
        ad, bd, s, dropped = a[k].double(), b[k].double(), scales[k].double(), xd[i] * m[i]
        t, st = s * (dropped @ ad.t()), s * (dropped.abs() @ ad.abs().t())
        u, su = s * (dyd[i] @ bd), s * (dyd[i].abs() @ bd.abs())
        t_ref[i], t_size[i] = t, st
        y_ref[i] += t @ bd.t()
        y_size[i] += st @ bd.abs().t()
        y_off[i] = (chain(cin) + 4 * U) * (st @ bd.abs().t())
        through = m[i] * (su @ ad.abs())
        dx_ref[i] += m[i] * (u @ ad)
        dx_size[i] += through
        dx_off[i] = (chain(cout) + 4 * U) * through
        # (join's sums add chunks to what a chunk's rows are: no more additions in all than there are rows)
        check("da", da[k], u.t() @ dropped, (chain(len(i)) + chain(cout) + 6 * U) * (su.t() @ dropped.abs()))
        check("db", db[k], dyd[i].t() @ t, (chain(len(i)) + chain(cin) + 6 * U) * (dyd[i].abs().t() @ st))
    check("inner", inner, t_ref, (chain(cin) + 4 * U) * t_size)
    check("y", y, y_ref, chain(cin + rank) * y_size + y_off + ut * y_ref.abs())
    check("dx", dx, dx_ref, chain(cout + rank) * dx_size + dx_off + ut * dx_ref.abs())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,h,w,cin,cout,rank,count,p", [
    (1100, 1, 1, 456, 520, 12, 3, 0.1),          # 64 x 64 in both directions, rows of whole 16-byte pieces
    (1100, 1, 1, 456, 520, 33, 2, 0.0),
    (19, 15, 13, 528, 256, 12, 5, 0.0),          # maps, as they come
    (19, 15, 13, 528, 256, 5, 5, 0.4),
    (300, 2, 2, 456, 520, 16, 40, 0.1),          # many adapters to a tile
    (1100, 1, 1, 453, 519, 12, 3, 0.1)])         # rows that are not
def test_tiles_of_64(n, h, w, cin, cout, rank, count, p, dtype):
    compare(n, h, w, cin, cout, rank, count, p, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,h,w,cin,cout,rank,count,p", [
    (2052, 1, 1, 1032, 1160, 16, 3, 0.1),        # 128 x 128
    (2100, 1, 1, 1036, 1160, 70, 2, 0.4),        # c_in no multiple of eight: the mask drawn in the product beside da too
    (11, 15, 13, 1032, 1160, 8, 4, 0.1)])
def test_tiles_of_128(n, h, w, cin, cout, rank, count, p, dtype):
    compare(n, h, w, cin, cout, rank, count, p, dtype)


@pytest.mark.parametrize("n,h,w,cin,cout,rank,count,p,dtype", [
    (16384 + 37, 1, 1, 264, 7900, 16, 2, 0.1, "bf16"),       # 33 blocks of columns: 31 chunks of 544 rows, windows of 256, 256 and 32
    (15872, 1, 1, 264, 7900, 40, 3, 0.0, "bf16"),            # of 512
    (16384 + 37, 1, 1, 136, 3900, 16, 2, 0.1, "f32"),
    (85, 15, 13, 264, 7900, 16, 3, 0.1, "bf16")])            # maps
def test_sums_over_many_rows(n, h, w, cin, cout, rank, count, p, dtype):
    compare(n, h, w, cin, cout, rank, count, p, dtype)


def whole(n, h, w, cin, cout, rank, count, p, dtype):
    """Every input -1, 0 or 1 (p 0 or 1/2: what is kept counts twice): all sums are whole numbers below 2^24, so every output is the formula's, rounded once to its type."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(case_seed((n, h, w, cin, cout, rank, count, p, dtype), 1))
    num = lambda *s: torch.randint(-1, 2, s, device="cuda", generator=gen).to(dt)
    rows = n * h * w
    x, wt, a, b, dy = num(n, h, w, cin), num(cout, cin), num(count, rank, cin), num(count, cout, rank), num(n, h, w, cout)
    ids = torch.randint(-1, count, (n,), device="cuda", generator=gen, dtype=torch.int32)
    drop = B.dropout_desc(p, 78, 4) if p else None
    nan = float("nan")
    y, dx, inner = torch.full_like(dy, nan), torch.full_like(x, nan), torch.full((n, h, w, rank), nan, device="cuda")
    da, db = torch.full(a.shape, nan, device="cuda"), torch.full(b.shape, nan, device="cuda")
    N = B.NHWC
    ws = torch.full((max(B.adapter_fwd_workspace_bytes(N(x), a, b), B.adapter_bwd_workspace_bytes(N(x), a, b)),), 255, dtype=torch.uint8, device="cuda")
    B.adapter_fwd(N(x), wt, None, a, b, ids, N(y), ws, drop=drop, inner=inner)
    B.adapter_bwd(N(dy), N(x), wt, a, b, ids, inner, N(dx), da, db, ws, drop=drop)
    xd, dyd, wd = x.double().view(rows, cin), dy.double().view(rows, cout), wt.double()
    m = torch.from_numpy(O.mask((rows, cin), p, 78, 4)).cuda() if p else torch.ones((1, cin), dtype=torch.float64, device="cuda").expand(rows, cin)
    of = ids.repeat_interleave(h * w)
    y_ref, dx_ref, t_ref = xd @ wd.t(), dyd @ wd, torch.zeros((rows, rank), dtype=torch.float64, device="cuda")
    for k in range(count):
        i = (of == k).nonzero().view(-1)
        ad, bd, dropped = a[k].double(), b[k].double(), xd[i] * m[i]
        t, u = dropped @ ad.t(), dyd[i] @ bd
        t_ref[i] = t
        y_ref[i] += t @ bd.t()
        dx_ref[i] += m[i] * (u @ ad)
        assert torch.equal(da[k].double(), u.t() @ dropped) and torch.equal(db[k].double(), dyd[i].t() @ t)
    assert max(t.abs().max().item() for t in (y_ref, dx_ref, t_ref, da.double(), db.double())) < 2 ** 24
    assert torch.equal(inner.view(rows, rank).double(), t_ref)
    assert torch.equal(y.view(rows, cout), y_ref.float().to(dt)) and torch.equal(dx.view(rows, cin), dx_ref.float().to(dt))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("p", [0.0, 0.5])
@pytest.mark.parametrize("n,h,w,cin,cout,rank,count", [
    (5, 1, 1, 1000, 1024, 8, 2), (64, 1, 1, 520, 456, 16, 64), (300, 1, 1, 40, 24, 100, 150),                                     # few rows, many adapters
    (1100, 1, 1, 456, 520, 12, 3), (19, 15, 13, 528, 256, 12, 5), (1100, 1, 1, 453, 519, 33, 3),                                  # tiles of 64
    (2052, 1, 1, 1032, 1160, 16, 3), (2100, 1, 1, 1036, 1160, 70, 2), (4100, 1, 1, 4104, 4112, 17, 5), (4100, 1, 1, 4099, 4101, 5, 2),      # of 128 and of 256
    (16384 + 37, 1, 1, 264, 7900, 16, 2), (15872, 1, 1, 264, 7900, 40, 3), (16384 + 37, 1, 1, 136, 3900, 16, 2), (85, 15, 13, 264, 7900, 16, 3)])      # sums over many rows
def test_whole_numbers(n, h, w, cin, cout, rank, count, p, dtype):
    whole(n, h, w, cin, cout, rank, count, p, dtype)
