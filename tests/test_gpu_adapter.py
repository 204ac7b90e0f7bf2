"""Adapters beside a shared projection, and their gradient, on the GPU against the formulas in 64 bits.

A sum of n products accumulated in fp32 in any order is off by at most 2 n 2^-24 times the sum of the products' magnitudes (the matrix unit may cut where others round: 2^-23
for each addition); products of two bf16 numbers are exact in fp32, those of two fp32 numbers add 2^-24 each, inside the factor 2 for n >= 2 (n + 4 is taken for n).  inner and
u are held in fp32 and enter bf16 products as two pieces, which keep them to 2^-17.  The result is rounded to its type: 2^-8 of its size in bf16, 2^-24 in fp32."""
import numpy as np
import pytest

import adapt_oracle as O
from paper_1708_04728_amd import binding as B
from util import case_seed, note

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24


def chain(n):
    return 2 * (n + 4) * U


class Case:
    def __init__(self, n, h, w, cin, cout, rank, count, dtype, p=0.0, ids=None, offset=0, scales=True):
        rng = np.random.default_rng(case_seed((n, h, w, cin, cout, rank, count, dtype, p, offset)))
        self.n, self.h, self.w, self.cin, self.cout, self.rank, self.count, self.p, self.offset = n, h, w, cin, cout, rank, count, p, offset
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.ut = 2.0 ** -8 if dtype == "bf16" else U
        pieces = 2.0 ** -17 if dtype == "bf16" else 0.0
        self.pieces = pieces
        num = lambda *s: torch.from_numpy(rng.standard_normal(s)).to(self.dtype)
        self.x, self.wt, self.a, self.b = num(n, h, w, cin), num(cout, cin), num(count, rank, cin), num(count, cout, rank)
        self.dy, self.bias = num(n, h, w, cout), torch.from_numpy(rng.standard_normal(cout)).float()
        self.scales = torch.from_numpy(rng.uniform(0.5, 2, count)).float() if scales else None
        self.ids = np.array(rng.integers(-1, count + 1, n) if ids is None else ids)       # some of none: -1 and `count`
        self.seed, self.place = 0xABCDEF0123456789, 3 * 2 ** 32 + n

    def wide(self, t):
        return t.double().numpy().reshape(-1, t.shape[-1])

    def dev(self, t):
        flat = torch.full((t.numel() + self.offset + 16,), float("nan"), dtype=t.dtype, device="cuda")
        out = flat[self.offset:self.offset + t.numel()].view(t.shape)
        out.copy_(t)
        return out

    def wrap(self, t):
        return B.NHWC(t)

    def gpu(self):
        f = self
        f.gx, f.gw, f.ga, f.gb, f.gdy, f.gbias = (f.dev(t) for t in (f.x, f.wt, f.a, f.b, f.dy, f.bias))
        f.gscales = None if f.scales is None else f.dev(f.scales)
        f.gids = torch.from_numpy(f.ids.astype(np.int32)).cuda()
        f.drop = B.dropout_desc(f.p, f.seed, f.place) if f.p else None
        f.y = f.dev(torch.full((f.n, f.h, f.w, f.cout), float("nan"), dtype=f.dtype))
        f.dx = f.dev(torch.full((f.n, f.h, f.w, f.cin), float("nan"), dtype=f.dtype))
        f.inner = torch.full((f.n, f.h, f.w, f.rank), float("nan"), device="cuda")
        f.da, f.db = (torch.full(t.shape, float("nan"), device="cuda") for t in (f.a, f.b))
        need = max(B.adapter_fwd_workspace_bytes(B.NHWC(f.gx), f.ga, f.gb), B.adapter_bwd_workspace_bytes(B.NHWC(f.gx), f.ga, f.gb), 256)
        f.ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        return f

    def forward(self, keep=True, stream=None, bias=True):
        f = self
        B.adapter_fwd(B.NHWC(f.gx), f.gw, f.gbias if bias else None, f.ga, f.gb, f.gids, B.NHWC(f.y), f.ws, scales=f.gscales, drop=f.drop, inner=f.inner if keep else None, stream=stream)

    def backward(self, dx=True, da=True, db=True, stream=None):
        f = self
        B.adapter_bwd(B.NHWC(f.gdy), B.NHWC(f.gx), f.gw, f.ga, f.gb, f.gids, f.inner if db else None, B.NHWC(f.dx) if dx else None, f.da if da else None, f.db if db else None,
                      f.ws, scales=f.gscales, drop=f.drop, stream=stream)

    def expect(self, bias=True):
        """What the formulas give, and bounds on how far off each may be."""
        f = self
        x, w, dy = f.wide(f.x), f.wt.double().numpy(), f.wide(f.dy)
        a, b = f.a.double().numpy(), f.b.double().numpy()
        bias = f.bias.double().numpy() if bias else None
        ids = np.repeat(f.ids, f.h * f.w)
        scales = np.ones(f.count) if f.scales is None else f.scales.double().numpy()
        m = O.mask(x.shape, f.p, f.seed, f.place)
        size = lambda *v: [np.abs(t) for t in v]
        y, inner = O.adapter_fwd(x, w, bias, a, b, ids, scales, m)
        ax, aw, aa, ab, ady = size(x, w, a, b, dy)
        sy, sinner = O.adapter_fwd(ax, aw, None if bias is None else np.abs(bias), aa, ab, ids, scales, m)
        inner_tol = (chain(f.cin) + 4 * U) * sinner
        through, _ = O.adapter_fwd(0 * ax, 0 * aw, None, aa, ab, ids, scales, m)
        lift = lambda t: O.adapter_bwd(0 * dy, x, 0 * w, a, b, ids, scales, m, t)
        by_b = np.zeros(y.shape)
        for i, k in enumerate(ids):
            if 0 <= k < f.count:
                by_b[i] = ab[k] @ (inner_tol[i] + f.pieces * np.abs(inner[i]))
        f.y_ref, f.y_tol = y, chain(f.cin + f.rank) * sy + by_b + f.ut * np.abs(y) + 1e-37
        f.inner_ref, f.inner_tol = inner, inner_tol + 1e-37
        dx, da, db = O.adapter_bwd(dy, x, w, a, b, ids, scales, m, inner)
        sdx, sda, sdb = O.adapter_bwd(ady, ax, aw, aa, ab, ids, scales, m, sinner)
        most = max([int((ids == k).sum()) for k in range(f.count)] + [1])
        # u's own error, (c_out chain and its pieces) of its magnitudes, reaches dx and dA multiplied as u is: part of their sums of magnitudes
        own = sdx - ady @ aw
        f.dx_ref, f.dx_tol = dx, chain(f.cout + f.rank) * sdx + (chain(f.cout) + 4 * U + f.pieces) * own + f.ut * np.abs(dx) + 1e-37
        f.da_ref, f.da_tol = da, (chain(most) + chain(f.cout) + 6 * U + f.pieces) * sda + 1e-37
        # inner as it was computed: off by inner_tol, inside chain(c_in) of its magnitudes
        f.db_ref, f.db_tol = db, (chain(most) + chain(f.cin) + 6 * U + f.pieces) * sdb + 1e-37
        return f

    def close(self, what, got, ref, tol):
        got = got.double().cpu().numpy().reshape(ref.shape)
        assert np.isfinite(got).all(), what
        assert note(what + " / bound", np.max(np.abs(got - ref) / tol, initial=0.0), 1.0)

    def check(self, forward=True, backward=True):
        f = self
        if forward:
            f.close("y", f.y, f.y_ref, f.y_tol)
            f.close("inner", f.inner, f.inner_ref, f.inner_tol)
        if backward:
            f.close("dx", f.dx, f.dx_ref, f.dx_tol)
            f.close("da", f.da, f.da_ref, f.da_tol)
            f.close("db", f.db, f.db_ref, f.db_tol)


SHAPES = [  # n, h, w, c_in, c_out, rank, adapters, p
    (1, 1, 1, 1, 1, 1, 1, 0.0), (1, 1, 1, 1024, 1000, 8, 1, 0.0), (2, 1, 1, 40, 24, 3, 5, 0.4), (17, 1, 1, 33, 65, 16, 4, 0.1), (64, 1, 1, 512, 256, 16, 64, 0.0),
    (65, 1, 1, 100, 90, 12, 3, 0.4), (200, 1, 1, 257, 129, 17, 7, 0.5), (3, 15, 13, 48, 72, 5, 2, 0.1), (5, 7, 7, 832, 128, 24, 3, 0.0), (130, 3, 2, 64, 64, 32, 9, 0.4),
    (1, 9, 31, 31, 33, 40, 1, 0.9), (300, 1, 1, 96, 160, 64, 20, 0.1), (70, 2, 2, 72, 40, 100, 2, 0.4), (50, 1, 1, 130, 70, 128, 60, 0.0), (600, 1, 1, 136, 200, 8, 1, 0.1),
    (700, 1, 1, 64, 48, 4, 500, 0.1), (12, 1, 1, 2048, 33, 16, 2, 0.4), (300, 1, 1, 300, 520, 16, 2, 0.4)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,h,w,cin,cout,rank,count,p", SHAPES)
def test_against_the_formulas(n, h, w, cin, cout, rank, count, p, dtype):
    f = Case(n, h, w, cin, cout, rank, count, dtype, p).gpu().expect()
    f.forward()
    f.backward()
    f.check()


LARGE = [  # rows, c_in, c_out, rank, adapters, p: tiles of 128 and of 256 in both directions, aligned rows and others, a last stage that is no whole one
    (2048, 136, 2048, 16, 5, 0.1, "bf16"), (1500, 133, 1999, 20, 3, 0.4, "bf16"), (4096, 264, 4096, 16, 8, 0.1, "bf16"), (4100, 131, 4100, 5, 3, 0.0, "bf16"),
    (2000, 136, 2100, 16, 5, 0.4, "f32"), (4096, 72, 4096, 33, 4, 0.0, "f32"), (4097, 67, 4101, 8, 2, 0.4, "f32")]


@pytest.mark.parametrize("rows,cin,cout,rank,count,p,dtype", LARGE)
@pytest.mark.parametrize("turned", [False, True])
def test_large_tiles(rows, cin, cout, rank, count, p, dtype, turned):
    """y of a projection to many channels, and (turned) dx of one from many; the same formulas and bounds, in 64 bits on the device."""
    cin, cout = (cout, cin) if turned else (cin, cout)
    rng = np.random.default_rng(case_seed((rows, cin, cout, rank, count, p, dtype)))
    dt, ut = (torch.bfloat16, 2.0 ** -8) if dtype == "bf16" else (torch.float32, U)
    pieces = 2.0 ** -17 if dtype == "bf16" else 0.0
    num = lambda *s: torch.from_numpy(rng.standard_normal(s, dtype=np.float32)).to(dt).cuda()
    x, w, a, b, dy, bias = num(rows, cin), num(cout, cin), num(count, rank, cin), num(count, cout, rank), num(rows, cout), num(cout).float()
    ids = torch.from_numpy(rng.integers(-1, count, rows).astype(np.int32)).cuda()
    drop = B.dropout_desc(p, 77, 3) if p else None
    y, dx, inner = torch.empty_like(dy), torch.empty_like(x), torch.empty((rows, rank), device="cuda")
    da, db = torch.empty(a.shape, device="cuda"), torch.empty(b.shape, device="cuda")
    ws = torch.empty(max(B.adapter_fwd_workspace_bytes(x, a, b), B.adapter_bwd_workspace_bytes(x, a, b)), dtype=torch.uint8, device="cuda")
    B.adapter_fwd(x, w, bias, a, b, ids, y, ws, drop=drop, inner=inner)
    B.adapter_bwd(dy, x, w, a, b, ids, inner, dx, da, db, ws, drop=drop)
    only, _, _ = B.adapter_bwd(dy, x, w, a, b, ids, None, torch.empty_like(x), None, None, ws, drop=drop)      # the mask drawn in the product itself
    assert torch.equal(only, dx)
    m = torch.from_numpy(O.mask((rows, cin), p, 77, 3)).cuda()
    chosen = (ids[:, None] == torch.arange(count, device="cuda")).double()
    xd, wd, ad, bd, dyd = (t.double() for t in (x, w, a.view(-1, cin), b.permute(0, 2, 1).reshape(-1, cout), dy))
    own = chosen.repeat_interleave(rank, 1)
    def check(what, got, ref, tol):
        assert note(what + " / bound", ((got.double() - ref).abs() / tol).max().item(), 1.0)
    if not turned:
        t, st = own * ((xd * m) @ ad.t()), own * ((xd.abs() * m) @ ad.abs().t())
        ref = xd @ wd.t() + bias.double() + t @ bd
        off = (chain(cin) + 4 * U) * st + pieces * t.abs()
        check("y", y, ref, chain(cin + rank) * (xd.abs() @ wd.abs().t() + bias.double().abs() + st @ bd.abs()) + off @ bd.abs() + ut * ref.abs() + 1e-37)
    else:
        u, su = own * (dyd @ bd.t()), own * (dyd.abs() @ bd.abs().t())
        ref = dyd @ wd + m * (u @ ad)
        through = m * (su @ ad.abs())
        check("dx", dx, ref, chain(cout + rank) * (dyd.abs() @ wd.abs() + through) + (chain(cout) + 4 * U + pieces) * through + ut * ref.abs() + 1e-37)
        da_ref, s_da = u.t() @ (xd * m), su.t() @ (xd.abs() * m)
        most = int(chosen.sum(0).max().item())
        check("da", da.view(-1, cin), da_ref, (chain(most) + chain(cout) + 6 * U) * s_da + 1e-37)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [1, 3, 8])
def test_tensors_at_any_address(dtype, offset):
    f = Case(70, 1, 1, 64, 80, 8, 3, dtype, 0.4, offset=offset).gpu().expect()
    f.forward()
    f.backward()
    f.check()


@pytest.mark.parametrize("ids", [[-1] * 20, [0] * 20, [3] * 20, [-5, 2 ** 31 - 1, -2 ** 31, 4] * 5, list(range(4)) * 5, sorted(list(range(4)) * 5), [0] * 19 + [3]])
def test_who_has_which_adapter(ids):
    f = Case(20, 2, 3, 40, 56, 6, 4, "bf16", 0.1, ids=ids).gpu().expect()
    f.forward()
    f.backward()
    f.check()


def test_parts_of_a_call():
    f = Case(90, 1, 1, 72, 40, 8, 3, "bf16", scales=False).gpu().expect(bias=False)
    f.forward(keep=False, bias=False)
    f.close("y", f.y, f.y_ref, f.y_tol)
    f.forward(bias=False)
    f.backward(da=False, db=False)
    f.close("dx", f.dx, f.dx_ref, f.dx_tol)
    assert torch.isnan(f.da).all() and torch.isnan(f.db).all()
    f.dx.fill_(float("nan"))
    f.backward(dx=False, db=False)
    f.close("da", f.da, f.da_ref, f.da_tol)
    f.backward(dx=False, da=False)
    f.close("db", f.db, f.db_ref, f.db_tol)
    assert torch.isnan(f.dx).all()


def test_rows_as_a_matrix_and_no_rows():
    f = Case(30, 1, 1, 72, 40, 8, 3, "f32").gpu().expect()
    x, y, dy, dx = (t.view(30, -1) for t in (f.gx, f.y, f.gdy, f.dx))
    B.adapter_fwd(x, f.gw.view(40, 72, 1, 1), f.gbias, f.ga, f.gb, f.gids, y, f.ws, scales=f.gscales, inner=f.inner)
    B.adapter_bwd(dy, x, f.gw, f.ga, f.gb, f.gids, f.inner, dx, f.da, f.db, f.ws, scales=f.gscales)
    f.check()
    e = f.gx[:0].view(0, 72)
    f.da.fill_(5.0)
    B.adapter_fwd(e, f.gw, f.gbias, f.ga, f.gb, f.gids[:0], f.y[:0].view(0, 40), f.ws)
    B.adapter_bwd(f.gdy[:0].view(0, 40), e, f.gw, f.ga, f.gb, f.gids[:0], f.inner[:0], e, f.da, f.db, f.ws)
    assert (f.da == 0).all() and (f.db == 0).all()
    a, b = f.ga[:0], f.gb[:0]                                     # no adapters: the projection alone
    B.adapter_fwd(x, f.gw, f.gbias, a, b, f.gids, y, f.ws, inner=f.inner)
    ref = f.wide(f.x) @ f.wt.double().numpy().T + f.bias.double().numpy()
    assert np.abs(y.double().cpu().numpy() - ref).max() < chain(72) * 72 * 25 and (f.inner == 0).all()
    B.adapter_bwd(dy, x, f.gw, a, b, f.gids, f.inner, dx, f.da[:0], f.db[:0], f.ws)
    assert np.abs(dx.double().cpu().numpy() - f.wide(f.dy) @ f.wt.double().numpy()).max() < chain(40) * 40 * 25


@pytest.mark.parametrize("n", [5, 400])
def test_a_projection_without_adapters_asks_for_none(n):
    """count = 0 with A, B and ids NULL, by the C entry points."""
    import ctypes as C
    f = Case(n, 1, 1, 72, 136, 8, 0, "f32", ids=[-1] * n).gpu()
    xd, yd, ad = B.dr_tensor(n, 72, 1, 1, 0, 1), B.dr_tensor(n, 136, 1, 1, 0, 1), B.dr_adapters(0, 8, 72, 136)
    L, p, need, stream = B.lib(), B._ptr, C.c_size_t(0), torch.cuda.current_stream().cuda_stream
    for size in (L.dr_adapter_fwd_workspace_bytes, L.dr_adapter_bwd_workspace_bytes):
        assert size(xd, ad, need) == B.DR_OK and need.value <= f.ws.numel()
    assert L.dr_adapter_fwd(xd, p(f.gx), ad, p(f.gw), p(f.gbias), None, None, None, None, None, yd, p(f.y), p(f.inner), p(f.ws), f.ws.numel(), stream) == B.DR_OK
    assert L.dr_adapter_bwd(yd, p(f.gdy), xd, p(f.gx), ad, p(f.gw), None, None, None, None, None, None, p(f.dx), p(f.da), p(f.db), p(f.ws), f.ws.numel(), stream) == B.DR_OK
    w = f.wt.double().numpy()
    y, dx = f.wide(f.x) @ w.T + f.bias.double().numpy(), f.wide(f.dy) @ w
    f.close("y", f.y, y, chain(72) * (np.abs(f.wide(f.x)) @ np.abs(w).T + np.abs(f.bias.double().numpy())) + U * np.abs(y))
    f.close("dx", f.dx, dx, chain(136) * (np.abs(f.wide(f.dy)) @ np.abs(w)) + U * np.abs(dx))
    assert (f.inner == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [24, 300])
def test_one_request_does_not_reach_another(dtype, n):
    """An adapter, an input and a gradient that hold NaN and infinities: their own rows become NaN, no other bit changes."""
    clean = Case(n, 1, 1, 72, 136, 8, 4, dtype, 0.4).gpu()
    clean.forward()
    clean.backward()
    f = Case(n, 1, 1, 72, 136, 8, 4, dtype, 0.4).gpu()
    f.ga[1, 2, 5], f.gb[1, 7, 3], f.gb[1, 9, 1] = float("nan"), float("inf"), float("nan")
    odd = int(np.nonzero(f.ids == 2)[0][0])
    f.gx[odd] = float("inf")
    f.forward()
    hit = torch.from_numpy((f.ids == 1) | (np.arange(n) == odd)).cuda()
    assert torch.equal(f.y[~hit], clean.y[~hit]) and torch.equal(f.inner[~hit], clean.inner[~hit])
    assert not torch.isfinite(f.y[hit]).all()
    f.gx.copy_(clean.gx)
    f.gdy[odd, 0, 0, 3] = float("nan")
    f.inner.copy_(clean.inner)
    f.backward()
    assert torch.equal(f.dx[~hit], clean.dx[~hit])
    for k in (0, 3):
        assert torch.equal(f.da[k], clean.da[k]) and torch.equal(f.db[k], clean.db[k])
    assert torch.isnan(f.db[2][3]).all() and torch.isfinite(f.db[2][4]).all()


def test_the_same_bits_again():
    f = Case(500, 1, 1, 264, 136, 16, 5, "bf16", 0.1).gpu()
    f.forward()
    f.backward()
    first = [t.clone() for t in (f.y, f.inner, f.dx, f.da, f.db)]
    for _ in range(3):
        f.forward()
        f.backward()
        for a, b in zip(first, (f.y, f.inner, f.dx, f.da, f.db)):
            assert torch.equal(a, b)


def test_recorded_and_on_two_streams():
    """Two recorded graphs with a workspace each, replayed side by side on streams of their own while their inputs, ids and masks change."""
    cases = [Case(100, 1, 1, 136, 72, 8, 3, "bf16", 0.4).gpu(), Case(9, 5, 5, 64, 48, 4, 2, "f32", 0.1).gpu()]
    streams = [torch.cuda.Stream() for _ in cases]
    steps, graphs = [], []
    for f, s in zip(cases, streams):
        step = torch.zeros(1, dtype=torch.int64, device="cuda")
        f.drop = B.dropout_desc(f.p, f.seed, f.place, step)
        steps.append(step)
        s.wait_stream(torch.cuda.current_stream())
        with B.capture(s, (f, step)) as c:
            f.forward(stream=s)
            f.backward(stream=s)
        graphs.append(c.graph)
    for turn in range(3):
        for f, step in zip(cases, steps):
            step.fill_(turn)
            f.gx.mul_(1.25)
            f.gids.copy_(torch.roll(f.gids, 1))
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            g.launch(s)
        torch.cuda.synchronize()
        for f in cases:
            f.x = f.gx.cpu()
            f.ids = f.gids.cpu().numpy()
            place, f.place = f.place, f.place + turn
            f.expect().check()
            f.place = place
