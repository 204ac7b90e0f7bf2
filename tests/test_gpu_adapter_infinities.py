"""Infinities and the largest numbers in adapters, inputs, gradients and inner: the formula's answer (+-inf, NaN or a number) in every kernel, whatever a call's number of rows.

What is computed from numbers alone keeps the bounds of a sum of n products in fp32: 2 (n + 4) 2^-24 of the magnitudes, and the rounding of the result.  A number that lies within
those bounds of a type's largest is not asked for here."""
import pytest

import adapt_oracle as O
from paper_1708_04728_amd import binding as B
from util import case_seed, note

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24
INF = float("inf")
BEYOND = 1.5 * 2.0 ** 119      # added to bf16's largest, 2^128 - 2^120: a number of fp32 that bf16 rounds to infinity
SIZES = [(24, 72, 136), (1100, 72, 520), (2048, 72, 2048), (4096, 72, 4096), (4096, 77, 4099)]      # few rows; tiles of 64, of 128, of 256; rows that are not aligned
RANK, COUNT = 5, 4


def normal(shape, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, device="cuda", generator=gen).to(dtype)


def chain(n):
    return 2 * (n + 4) * U


def check(what, got, ref, size, n, dtype):
    """got against ref in 64 bits, of which +-inf, NaN and numbers beyond the type's largest have to be met; size: the sum of magnitudes of a number's n products."""
    ref = ref.float().double()
    kind = ref.to(dtype)
    assert torch.equal(torch.isnan(got), torch.isnan(kind)), what
    odd = torch.isinf(kind)
    assert torch.equal(torch.isinf(got), odd) and torch.equal(got[odd], kind[odd]), what
    number = torch.isfinite(kind)
    if not number.any():
        return
    ut = 2.0 ** -8 if dtype == torch.bfloat16 else U
    off = (got.double() - ref).abs()[number] / (chain(n) * size[number] + ut * ref[number].abs() + 1e-37)
    assert note(what + " / bound", off.max().item(), 1.0)


def product(x, y):
    """x (n, k) times y (k, m) in 64 bits and the same of magnitudes; 0 times an infinity is NaN as in the formula."""
    return x.double() @ y.double(), x.double().abs() @ y.double().abs()


def ids_of(rows):
    ids = (torch.arange(rows, device="cuda") * 7 % (COUNT + 1)).to(torch.int32)      # COUNT: none
    return ids


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cin,cout", SIZES)
def test_forward(rows, cin, cout, dtype):
    seed = case_seed((rows, cin, cout, str(dtype)))
    x, w = normal((rows, cin), dtype, seed), normal((cout, cin), dtype, seed + 1)
    a, b, ids = normal((COUNT, RANK, cin), dtype, seed + 2), normal((COUNT, cout, RANK), dtype, seed + 3), ids_of(rows)
    of = lambda k: [int(i) for i in (ids == k).nonzero().view(-1)[:4]]
    w[:, :3] = 0
    a[:, :, :3] = 0
    x[:, :3] = 0
    # adapter 0: inner is infinite in rank 0 and beyond bf16's largest number in rank 1, whose B is small
    i, j, k, _ = of(0)
    most = torch.finfo(torch.bfloat16).max
    a[0, 0, 0], x[i, 0], x[j, 0] = 2.0 ** 100, 2.0 ** 100, -2.0 ** 100
    a[0, 1, 1], a[0, 1, 2], x[k, 1], x[k, 2] = 1.0, 1.0, most, BEYOND
    b[0, :, 1] *= 2.0 ** -100
    # adapter 1: B is infinite; inner of one bit, of many, and zero
    b[1, 7, 0], b[1, 9, 1] = INF, -INF
    i, j = of(1)[:2]
    x[i] = 0
    x[i, 4] = 1
    a[1, :, 4] = torch.tensor([1.0, -2.0, 0.5, 0.25, 4.0])
    x[j] = 0
    y, inner = torch.empty((rows, cout), dtype=dtype, device="cuda"), torch.empty((rows, RANK), device="cuda")
    ws = torch.empty(max(256, B.adapter_fwd_workspace_bytes(x, a, b)), dtype=torch.uint8, device="cuda")
    B.adapter_fwd(x, w, None, a, b, ids, y, ws, inner=inner)
    ref, size = product(x, w.t())
    t, st = torch.zeros((rows, RANK), dtype=torch.float64, device="cuda"), torch.zeros((rows, RANK), dtype=torch.float64, device="cuda")
    for m in range(COUNT):
        r = (ids == m).nonzero().view(-1)
        t[r], st[r] = product(x[r], a[m].t())
        t[r] = t[r].float().double()                               # inner is held in fp32
        part, spart = product(t[r], b[m].t())
        ref[r] += part
        size[r] += spart
    check("inner", inner, t, st, cin, torch.float32)
    assert torch.isinf(inner).sum() == 2 and (inner.abs() > most).sum() == 3
    # (inner's own error, chain(c_in) of its magnitudes, is at most chain(c_in) of size where inner's magnitudes are its size; where they cancel it is not, so they are added)
    for m in range(COUNT):
        r = (ids == m).nonzero().view(-1)
        size[r] += torch.where(torch.isfinite(st[r]), st[r], 0.0) @ torch.where(torch.isfinite(b[m]), b[m], 0.0).double().abs().t()
    check("y", y, ref, size, cin + RANK, dtype)
    assert torch.isinf(y).any() and torch.isnan(y[j]).sum() == 2


@pytest.mark.parametrize("p", [0.0, 0.4])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cout,cin", SIZES)
def test_gradient(rows, cin, cout, dtype, p):
    seed = case_seed((rows, cin, cout, str(dtype), p))
    x, w, dy = normal((rows, cin), dtype, seed), normal((cout, cin), dtype, seed + 1), normal((rows, cout), dtype, seed + 4)
    a, b, ids = normal((COUNT, RANK, cin), dtype, seed + 2), normal((COUNT, cout, RANK), dtype, seed + 3), ids_of(rows)
    inner = normal((rows, RANK), torch.float32, seed + 5)
    of = lambda k: [int(i) for i in (ids == k).nonzero().view(-1)[:4]]
    most = torch.finfo(torch.bfloat16).max
    w[:3] = 0
    b[:, :3] = 0
    dy[:, :3] = 0
    # adapter 0: u infinite in rank 0 of one row, beyond bf16's largest in rank 1 of another, whose A, x and inner are small
    i, j = of(0)[:2]
    b[0, 0, 0], dy[i, 0] = 2.0 ** 20, -2.0 ** 120
    b[0, 1, 1], b[0, 2, 1], dy[j, 1], dy[j, 2] = 1.0, 1.0, most, BEYOND
    a[0, 1] *= 2.0 ** -100
    x[j] *= 2.0 ** -20
    inner[[i, j]] *= 2.0 ** -20
    # adapter 1: an infinite x, an infinite inner and one beyond bf16's largest
    i, j, k, _ = of(1)
    x[i, 5], x[i, 6] = INF, -INF
    inner[j, 0], inner[k, 1] = -INF, most + BEYOND
    dy[k] *= 2.0 ** -20
    # adapter 2: an infinite dy
    i = of(2)[0]
    dy[i, 4] = -INF
    # adapter 3: A infinite
    a[3, 2, 8] = INF
    drop = B.dropout_desc(p, 21, 6) if p else None
    dx, da, db = torch.empty_like(x), torch.empty(a.shape, device="cuda"), torch.empty(b.shape, device="cuda")
    ws = torch.empty(max(256, B.adapter_bwd_workspace_bytes(x, a, b)), dtype=torch.uint8, device="cuda")
    B.adapter_bwd(dy, x, w, a, b, ids, inner, dx, da, db, ws, drop=drop)
    only, _, _ = B.adapter_bwd(dy, x, w, a, b, ids, None, torch.empty_like(x), None, None, ws, drop=drop)
    assert torch.equal(torch.nan_to_num(only, nan=7.0), torch.nan_to_num(dx, nan=7.0))
    m = torch.from_numpy(O.mask((rows, cin), p, 21, 6)).cuda()
    masked = lambda t, m: torch.where(m > 0, t * m, 0.0)
    ref, size = product(dy, w)
    for n in range(COUNT):
        r = (ids == n).nonzero().view(-1)
        u, su = product(dy[r], b[n])
        u = u.float().double()
        back, sback = product(u, a[n])
        ref[r] += masked(back, m[r])
        finite = lambda t: torch.where(torch.isfinite(t), t, 0.0).double()
        # (u's own error is chain(c_out) of its magnitudes)
        size[r] += masked(sback + finite(su) @ finite(a[n]).abs(), m[r])
        dropped = masked(x[r].double(), m[r])
        ref_a, size_a = product(u.t(), dropped)
        check("da", da[n], ref_a, size_a + finite(su).t() @ finite(dropped).abs(), len(r) + cout, torch.float32)
        ref_b, size_b = product(dy[r].t(), inner[r])
        check("db", db[n], ref_b, size_b, len(r), torch.float32)
    check("dx", dx, ref, size, cout + RANK, dtype)
    assert torch.isinf(dx).any() and torch.isinf(da).any() and torch.isinf(db).any()
