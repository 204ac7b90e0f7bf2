"""All 32 bits of inner and of its gradient reach y and dx, in every kernel of the wide product.

Per pixel inner = 1 + 2^-9 + 2^-17 and the projection gives -(1 + 2^-9), times powers of two that differ by pixel and by output, so y = 2^-17 times them: of inner's 18 bits the
first 16 cancel.  Every product is exact in fp32 and at most six additions have two terms that are not zero, of sums below 2: off by at most 6 x 2 x 2^-23 < 2^-19, and by the
rounding of the result."""
import pytest

import adapt_oracle as O
from paper_1708_04728_amd import binding as B
from util import note

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

SIZES = [(24, 72, 136), (1100, 72, 520), (2048, 72, 2048), (4096, 72, 4096), (4096, 77, 4099)]      # few rows; tiles of 64, of 128, of 256; rows that are not aligned


def powers(n, dtype, lo=-3):
    """n signed powers of two 2^lo .. 2^(lo + 6), none like its neighbours."""
    i = torch.arange(n, device="cuda")
    return (torch.where(i % 2 == 0, 1.0, -1.0) * torch.exp2((i * 5 % 7 + lo).float())).to(dtype)


def parts(scale, n, values):
    """(len(scale), n): `values` in columns 1, 34, 65 times scale, zeros elsewhere (columns of different steps of the contraction)."""
    out = torch.zeros((len(scale), n), dtype=scale.dtype, device="cuda")
    for c, v in zip((1, 34, 65), values):
        out[:, c] = scale * v
    return out


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,narrow,wide", SIZES)
@pytest.mark.parametrize("rank", [1, 19])
def test_what_cancels(rows, narrow, wide, rank, dtype):
    ut = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    per_row, per_out = powers(rows, dtype), powers(wide, dtype, -2)
    v = parts(per_row, narrow, (1.0, 2.0 ** -4, 2.0 ** -8))                              # x, or dy
    w = parts(per_out, narrow, (-1.0, -2.0 ** -5, 0.0))                                   # (wide, narrow)
    factor = torch.zeros((2, rank, narrow), dtype=dtype, device="cuda")                   # A, or B transposed
    factor[1, rank - 1] = parts(torch.ones(1, dtype=dtype, device="cuda"), narrow, (1.0, 2.0 ** -5, 2.0 ** -9))[0]
    other = torch.zeros((2, wide, rank), dtype=dtype, device="cuda")                      # B, or A transposed
    other[1, :, rank - 1] = per_out
    ids = torch.ones(rows, dtype=torch.int32, device="cuda")
    size = (per_row.double()[:, None] * per_out.double()[None]).abs()
    ref = per_row.double()[:, None] * per_out.double()[None] * 2.0 ** -17

    def check(what, got, ref):
        assert note(what + " / bound", ((got.double() - ref).abs() / (2.0 ** -19 * size + ut * ref.abs())).max().item(), 1.0 + 1e-9)

    ws = torch.empty(B.adapter_bwd_workspace_bytes(torch.empty((rows, max(narrow, wide)), dtype=dtype, device="cuda"), torch.empty((2, rank, max(narrow, wide)), dtype=dtype, device="cuda"),
                                                   torch.empty((2, max(narrow, wide), rank), dtype=dtype, device="cuda")), dtype=torch.uint8, device="cuda")
    y = torch.empty((rows, wide), dtype=dtype, device="cuda")
    B.adapter_fwd(v, w, None, factor, other, ids, y, ws)
    check("y", y, ref)
    # the gradient of a projection from `wide` to `narrow` channels: W is (narrow, wide)
    a, b = other.transpose(1, 2).contiguous(), factor.transpose(1, 2).contiguous()
    dx = torch.empty((rows, wide), dtype=dtype, device="cuda")
    B.adapter_bwd(v, torch.zeros_like(dx), w.t().contiguous(), a, b, ids, None, dx, None, None, ws)
    check("dx", dx, ref)
    # with dropout (p = 1/2: what is kept counts twice), the mask drawn in the product and, beside da, left by the sums
    m = torch.from_numpy(O.mask((rows, wide), 0.5, 11, 5)).cuda()
    drop = B.dropout_desc(0.5, 11, 5)
    x = torch.ones((rows, wide), dtype=dtype, device="cuda")
    whole = torch.where(m > 0, 2 * ref, -2 * (1 + 2.0 ** -9) * per_row.double()[:, None] * per_out.double()[None])
    size = 2 * size
    for da in (None, torch.empty(a.shape, device="cuda")):
        B.adapter_bwd(v, x, (2 * w).t().contiguous(), a, b, ids, None, dx, da, None, ws, drop=drop)
        check("dx with dropout", dx, whole)
