"""Dropout on the GPU: every bit of it is given by the definition (one product rounded to fp32, then to the type)."""
import numpy as np
import pytest

import adapt_oracle as O
from paper_1708_04728_amd import binding as B
from util import kernel_launches

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def reference(x, p, seed, place):
    """x: a tensor of the host."""
    t = O.border(p)
    scale = np.float32(0 if t == 65536 else 65536.0 / (65536 - t))
    keep = O.draws(x.numel(), seed, place).reshape(x.shape) >= t
    return torch.where(torch.from_numpy(keep), x.float() * float(scale), torch.zeros(())).to(x.dtype)


def at_offset(t, offset):
    flat = torch.full((t.numel() + offset + 9,), 77.0, dtype=t.dtype, device="cuda")
    out = flat[offset:offset + t.numel()].view(t.shape)
    out.copy_(t)
    return flat, out


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape,p,offset", [((1, 1), 0.5, 0), ((1, 7), 0.4, 1), ((3, 8), 0.1, 0), ((5, 1000), 0.4, 3), ((2, 3, 17, 19), 0.5, 0), ((1 << 11, 1031), 0.25, 1),
                                            ((1, (1 << 23) + 5), 0.9, 0), ((4, 33), 0.0, 0), ((4, 33), 1.0, 0), ((4, 33), 1e-6, 0)])
def test_every_bit(dtype, shape, p, offset):
    gen = torch.Generator().manual_seed(sum(shape) + offset)
    x = torch.randn(shape, generator=gen).to(dtype)
    seed, place = 0xFEDCBA9876543210 + sum(shape), 2 ** 35 + offset
    fx, dx = at_offset(x, offset)
    fy, dy = at_offset(torch.zeros_like(x), offset)
    B.dropout_fwd(dx, B.dropout_desc(p, seed % 2 ** 64, place), dy)
    ref = reference(x, p, seed % 2 ** 64, place)
    assert torch.equal(dy.cpu(), ref)
    for f, keep in ((fx, None), (fy, None)):                      # nothing beside the tensor is written
        assert (f[:offset] == 77).all() and (f[offset + x.numel():] == 77).all()
    B.dropout_fwd(dx, B.dropout_desc(p, seed % 2 ** 64, place), dx)          # in place
    assert torch.equal(dx.cpu(), ref)


def test_what_is_dropped_is_zero_whatever_it_was():
    x = torch.full((3, 999), float("nan"), device="cuda")
    x[1] = float("inf")
    x[2] = -float("inf")
    y = B.dropout_fwd(x, B.dropout_desc(0.5, 5, 6), torch.empty_like(x)).cpu()
    keep = O.mask((3, 999), 0.5, 5, 6) > 0
    assert (y.numpy()[~keep] == 0).all() and not np.signbit(y.numpy()[~keep]).any()
    assert np.isnan(y[0].numpy()[keep[0]]).all() and (y[1].numpy()[keep[1]] == np.inf).all() and (y[2].numpy()[keep[2]] == -np.inf).all()


def test_maps_and_empty():
    x = torch.randn((2, 5, 4, 3), device="cuda")
    drop = B.dropout_desc(0.5, 1)
    y, z = torch.empty_like(x), torch.empty_like(x)
    B.dropout_fwd(B.NHWC(x), drop, B.NHWC(y))
    B.dropout_fwd(x, drop, z)
    assert torch.equal(y, z) and torch.equal(y.cpu(), reference(x.cpu(), 0.5, 1, 0))       # elements count in memory order
    e = torch.empty((0, 5), device="cuda")
    B.dropout_fwd(e, drop, e)
    torch.cuda.synchronize()


def test_a_recorded_call_draws_by_the_step():
    x = torch.randn((64, 333), device="cuda")
    y, step = torch.empty_like(x), torch.zeros(1, dtype=torch.int64, device="cuda")
    drop = B.dropout_desc(0.4, 9, 2 ** 64 - 2, step)              # the sum of offset and step wraps
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with B.capture(side, (x, y, step)) as c:
        B.dropout_fwd(x, drop, y, stream=side)
    for i in range(4):
        step.fill_(i)
        x.mul_(1.5)
        c.graph.launch()
        assert torch.equal(y.cpu(), reference(x.cpu(), 0.4, 9, (2 ** 64 - 2 + i) % 2 ** 64))
    assert kernel_launches(lambda: B.dropout_fwd(x, drop, y)) == 1
