"""The softmax loss and its gradient on the GPU against the formulas in 64 bits.

With u = 2^-24, R = max |z - top| over the row's finite logits and P the sum of exponentials:
* an exponential's argument z - top is rounded once (|z - top| u relative to the exponential), the exponential itself is good to 4 u;
* P is added over at most 64 terms of a lane, 6 exchanges and 16 waves (rows in registers), or over 8 terms of each of C / 8192 turns with one product by exp(old - new top), which rounds as the
  exponentials do, each: relative error at most (90 + C / 1024 + 2 R + 8) u =: E u;
* the logarithm adds 2 u |log P| and E u; the label's logit 2 u R; smoothing e times a mean of z - top, added along at most 90 + C / 1024 terms: e (95 + C / 1024) u (R + |top|)
  (the long kernel adds z itself and takes C top off).
* dz = g (p - target): p is off by (2 E + R + 8) u p, the difference by 3 u (p + target) g, and the result is rounded to its type.  Exponentials below 2^-126 become 0."""
import numpy as np
import pytest

import adapt_oracle as O
from paper_1708_04728_amd import binding as B
from util import note

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24


def run(z, labels, smoothing=0.0, mean=True, inplace=False, gradient=True):
    n = len(z)
    ws = torch.full((max(B.softmax_loss_workspace_bytes(z), 256),), 255, dtype=torch.uint8, device="cuda")
    loss, row = torch.full((1,), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda")
    dz = (z if inplace else torch.full_like(z, 7.0)) if gradient else None
    B.softmax_loss_grad(z, torch.as_tensor(labels, dtype=torch.int32).cuda(), dz, loss, ws, smoothing, mean, row)
    return loss.item(), row.double().cpu().numpy(), None if dz is None else dz.double().cpu().numpy()


def check(z, labels, smoothing, mean, got):
    """z: host tensor."""
    zz = z.double().numpy()
    e = float(np.float32(smoothing))
    loss, row, dz = O.softmax_loss(zz, labels, e, mean)
    rows, c = zz.shape
    has = np.array([0 <= t < c for t in labels])
    n = max(has.sum(), 1)
    g = 1.0 / n if mean else 1.0
    top = zz.max(1)
    r = (top[:, None] - zz).max(1)
    p = np.exp(zz - top[:, None])
    lse = np.log(p.sum(1))
    big = 90 + c / 1024 + 2 * r + 8
    row_tol = U * (big * 2 + 2 * lse + 2 * r + e * (95 + c / 1024) * 2 * (r + np.abs(top)) + 4 * np.abs(row)) * has
    p = p / p.sum(1)[:, None]
    target = np.full((rows, c), e / c)
    target[np.arange(rows)[has], np.array(labels)[has]] += 1 - e
    ut = 2.0 ** -8 if z.dtype == torch.bfloat16 else U
    dz_tol = (g * U * ((2 * big + r + 8)[:, None] * p + 4 * (p + target)) + ut * np.abs(dz) + 2.0 ** -126) * has[:, None]
    assert note("row loss / bound", np.max(np.abs(got[1] - row) / np.maximum(row_tol, 1e-300), initial=0.0), 1.0)
    assert note("loss / bound", abs(got[0] - loss) / (row_tol.sum() * g + 2 * U * abs(loss) + 1e-30), 1.0)
    if got[2] is not None:
        assert note("gradient / bound", np.max(np.abs(got[2] - dz) / np.maximum(dz_tol, 1e-300), initial=0.0), 1.0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,classes", [(1, 1), (1, 2), (3, 7), (9, 64), (33, 513), (128, 1000), (5, 1025), (7, 2049), (4, 4100), (3, 8193), (3, 16385), (2, 32003), (2, 50001), (2, 65537),
                                          (2, 131075), (2500, 11)])
def test_against_the_formulas(dtype, rows, classes):
    rng = np.random.default_rng(rows * 7 + classes)
    z = torch.from_numpy(3 * rng.standard_normal((rows, classes))).to(dtype)
    labels = rng.integers(0, classes, rows)
    if rows > 2:
        labels[rng.integers(0, rows, max(1, rows // 8))] = -1
        labels[0] = classes                                       # no class either
    for smoothing, mean, inplace in ((0.0, True, False), (0.1, True, True), (0.1, False, False)):
        check(z, labels, smoothing, mean, run(z.cuda(), labels, smoothing, mean, inplace))


def test_range_of_logits():
    z = torch.tensor([[1e4, -1e4, 0.0, 9999.0], [-3e38, 3e38, 0.0, 1.0], [-80.0, -90.0, -100.0, -101.0], [5.0, 5.0, 5.0, 5.0]])
    check(z, [3, 1, 0, 2], 0.0, True, run(z.cuda(), [3, 1, 0, 2]))


def test_masked_classes_and_rows_without_a_number():
    inf = float("inf")
    for classes in (5, 3000, 20000, 70000):
        z = torch.full((6, classes), -inf)
        z[:, :3] = torch.tensor([1.0, 2.0, 0.5])
        z[1, 2] = float("nan")
        z[2] = -inf
        z[3, 0] = inf
        z[4] = float("nan")                                       # no label: nothing is asked of it
        labels = [1, 0, 0, 1, -7, 4]
        loss, row, dz = run(z.cuda(), labels, mean=False)
        p = np.exp([1.0, 2.0, 0.5]) / np.exp([1.0, 2.0, 0.5]).sum()
        assert abs(row[0] + np.log(p[1])) < 1e-6 and np.abs(dz[0, :3] - (p - [0, 1, 0])).max() < 1e-6 and (dz[0, 3:] == 0).all()
        assert np.isnan(row[1:4]).all() and np.isnan(dz[1, :3]).all() and np.isnan(dz[2]).all()
        assert np.isnan(dz[3]).any() and row[4] == 0 and (dz[4] == 0).all()
        assert row[5] == inf and dz[5, 4] == -1 and np.abs(dz[5, :3] - p).max() < 1e-6      # the label's class is masked
        assert np.isnan(loss)


def test_no_label_at_all_and_no_rows():
    z = torch.randn((9, 30), device="cuda")
    loss, row, dz = run(z, [-1] * 9)
    assert loss == 0 and (row == 0).all() and (dz == 0).all()
    loss, row, dz = run(torch.empty((0, 30), device="cuda"), [])
    assert loss == 0
    check(z.cpu(), list(range(9)), 0.1, True, run(z, list(range(9)), 0.1, gradient=False))


def test_one_row_beside_others_has_the_bits_of_one_alone():
    z = torch.randn((40, 1000), device="cuda").bfloat16()
    labels = list(range(40))
    _, row, dz = run(z, labels, mean=False)
    _, alone, dalone = run(z[17:18].contiguous(), [17], mean=False)
    assert row[17] == alone[0] and (dz[17] == dalone[0]).all()


def test_unaligned_rows_and_a_recorded_call():
    flat = torch.full((3 * 1001 + 9,), 5.0, dtype=torch.bfloat16, device="cuda")
    z = flat[3:3 + 3 * 1001].view(3, 1001)
    z.copy_(torch.randn((3, 1001), device="cuda"))
    host = z.cpu()
    labels = torch.tensor([7, 1000, -1], dtype=torch.int32, device="cuda")
    check(host, labels.tolist(), 0.0, True, run(z, labels.tolist(), inplace=True))
    assert (flat[:3] == 5).all() and (flat[3 + 3 * 1001:] == 5).all()
    z.copy_(host)
    dz, loss, row, ws = torch.empty_like(z), torch.empty(1, device="cuda"), torch.empty(3, device="cuda"), torch.empty(B.softmax_loss_workspace_bytes(z), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with B.capture(side, (z, labels, dz, loss, row, ws)) as c:
        B.softmax_loss_grad(z, labels, dz, loss, ws, 0.1, row_loss=row, stream=side)
    for i in range(3):
        z.mul_(1.25)
        labels.copy_((labels + 1) % 1001)
        c.graph.launch()
        got = (loss.item(), row.double().cpu().numpy(), dz.double().cpu().numpy())
        check(z.cpu(), labels.tolist(), 0.1, True, got)
