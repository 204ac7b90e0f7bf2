"""The softmax loss where its terms are as large as fp32 holds: masked classes at the type's lowest value beside smoothing, labels among them, and smoothing 1.

The loss l = log sum exp d - (1 - e) d_t - e mean d, d = z - top: each of the three is a number of fp32 here, if their parts are added without going beyond it.  Bound: log and its sum as below
1e-5 in all, the label's part rounds twice (2 u of its size, u = 2^-24), the mean is a sum of C terms whose signs agree (d <= 0), at most C + 4 roundings along any path, and the whole one more each."""
import numpy as np
import pytest

from paper_1708_04728_amd import binding as B
from util import note

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24
CLASSES = [5, 30, 700, 1500, 3000, 7000, 12000, 20000, 50001, 70003]


def run(z, labels, smoothing):
    dz, row, loss = torch.full_like(z, 7.0), torch.empty(len(z), device="cuda"), torch.empty(1, device="cuda")
    ws = torch.empty(max(256, B.softmax_loss_workspace_bytes(z)), dtype=torch.uint8, device="cuda")
    B.softmax_loss_grad(z, torch.tensor(labels, dtype=torch.int32, device="cuda"), dz, loss, ws, smoothing, False, row)
    return row.double().cpu().numpy(), dz.double().cpu().numpy()


def expect(z, labels, e):
    z = z.double().cpu().numpy()
    top = z.max(1)
    d = z - top[:, None]
    p = np.exp(d)
    lse = np.log(p.sum(1))
    label = d[np.arange(len(z)), labels]
    parts = [lse, -(1 - e) * label, -e * d.mean(1)]
    tol = 1e-5 + 3 * U * np.abs(parts[1]) + (z.shape[1] + 6) * U * np.abs(parts[2])
    target = np.full(z.shape, e / z.shape[1])
    target[np.arange(len(z)), labels] += 1 - e
    return sum(parts), tol, p / p.sum(1)[:, None] - target


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("classes", CLASSES)
def test_masks_of_the_lowest_value(classes, dtype):
    lowest, e = torch.finfo(dtype).min, float(np.float32(0.01))
    z = torch.randn((4, classes), generator=torch.Generator().manual_seed(classes)).to(dtype)
    z[1, 1:4] = lowest                                            # a few masked
    z[2, 1:] = lowest                                             # all but the label
    z[3, :classes // 2] = lowest                                  # half of them, the label too
    z[3, classes - 1] = 300.0
    labels = [0, 4, 0, 1]
    ref, tol, grad = expect(z, labels, e)
    row, dz = run(z.cuda(), labels, e)
    assert np.isfinite(ref).all() and np.abs(ref).max() < 3.4e38 and np.isfinite(row).all()
    assert note("row loss / bound", np.max(np.abs(row - ref) / tol), 1.0)
    ut = 2.0 ** -8 if dtype == torch.bfloat16 else U
    # probabilities are good to 1e-4 of themselves (logits below 8 beside a sum of at most 70003 terms), the smoothing's part and the result round
    assert note("gradient / bound", np.max(np.abs(dz - grad) / (1e-4 * (grad + 1) * (grad > 0) + (ut + 1e-5) * np.abs(grad) + 1e-6 * e)), 1.0)


@pytest.mark.parametrize("classes", CLASSES)
def test_a_label_as_far_below_as_its_part_allows(classes):
    z = torch.zeros((2, classes))
    z[:, 0], z[:, 1] = 3e38, -3e38
    e = float(np.float32(0.75))                                   # 6e38 from the largest: beyond fp32, its quarter is not
    ref, tol, _ = expect(z, [0, 1], e)
    ok = np.abs(ref) < 3.3e38
    row, _ = run(z.cuda(), [0, 1], e)
    assert ok[0] and note("row loss / bound", np.max((np.abs(row - ref) / tol)[ok]), 1.0)
    assert np.isinf(row[~ok]).all()


@pytest.mark.parametrize("classes", CLASSES)
def test_smoothing_of_one_asks_nothing_of_the_label(classes):
    """(1 - e) z_t is no part of the loss then, whatever the label's logit: with a masked class the mean is infinite, and so is the loss."""
    z = torch.zeros((2, classes))
    z[0, 1] = -float("inf")
    row, dz = run(z.cuda(), [1, 1], 1.0)
    assert row[0] == np.inf and abs(row[1] - np.log(classes)) < 1e-5
    ref = np.full(classes, 1 / (classes - 1) - 1 / classes)
    ref[1] = -1 / classes
    assert np.abs(dz[0] - ref).max() < 1e-6 and np.abs(dz[1]).max() < 1e-6
