"""Small probabilities in fp32: the exponential to its last bits, in every kernel of the softmax loss.

A row's largest logit is 0 and its label's, the others d = z lie in -85 .. -20 (exactly given) or are -inf, so that the sum rounds to 1: the others are at most 12 exp(-20) < 0.5 u together
(u = 2^-24), and nothing but the exponential shows in dz = exp(d).  The exponential: the argument's product with log2 e is rounded and what that loses is put back, up to |d| 0.05 u for ln 2 in 24
bits; the instruction is good to 2 u (one unit in the last place), the correction's product rounds once (u), as does the one with 1 / sum (u), and 1 / sum is within 0.5 u of what it stands for."""
import numpy as np
import pytest

from paper_1708_04728_amd import binding as B
from util import note

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24


@pytest.mark.parametrize("classes", [5, 12, 600, 1500, 3000, 7000, 12000, 20000, 50001, 70003])
def test_small_probabilities(classes):
    rows = 200
    rng = np.random.default_rng(classes)
    z = torch.full((rows, classes), -float("inf"))
    places = np.stack([rng.permutation(classes)[:min(classes, 12)] for _ in range(rows)])
    d = -rng.uniform(20, 85, places.shape).astype(np.float32)
    d[:, 0] = 0
    z[torch.arange(rows)[:, None], torch.from_numpy(places)] = torch.from_numpy(d)
    labels = torch.from_numpy(places[:, 0].astype(np.int32)).cuda()
    z = z.cuda()
    dz, loss = torch.full_like(z, 7.0), torch.empty(1, device="cuda")
    ws = torch.empty(max(256, B.softmax_loss_workspace_bytes(z)), dtype=torch.uint8, device="cuda")
    B.softmax_loss_grad(z, labels, dz, loss, ws, mean=False)
    got = dz.cpu()[torch.arange(rows)[:, None], torch.from_numpy(places)][:, 1:].double().numpy()
    size = np.abs(d[:, 1:].astype(np.float64))
    ref = np.exp(-size)
    assert note("error / bound", np.max(np.abs(got / ref - 1) / ((4.5 + 0.05 * size) * U)), 1.0)
    dz[torch.arange(rows, device="cuda")[:, None], torch.from_numpy(places).cuda()] = 0.0
    assert (dz == 0).all()
