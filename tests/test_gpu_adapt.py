"""Dropout, adapters and the softmax loss together, as adapt.py runs them, against the definitions in 64 bits."""
import numpy as np
import pytest

import adapt_oracle as O
from paper_1708_04728_amd import adapt, binding as B
from util import note

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def model_of(p, rows=20, c=72, classes=50, tasks=3, rank=4):
    gen = torch.Generator(device="cuda").manual_seed(4)
    w, bias = torch.randn((classes, c), device="cuda", generator=gen) * 0.2, torch.randn(classes, device="cuda", generator=gen)
    m = adapt.AdaptedClassifier(w, bias, tasks, rank, rows, p=p, seed=5, input_gradient=True, generator=gen)
    m.b.copy_(torch.randn(m.b.shape, device="cuda", generator=gen))
    x = torch.randn((rows, c), device="cuda", generator=gen).abs()
    ids = torch.randint(-1, tasks, (rows,), device="cuda", generator=gen, dtype=torch.int32)
    labels = torch.randint(-1, classes, (rows,), device="cuda", generator=gen, dtype=torch.int32)
    return m, x, ids, labels


def oracle_step(m, x, ids, labels, p, place, smoothing):
    f = lambda t: t.double().cpu().numpy()
    ids, labels = ids.tolist(), labels.tolist()
    mask = O.mask(tuple(x.shape), p, 5, place)
    args = (f(x), f(m.w))
    ad = (f(m.a), f(m.b), ids, np.ones(len(m.a)), mask)
    y, inner = O.adapter_fwd(*args, f(m.bias), *ad)
    loss, _, dy = O.softmax_loss(y, labels, float(np.float32(smoothing)), True)
    return (loss,) + O.adapter_bwd(dy, *args, *ad, inner)


@pytest.mark.parametrize("p", [0.0, 0.4])
def test_a_step(p):
    m, x, ids, labels = model_of(p)
    for step in range(3):
        loss, dx, da, db = oracle_step(m, x, ids, labels, p, step, 0.1)
        a, b = m.a.clone(), m.b.clone()
        m.step(x, ids, labels, 0.5, smoothing=0.1)
        # logits are sums of 72 + 4 products below 2 in size: off by 2 (76 + 4) 2^-24 of a sum of magnitudes below 60, 6e-4 at most of a logit; a gradient of the loss moves by
        # at most twice that in each of 50 terms beside its own sums, whose magnitudes are larger than their rms by less than 30
        for got, ref in ((m.da, da), (m.db, db), (m.dx, dx)):
            rms = np.sqrt((ref ** 2).mean())
            assert note("gradient, of its rms", np.abs(got.double().cpu().numpy() - ref).max() / rms, 2e-3)
        assert abs(m.loss.item() - loss) < 1.2e-3
        assert torch.equal(m.a, a - 0.5 * m.da) and torch.equal(m.b, b - 0.5 * m.db)


def test_gradient_by_differences():
    """The loss of a step moves as its gradient says: a central difference along a direction, masks as they were.  The loss is computed in fp32 (about 1e-6 off); over 2 d = 0.04 that is
    5e-5, and the third derivative along a direction of length one adds a few times d^2 / 6 = 7e-5 of a logit's cube, below 1e-2 of the derivative here."""
    m, x, ids, labels = model_of(0.4)
    m.gradients(x, ids, labels)
    da, db = m.da.clone(), m.db.clone()
    for grad, param in ((da, m.a), (db, m.b)):
        unit = grad / grad.norm()
        along = grad.norm().item()
        ends = []
        for d in (0.02, -0.02):
            at = param.clone()
            param.add_(unit, alpha=d)
            m.gradients(x, ids, labels)
            ends.append(m.loss.item())
            param.copy_(at)
        assert abs((ends[0] - ends[1]) / 0.04 - along) < 1e-2 * along + 5e-5


def test_a_recorded_step_draws_anew():
    m, x, ids, labels = model_of(0.4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with B.capture(side, (m, x, ids, labels)) as c:
        m.gradients(x, ids, labels, stream=side)
    for step in range(4):
        m.draws.fill_(step)
        c.graph.launch()
        recorded = [t.clone() for t in (m.loss, m.da, m.db, m.dx)]
        m.gradients(x, ids, labels)
        for a, b in zip(recorded, (m.loss, m.da, m.db, m.dx)):
            assert torch.equal(a, b)


def test_command_runs(capsys):
    adapt.main(batch=16, c=64, classes=40, tasks=2, rank=4, steps=3)
    assert "loss" in capsys.readouterr().out
