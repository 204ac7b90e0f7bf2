"""A classifier made for a larger batch than it is given (an epoch's last one)."""
import pytest

from paper_1708_04728_amd import adapt

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def model(rows, c, classes):
    gen = torch.Generator(device="cuda").manual_seed(4)
    w, bias = torch.randn((classes, c), device="cuda", generator=gen) * 0.2, torch.randn(classes, device="cuda", generator=gen)
    m = adapt.AdaptedClassifier(w, bias, 4, 8, rows, p=0.4, seed=5, input_gradient=True, generator=gen)
    m.b.copy_(torch.randn(m.b.shape, device="cuda", generator=gen))
    return m


@pytest.mark.parametrize("made_for,rows,c,classes", [(2049, 2048, 1024, 1000), (2500, 2000, 1024, 1000), (130, 1, 72, 50), (4200, 4096, 1024, 1000)])
def test_a_smaller_batch_has_the_bits_of_a_model_of_its_size(made_for, rows, c, classes):
    large, own = model(made_for, c, classes), model(rows, c, classes)
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn((rows, c), device="cuda", generator=gen).abs()
    ids = torch.randint(-1, 4, (rows,), device="cuda", generator=gen, dtype=torch.int32)
    labels = torch.randint(-1, classes, (rows,), device="cuda", generator=gen, dtype=torch.int32)
    for _ in range(2):
        for m in (large, own):
            m.step(x, ids, labels, 0.1)
        for a, b in ((large.loss, own.loss), (large.da, own.da), (large.db, own.db), (large.a, own.a), (large.b, own.b), (large.dx[:rows], own.dx)):
            assert torch.isfinite(a).all() and torch.equal(a, b)
