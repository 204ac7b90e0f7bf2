"""Newton-Schulz orthogonalisation and the descent step on it where the formulas have a limit to take."""
import numpy as np
import pytest

from paper_1708_04728_amd import binding as B
from test_gpu_orthogonal import DTYPES, array, gradient, on_gpu, run, scratch
from util import case_seed

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("coefficients", (B.NEWTON_SCHULZ, (12.5, -12.0, 0.5)))
def test_zeros_stay_zero_without_eps(dtype, coefficients):
    """0 / (0 + 0) is no update: matrices of zeros stay zero, by themselves and beside others, in every kernel that divides by the norm."""
    rng = np.random.default_rng(1)
    for shapes in ([(40, 60)], [(192, 576)], [(300, 700)], [(40, 60), (33, 31)], [(300, 700), (40, 60), (192, 576)]):
        zeros = [torch.zeros(s, dtype=DTYPES[dtype], device="cuda") for s in shapes]
        for o in run(zeros, eps=0.0, coefficients=coefficients, steps=2):
            assert torch.equal(o, torch.zeros_like(o))
        some = [on_gpu(gradient(rng, *s), dtype) for s in shapes]
        alone = run(some, eps=0.0, coefficients=coefficients, steps=2)
        mixed = run(zeros[:1] + some[1:], eps=0.0, coefficients=coefficients, steps=2)
        assert torch.equal(mixed[0], zeros[0]) and all(torch.equal(a, b) for a, b in zip(mixed[1:], alone[1:]))


@pytest.mark.parametrize("shapes", ([(64, 3, 7, 7)], [(192, 64, 3, 3)], [(300, 700)], [(64, 3, 7, 7), (192, 64, 3, 3), (300, 700), (24, 16, 5, 5)]))
def test_a_layer_without_gradient_keeps_its_weights(shapes):
    """All-zero gradient and momentum and eps = 0: the weights only decay."""
    rng = np.random.default_rng(case_seed(shapes))
    w = [on_gpu(rng.standard_normal(s)) for s in shapes]
    start = [t.clone() for t in w]
    g, m = ([torch.zeros_like(t) for t in w] for _ in range(2))
    params = B.muon_params(list(zip(w, g, m)))
    B.muon_step(params, scratch(B.muon_step_workspace_bytes(params)), 0.5, momentum=0.9, weight_decay=0.25, eps=0.0)
    torch.cuda.synchronize()
    for before, after, momentum in zip(start, w, m):
        assert not momentum.any() and np.array_equal(array(after), array(before * 0.875))
