"""Newton-Schulz orthogonalisation and the descent step on it where the formulas have a limit to take."""
import numpy as np
import pytest

from paper_1708_04728_amd import binding as B
from test_gpu_orthogonal import COEFFICIENTS, DTYPES, array, gradient, newton_schulz, on_gpu, run, scratch
from util import case_seed, note

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


@pytest.mark.parametrize("shape", ((20, 30), (64, 100), (100, 300), (300, 900)))
@pytest.mark.parametrize("coefficients,steps,below", (((1.0, 0.0, 0.0), 41, 40), ((1.1, -0.1, 0.0), 40, 40), ((1.5, -0.5, 0.0), 40, 60), (COEFFICIENTS, 30, 100), ((0.5, 0.0, 0.0), 40, 0),
                                                      ((0.5, 0.0, 0.0), 40, 20), ((0.5, 1.5, -1.0), 40, 40)))
def test_many_steps_on_small_norms(shape, coefficients, steps, below):
    """|G| = 2^-below eps (0: no eps).  Every X stays far below one, or far below the one before it, so that each step multiplies it by a and nothing else: an error u |X| in
    each of the steps + 1 matrices X, and one u in each of the a, come to at most (2 steps + 1) |a|^steps u 2^-below at the end."""
    coefficients = tuple(float(np.float32(v)) for v in coefficients)
    g = gradient(np.random.default_rng(case_seed((shape, steps), below)), *shape)
    g = (g / np.linalg.norm(g.astype(np.float64)) * 2.0 ** -10).astype(np.float32)
    eps = 2.0 ** (below - 10) if below else 0.0
    got, = run([on_gpu(g)], steps=steps, coefficients=coefficients, eps=eps)
    ref = newton_schulz(g.astype(np.float64), steps, coefficients, eps)
    assert note("|error|", np.linalg.norm(array(got) - ref) / ((2 * steps + 1) * abs(coefficients[0]) ** steps * 2.0 ** -23 * 2.0 ** -below), 1.0)
