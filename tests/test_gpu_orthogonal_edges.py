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


def directions(shape):
    """A matrix with one element a row (a column, where it is tall): singular values from 1 to 10^-28, 28 decades in all."""
    m = min(shape)
    g = np.zeros(shape, dtype=np.float32)
    i = np.arange(m)
    g[(i, (7 * i + 3) % shape[1]) if m == shape[0] else ((7 * i + 3) % shape[0], i)] = 10.0 ** np.linspace(0, -28, m)
    return g


def off_by(got, g, all_bits):
    """Largest ratio of an element's error to its bound.  Elements do not meet: each is s -> s (a + b s^2 + c s^4) five times.  Rounding X, Q and their product, five times, and X and
    the norm at the start come to at most 17 u s, which grows at most a-fold in a step; without all bits what is held is off by as much as 2^-33 of the largest instead, where that is more."""
    s = g.astype(np.float64) / (np.linalg.norm(g.astype(np.float64)) + float(np.float32(1e-7)))
    ref, (a, b, c) = s.copy(), COEFFICIENTS
    for _ in range(5):
        ref = ref * (a + b * ref ** 2 + c * ref ** 4)
    tol = 17 * a ** 5 * (2.0 ** -23 * s + (0 if all_bits else 2.0 ** -33 * (s > 0)))
    assert not got[s == 0].any()
    return (np.abs(got - ref)[s > 0] / tol[s > 0]).max()


@pytest.mark.parametrize("all_bits", (False, True))
@pytest.mark.parametrize("shape", ((2, 2), (40, 61), (64, 150), (61, 40), (192, 577), (290, 451), (700, 1300), (1501, 1500), (2700, 2600)))
def test_singular_values_far_apart(shape, all_bits):
    g = directions(shape)
    got, = run([on_gpu(g)], all_bits=all_bits)
    assert note("|error|", off_by(array(got), g, all_bits), 1.0)
    # in a list
    got = run([on_gpu(g), on_gpu(g[:1])], all_bits=all_bits)
    assert note("|error|", max(off_by(array(got[0]), g, all_bits), off_by(array(got[1]), g[:1], all_bits)), 1.0)


@pytest.mark.parametrize("shape", ((40, 61), (192, 577), (700, 1301)))
def test_a_step_on_singular_values_far_apart(shape):
    """From weights of zero without momentum and decay, a step of one: minus the orthogonalised gradient."""
    g = directions(shape)
    w, m = (torch.zeros(shape, device="cuda") for _ in range(2))
    params = B.muon_params([(w, on_gpu(g), m)])
    B.muon_step(params, scratch(B.muon_step_workspace_bytes(params)), 1.0, momentum=0.0, weight_decay=0.0, all_bits=True)
    torch.cuda.synchronize()
    assert note("|error|", off_by(-array(w), g, True), 1.0)


def test_all_bits_of_bf16_matrices():
    g = torch.from_numpy(directions((64, 150))).bfloat16().cuda()
    got, = run([g], all_bits=True)
    wide, = run([g.float()], all_bits=True)
    assert torch.equal(got, wide.bfloat16())
