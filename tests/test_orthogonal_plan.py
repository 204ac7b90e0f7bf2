"""Which kernel multiplies matrices of which size (csrc/orthogonal_plan.h), compiled for the host: a choice is one of the kernels, a contraction is shared only where every
wave keeps its k-blocks and there is a compute unit for every workgroup, and the sizes that the GPU tests run reach every kernel."""
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1708_04728_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include "orthogonal_plan.h"
int main()
{
    int cus, pieces, n;
    while (scanf("%d %d %d", &cus, &pieces, &n) == 3) {
        if (cus == 0) {                          // (n steps of a polynomial)
            double a, b, c;
            int growth;
            if (scanf("%lf %lf %lf", &a, &b, &c) != 3) return 1;
            const bool small = dr::stays_small(n, a, b, c, &growth);
            printf("%d %d\n", small, growth);
            continue;
        }
        dr::Group g;
        g.start();
        for (int i = 0; i < n; ++i) {
            int rows, cols;
            if (scanf("%d %d", &rows, &cols) != 2) return 1;
            g.add(rows, cols);
        }
        printf("%d %d %zu", g.whole, g.joined(cus), g.bytes(pieces, cus));
        for (int w = 0; w < dr::PRODUCTS; ++w) {
            const dr::Choice c = dr::choose(pieces, w, g.work[w], cus);
            printf(" %d %d %d %d", c.kernel, c.splits, g.work[w].tiles[c.kernel], g.work[w].longest);
        }
        printf("\n");
    }
}
"""
SIDE, WAVES, AHEAD = (1, 2, 4, 6, 8), (8, 8), (4, 1)


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("orthogonal_plan")
    (d / "plan.cpp").write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-I", CSRC, str(d / "plan.cpp"), "-o", str(d / "plan")])

    def ask(cases):
        """cases: (compute units, pieces, shapes)"""
        line = lambda cus, p, s: "%d %d %d " % (cus, p, len(s)) + " ".join("%d %d" % v for v in s)
        text = "\n".join(v if isinstance(v, str) else line(*v) for v in cases)
        out = subprocess.run([str(d / "plan")], input=text, capture_output=True, text=True, check=True, timeout=60).stdout.splitlines()
        assert len(out) == len(cases)
        return [[int(v) for v in line.split()] for line in out]
    return ask


def blocks(v):
    return -(-v // 32)


def check(case, plan):
    cus, pieces, shapes = case
    whole, joined, need, *products = plan
    assert bool(whole) == all((blocks(min(s)) == 1 and blocks(max(s)) <= 28) or (blocks(min(s)) == 2 and blocks(max(s)) <= 11) for s in shapes), case
    if joined:
        assert not whole and all(blocks(min(s)) <= 8 for s in shapes) and sum(blocks(min(s)) * blocks(max(s)) for s in shapes) <= 2 * cus, case
    square = lambda s: -(-min(s[0] * s[1], 4096 * 1024) // 4096)
    operands = sum((3 * blocks(min(s)) * blocks(max(s)) + 2 * blocks(min(s)) ** 2) * 2 * pieces * 1024 for s in shapes)
    for w in range(3):
        kernel, splits, tiles, longest = products[4 * w:4 * w + 4]
        assert 0 <= kernel < 5 and splits >= 1, case
        assert longest == 2 * max(blocks(max(s) if w == 0 else min(s)) for s in shapes), case
        T = SIDE[kernel]
        expect = sum(-(-blocks(min(s)) // T) * (-(-blocks(max(s)) // T)) if w == 2 else (-(-blocks(min(s)) // T)) * (-(-blocks(min(s)) // T) + 1) // 2 for s in shapes)
        assert tiles == expect, case
        if splits > 1:
            assert w == 0 and kernel < 2 and tiles * splits <= cus and splits * WAVES[kernel] * AHEAD[kernel] <= longest, case
    if not whole:
        squares = -(-(8 * sum(square(s) for s in shapes) + 256) // 1024) * 1024
        kernel, splits, tiles, _ = products[:4]
        assert need == squares + operands + (tiles * splits * SIDE[kernel] ** 2 * 4096 if splits > 1 else 0), case
    return joined, products


def test_choices_are_consistent(ask):
    rng = random.Random(3)
    size = lambda: max(1, int(2 ** rng.uniform(0, 13.5)))
    cases = [(rng.choice((256, 256, 304, 64, 1)), rng.choice((2, 3)), [(size(), size()) for _ in range(rng.choice((1, 1, 1, 2, 6, 64)))]) for _ in range(600)]
    for case, plan in zip(cases, ask(cases)):
        check(case, plan)


def test_the_gpu_tests_reach_every_kernel(ask):
    """... in either number of pieces, for a symmetric product and for the other, and with a contraction that workgroups share."""
    from test_gpu_orthogonal import LARGE, SHAPES
    for pieces in (2, 3):
        seen, shared, whole, together = set(), set(), False, False
        for shape, plan in zip(SHAPES + LARGE, ask([(256, pieces, [s]) for s in SHAPES + LARGE])):
            joined, products = check((256, pieces, [shape]), plan)
            whole, together = whole or plan[0], together or joined
            if not plan[0]:
                seen |= {(products[4 * w], w == 2) for w in ((0,) if joined else range(3))}
                shared |= {products[0]} if products[1] > 1 else set()
        assert whole and together and seen == {(k, w) for k in range(5) for w in (False, True)}, (pieces, sorted(seen))
        assert shared == {0, 1}, (pieces, shared)


def test_which_polynomials_stay_in_range(ask):
    """... against the largest values on a fine grid: fp16 pieces only where X, A and Q stay below 65504 over their scales, and the growth of a step is not underestimated."""
    import numpy as np
    rng = random.Random(4)
    cases = [(5, 3.4445, -4.7750, 2.0315), (5, 1.5, -0.5, 0.0), (64, 15 / 8, -10 / 8, 3 / 8), (1, 13.0, 0.0, 0.0), (3, 0.0, 0.0, 0.0), (2, 12.5, -12.0, 0.5), (4, 2.0, 0.0, 0.0),
             (2, float("nan"), 0.0, 0.0), (1, 1.0, float("inf"), 0.0)]
    cases += [(rng.randint(1, 8), rng.uniform(-6, 6), rng.uniform(-8, 8), rng.choice((0.0, rng.uniform(-4, 4)))) for _ in range(400)]
    answers = ask(["0 0 %d %r %r %r" % v for v in cases])
    assert answers[0] == [1, 2] and answers[1][0] and answers[2][0] and not any(answers[i][0] for i in (3, 5, 7, 8)) and 30 < sum(v[0] for v in answers[9:]) < 370
    for (steps, a, b, c), (small, growth) in zip(cases, answers):
        if not small:
            continue
        most = 1.0
        for _ in range(steps):
            s = np.linspace(0, most, 4001)
            q = np.abs(a + b * s ** 2 + c * s ** 4)
            assert most * 16384 < 65504 * 0.8 and most ** 2 * 4096 < 65504 * 0.8 and q.max() * 4096 < 65504 * 0.8 and q.max() <= 2.0 ** growth, (steps, a, b, c)
            most = (s * q).max()
