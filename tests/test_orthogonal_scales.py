"""The scale that a matrix far below eps is held at (csrc/orthogonal_plan.h), compiled for the host and followed step by step: what a step may multiply a singular value by
never takes it out of fp16's range, and what a step multiplies small ones by never takes more than a few bits from them, however many steps."""
import math
import os
import random
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1708_04728_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include "orthogonal_plan.h"
int main()
{
    int steps, shift;
    double a, b, c;
    while (scanf("%d %lf %lf %lf %d", &steps, &a, &b, &c, &shift) == 5) {
        int growth;
        float spare = 0.f;
        const bool small = dr::stays_small(steps, a, b, c, &growth, &spare);
        printf("%d", small);
        for (int k = 0; small && k <= steps; ++k) printf(" %d", dr::held_at(shift, growth, spare, k));
        printf("\n");
    }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("orthogonal_scales")
    (d / "scales.cpp").write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-I", CSRC, str(d / "scales.cpp"), "-o", str(d / "scales")])

    def ask(cases):
        """cases: (steps, a, b, c, shift); for each None (three pieces), or the powers of two that X is held at before step 0, 1, ... and at the end"""
        text = "\n".join("%d %r %r %r %d" % v for v in cases)
        out = subprocess.run([str(d / "scales")], input=text, capture_output=True, text=True, check=True, timeout=60).stdout.splitlines()
        assert len(out) == len(cases)
        return [[int(w) for w in v.split()[1:]] if v.split()[0] == "1" else None for v in out]
    return ask


NAMED = [(3.4445, -4.7750, 2.0315), (1.5, -0.5, 0.0), (1.875, -1.25, 0.375), (2.0, -1.5, 0.5), (1.1, -0.1, 0.0), (1.0, 0.0, 0.0), (0.5, 0.0, 0.0), (1.0, -0.5, 0.1), (0.5, 1.5, -1.0),
         (0.01, 0.0, 0.0), (0.0, 0.0, 0.0), (-3.4445, 4.7750, -2.0315)]


def test_published_polynomials_take_two_pieces_for_any_number_of_steps(ask):
    cases = [(steps, *v, 0) for v in NAMED[:4] for steps in (1, 2, 5, 12, 30, 64)]
    for case, held in zip(cases, ask(cases)):
        assert held == [0] * (case[0] + 1), case


def test_small_values_keep_their_bits(ask):
    rng = random.Random(7)
    cases = [(steps, *v, shift) for v in NAMED for steps in (1, 5, 12, 40, 41, 64) for shift in (0, 1, 5, 20, 40, 120, 276)]
    cases += [(rng.randint(1, 64), rng.uniform(0.9, 1.2), rng.uniform(-0.3, 0.05), 0.0, rng.randint(0, 276)) for _ in range(300)]
    cases += [(rng.randint(1, 12), rng.uniform(-4, 4), rng.uniform(-5, 5), rng.uniform(-2, 2), rng.randint(0, 276)) for _ in range(300)]
    asked = ask(cases)
    assert sum(v is not None for v in asked[len(NAMED) * 42:]) > 200
    for (steps, a, b, c, shift), held in zip(cases, asked):
        if held is None:
            continue
        # logarithms: the most that a singular value of 2^-shift at the start may be, and what the smallest become of one
        most, least = -float(shift), -float(shift)
        for k in range(steps + 1):
            assert 14 + held[k] + most < 15.9, (steps, a, b, c, shift, k)
            if held[k]:
                assert held[k] + least >= -4.0, (steps, a, b, c, shift, k)
            part = np.linspace(0, 1, 2001)                # of the largest
            t = (part * 2.0 ** max(most, -500.0)) ** 2
            most += math.log2((part * np.abs(a + b * t + c * t ** 2)).max())
            least += math.log2(abs(a))


def test_polynomials_that_are_small_themselves_take_three_pieces(ask):
    """Q is held multiplied by 2^12: below 2^-4 of one it would keep fewer than 33 bits below its largest value."""
    assert ask([(5, 0.01, 0.0, 0.0, 0), (1, 1e-6, 1e-7, 0.0, 0), (1, 0.0, 0.0, 0.0, 0), (1, 0.0, 1.0, 0.0, 0)]) == [None] * 4


def test_the_largest_value_of_nearly_cubic_polynomials(ask):
    """A coefficient c that is nearly nothing beside b: where X is largest, between 0 and 1, is found all the same."""
    cases = [(1, sign * a, -sign * a, sign * c, 0) for a in (8.0, 11.0, 12.0) for sign in (1, -1) for c in (0.0, 1e-9, -1e-9, 1e-13, 1e-15, -1e-15, 1e-17, -1e-17, 1e-25, -1e-38)]
    for (steps, a, b, c, _), held in zip(cases, ask(cases)):
        s = np.linspace(0, 1, 20001)
        most = (s * np.abs(a + b * s ** 2 + c * s ** 4)).max()
        assert (held is None) == (most > 3), (a, b, c, most)
