"""The definitions that the adapter, dropout and loss kernels are compared with: the generator against its published answers and the host's build of the kernels' own
lines, the gradients against differences.  No GPU needed."""
import os
import subprocess

import numpy as np
import pytest

import adapt_oracle as O

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1708_04728_amd", "csrc")


def test_published_answers():
    # the test vectors published with the generator: counter and key of zeros, and of ones
    assert O.philox(0, 0, 0) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert O.philox(2 ** 64 - 1, 2 ** 64 - 1, 2 ** 64 - 1) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


def test_draws_are_the_words_halves():
    d = O.draws(37, 0x123456789ABCDEF0, 2 ** 33 + 5)
    for i in range(37):
        word = O.philox(0x123456789ABCDEF0, i // 8, 2 ** 33 + 5)[i % 8 // 2]
        assert d[i] == (word >> 16 if i % 2 else word & 0xFFFF)


PROGRAM = r"""
#include <cstdio>
#include <initializer_list>
#include "philox.h"
int main()
{
    unsigned long long seed, block, place;
    while (scanf("%llu %llu %llu", &seed, &block, &place) == 3) {
        uint32_t r[4];
        dr::philox(seed, block, place, r);
        printf("%u %u %u %u", r[0], r[1], r[2], r[3]);
        for (int j = 0; j < 8; ++j) printf(" %u", dr::drop_draw(r, j));
        printf("\n");
    }
    for (float p : {0.f, 1e-6f, 0.1f, 0.4f, 0.5f, 0.999999f, 1.f}) printf("%u %.9g\n", dr::drop_border(p), dr::drop_scale(dr::drop_border(p)));
}
"""


def test_kernels_own_lines(tmp_path):
    src = tmp_path / "philox.cpp"
    src.write_text(PROGRAM)
    exe = str(tmp_path / "philox")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-I", CSRC, str(src), "-o", exe])
    asked = [(0, 0, 0), (2 ** 64 - 1, 2 ** 64 - 1, 2 ** 64 - 1), (0x9E37, 123456789, 7), (2 ** 63 + 11, 2 ** 32 + 3, 2 ** 40)]
    out = subprocess.run([exe], input="\n".join("%d %d %d" % q for q in asked), capture_output=True, text=True, check=True).stdout.split("\n")
    for q, line in zip(asked, out):
        got = [int(v) for v in line.split()]
        words = O.philox(*q)
        assert got[:4] == words and got[4:] == [h for v in words for h in (v & 0xFFFF, v >> 16)]
    for p, line in zip((0.0, 1e-6, 0.1, 0.4, 0.5, 0.999999, 1.0), out[len(asked):]):
        t, scale = line.split()
        assert int(t) == O.border(p)
        assert np.float32(scale) == (0 if int(t) == 65536 else np.float32(65536.0 / (65536 - int(t))))


def differences(f, v, d=1e-6):
    g = np.zeros(v.shape)
    for i in np.ndindex(v.shape):
        at = v[i]
        v[i] = at + d
        up = f()
        v[i] = at - d
        g[i] = (up - f()) / (2 * d)
        v[i] = at
    return g


@pytest.mark.parametrize("p", [0.0, 0.4])
def test_adapter_gradient_against_differences(p):
    rng = np.random.default_rng(1)
    x, w, bias = rng.standard_normal((7, 5)), rng.standard_normal((4, 5)), rng.standard_normal(4)
    a, b, scales = rng.standard_normal((3, 2, 5)), rng.standard_normal((3, 4, 2)), rng.uniform(0.5, 2, 3)
    ids, m, dy = [0, 2, -1, 2, 0, 7, 2], O.mask((7, 5), p, 3, 4), rng.standard_normal((7, 4))
    value = lambda: (O.adapter_fwd(x, w, bias, a, b, ids, scales, m)[0] * dy).sum()
    inner = O.adapter_fwd(x, w, bias, a, b, ids, scales, m)[1]
    for got, v in zip(O.adapter_bwd(dy, x, w, a, b, ids, scales, m, inner), (x, a, b)):
        # a central difference of a polynomial of degree 2 in each variable: exact but for roundings, 1e-16 / 1e-6 of values below 100
        assert np.abs(got - differences(value, v)).max() < 1e-7


@pytest.mark.parametrize("smoothing,mean", [(0.0, True), (0.1, True), (0.3, False), (1.0, True)])
def test_loss_gradient_against_differences(smoothing, mean):
    rng = np.random.default_rng(2)
    z, labels = rng.standard_normal((6, 5)), [0, 4, -1, 2, 5, 2]
    dz = O.softmax_loss(z, labels, smoothing, mean)[2]
    # third derivatives of a log-sum-exp are below 1: the difference is off by 1e-12 / 6, roundings add 1e-16 / 1e-6 of values below 20
    assert np.abs(dz - differences(lambda: O.softmax_loss(z, labels, smoothing, mean)[0], z)).max() < 1e-8
