"""Which kernels the sizes of tests/test_gpu_orthogonal_paths.py reach (csrc/orthogonal_plan.h, compiled for the host): a single matrix and a list have kernels of their own, and so
have results and descent steps, either number of pieces and the two kinds of product.  Every test there runs all of its sizes in all of these."""
from test_orthogonal_plan import ask, check        # noqa: F401 (a fixture)


def test_every_kernel_is_compared(ask):        # noqa: F811
    from test_gpu_orthogonal_paths import LISTS, SINGLES
    for what, lists in (("single", [[s] for s in SINGLES]), ("list", list(LISTS.values()))):
        for pieces in (2, 3):
            # (a list runs up to 64 of its matrices at a time, without the empty ones)
            cases = [(256, pieces, part) for s in lists for full in ([v for v in s if min(v)],) for part in (full[i:i + 64] for i in range(0, len(full), 64))]
            symmetric, other, shared, whole, together = set(), set(), set(), False, False
            for case, plan in zip(cases, ask(cases)):
                joined, products = check(case, plan)
                whole, together = whole or bool(plan[0]), together or bool(joined)
                if plan[0]:
                    continue
                symmetric.add(products[0])
                if products[1] > 1:
                    shared.add(products[0])
                if not joined:
                    symmetric.add(products[4])
                    other.add(products[8])
            print(what, pieces, symmetric, other, shared, whole, together)
            assert symmetric == set(range(5)) and other == set(range(5)) and shared == {0, 1} and together, (what, pieces)
            assert whole == (what == "list"), what      # (single ones: tests/test_gpu_orthogonal.py)
