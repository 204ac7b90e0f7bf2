"""Which parameters a layer's dict has to hold, on the host."""
import numpy as np
import pytest

from paper_1708_04728_amd import graph as G


def vectors(*names):
    return {k: np.full(3, i, dtype=np.float32) for i, k in enumerate(names)}


def test_normalisations():
    bn, norm = vectors("gamma", "beta", "mean", "var"), vectors("gamma", "beta")
    assert [t[0].item() for t in G.flat_params([bn, norm], device="cpu")] == [0, 1, 2, 3, 0, 1]


@pytest.mark.parametrize("names", (("gamma", "beta", "mean"), ("gamma", "beta", "var"), ("gamma",), ("beta",), ("mean", "var"), ()))
def test_a_normalisation_lacks_a_vector(names):
    """The network would read the vectors of the layers behind it in its place, and past the list's end."""
    with pytest.raises(KeyError):
        G.flat_params([vectors(*names)], device="cpu")
