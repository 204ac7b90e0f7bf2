"""Which tensors the binding takes for layer normalisation and orthogonalised updates, on the host.  No GPU needed: tensors of the meta device have no memory."""
import pytest
import torch

from paper_1708_04728_amd import binding as B


@pytest.mark.parametrize("shape", ((8,), (2, 5, 8), (2, 8, 3, 3, 3), ()))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
def test_layernorm_takes_rows_and_maps(shape, dtype):
    """Over which dimension (batch, tokens, channels) would be normalised is not for the binding to guess."""
    t = torch.empty(shape, dtype=dtype, device="meta")
    with pytest.raises(ValueError, match="channels"):
        B.layernorm_fwd(t, None, None, 1e-5, False, t)
    with pytest.raises(ValueError, match="channels"):
        B.layernorm_bwd(t, t, None, None, None, t, None, None, None)
    with pytest.raises(ValueError, match="channels"):
        B.layernorm_bwd_workspace_bytes(t)


def test_layernorm_workspace_of_rows_and_maps():
    need = [B.layernorm_bwd_workspace_bytes(t) for t in (torch.empty(18, 8), torch.empty(18, 8, 1, 1), torch.empty(2, 8, 3, 3), B.NHWC(torch.empty(2, 3, 3, 8)))]
    assert need[0] > 0 and need == [need[0]] * 4


@pytest.mark.parametrize("shape", ((2 ** 32 + 2, 1), (1, 2 ** 32 + 8), (2 ** 32 + 2, 1, 1, 1), (1, 4, 2 ** 32 + 3, 1), (2 ** 16, 2 ** 15)))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
def test_sizes_beyond_31_bits(shape, dtype):
    """A dimension that passes 32 bits would reach the library as what is left of it, and most of the tensor be left out."""
    t = torch.empty(shape, dtype=dtype, device="meta")
    refused = pytest.raises((ValueError, B.DeepRebirthError), match="2\\^31-1 elements")
    with refused:
        B.layernorm_fwd(t, None, None, 1e-5, False, t)
    with refused:
        B.layernorm_bwd_workspace_bytes(t)
    with refused:
        B.orthogonalise_workspace_bytes([t])
    with refused:
        B.orthogonalise([torch.empty(3, 4, dtype=dtype, device="meta"), t], [torch.empty(3, 4, dtype=dtype, device="meta"), t], None)
    if dtype == torch.float32:
        with refused:
            B.muon_step_workspace_bytes(B.muon_params([(t, t, t)]))
