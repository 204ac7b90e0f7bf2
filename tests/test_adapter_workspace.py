"""What dr_adapter_*_workspace_bytes ask for, on the host: scratch that serves a batch serves every smaller one.  No GPU needed."""
import ctypes as C

import pytest

from paper_1708_04728_amd import binding as B


def need(size, rows, cin, cout, rank, count, dtype, hw=1):
    n = C.c_size_t(0)
    assert size(B.dr_tensor(rows, cin, 1, hw, dtype, B.DR_NHWC), B.dr_adapters(count, rank, cin, cout), n) == B.DR_OK
    return n.value


@pytest.mark.parametrize("dtype", [B.DR_F32, B.DR_BF16])
@pytest.mark.parametrize("cin,cout,rank,count,hw,most", [(1024, 1000, 8, 4, 1, 9000), (4096, 4096, 16, 8, 1, 4200), (72, 50, 4, 3, 1, 40000), (528, 256, 12, 5, 195, 400), (7, 9, 1, 0, 1, 40000),
                                                         (64, 40000, 3, 2, 1, 1000)])
def test_a_larger_batch_asks_for_no_less(cin, cout, rank, count, hw, most, dtype):
    L = B.lib()
    for size in (L.dr_adapter_fwd_workspace_bytes, L.dr_adapter_bwd_workspace_bytes):
        asked = [need(size, rows, cin, cout, rank, count, dtype, hw) for rows in range(most)]
        assert [i for i in range(1, most) if asked[i] < asked[i - 1]] == []


def test_channels_beyond_a_launch_are_refused():
    L = B.lib()
    n = C.c_size_t(0)
    for size in (L.dr_adapter_fwd_workspace_bytes, L.dr_adapter_bwd_workspace_bytes):
        for cin, cout in ((1, 1 << 30), (1 << 30, 1), (1, (1 << 29) + 1)):
            assert size(B.dr_tensor(1, cin, 1, 1, B.DR_F32, B.DR_NHWC), B.dr_adapters(0, 1, cin, cout), n) == B.DR_ERR_UNSUPPORTED and "2^29" in B.last_error()
        assert size(B.dr_tensor(1, 1, 1, 1, B.DR_F32, B.DR_NHWC), B.dr_adapters(0, 1, 1, 1 << 29), n) == B.DR_OK
