"""What dr_dropout_fwd, dr_softmax_loss_* and dr_adapter_* refuse, on the host, before anything is launched.  No GPU needed."""
import ctypes as C

import pytest
import torch

from paper_1708_04728_amd import binding as B

FAKE, OTHER = C.c_void_p(4096), C.c_void_p(1 << 20)      # never dereferenced


def tensor(n, c, h=1, w=1, dtype=B.DR_F32, layout=B.DR_NHWC):
    return B.dr_tensor(n, c, h, w, dtype, layout)


def test_dropout_refuses():
    L = B.lib()
    drop = lambda p=0.5: B.dr_dropout(p, 1, 2, None)
    call = lambda d=tensor(2, 8, 3, 3), x=FAKE, p=drop(), y=FAKE: L.dr_dropout_fwd(d, x, p, y, None)
    assert call(d=None) == B.DR_ERR_NULL and call(x=None) == B.DR_ERR_NULL and call(y=None) == B.DR_ERR_NULL and call(p=None) == B.DR_ERR_NULL
    for p in (-0.1, 1.1, float("nan"), float("inf")):
        assert call(p=drop(p)) == B.DR_ERR_SHAPE and "probability" in B.last_error()
    assert call(d=tensor(2, -8)) == B.DR_ERR_SHAPE and call(d=tensor(2, 8, dtype=5)) == B.DR_ERR_UNSUPPORTED
    assert call(d=tensor(1 << 16, 1 << 15)) == B.DR_ERR_UNSUPPORTED
    assert call(d=tensor(0, 8), x=None, y=None) == B.DR_OK


def test_softmax_loss_refuses():
    L = B.lib()
    need = C.c_size_t(0)
    assert L.dr_softmax_loss_workspace_bytes(tensor(5, 7), None) == B.DR_ERR_NULL
    assert L.dr_softmax_loss_workspace_bytes(tensor(5, 7), need) == B.DR_OK and need.value >= 20
    call = lambda d=tensor(5, 7), z=FAKE, labels=FAKE, e=0.0, ws=FAKE, n=need.value: L.dr_softmax_loss_grad(d, z, labels, e, 1, FAKE, FAKE, FAKE, ws, n, None)
    assert call(d=None) == B.DR_ERR_NULL and call(z=None) == B.DR_ERR_NULL and call(labels=None) == B.DR_ERR_NULL
    assert call(d=tensor(5, 7, 1, 2)) == B.DR_ERR_SHAPE and call(d=tensor(5, 0)) == B.DR_ERR_SHAPE and call(d=tensor(5, 7, dtype=9)) == B.DR_ERR_UNSUPPORTED
    assert call(d=tensor((1 << 30) + 1, 1)) == B.DR_ERR_UNSUPPORTED and call(d=tensor(1, (1 << 30) + 1)) == B.DR_ERR_UNSUPPORTED
    for e in (-0.1, 1.5, float("nan")):
        assert call(e=e) == B.DR_ERR_SHAPE and "smoothing" in B.last_error()
    assert call(ws=None) == B.DR_ERR_WORKSPACE and call(n=need.value - 1) == B.DR_ERR_WORKSPACE and call(ws=C.c_void_p(4096 + 16)) == B.DR_ERR_WORKSPACE


def test_adapters_refuse():
    L = B.lib()
    xd, yd, ad = tensor(3, 8, 2, 2), tensor(3, 5, 2, 2), B.dr_adapters(2, 4, 8, 5)
    need = C.c_size_t(0)
    for size in (L.dr_adapter_fwd_workspace_bytes, L.dr_adapter_bwd_workspace_bytes):
        assert size(xd, ad, None) == B.DR_ERR_NULL and size(xd, None, need) == B.DR_ERR_NULL and size(None, ad, need) == B.DR_ERR_NULL
        for bad in (B.dr_adapters(2, 0, 8, 5), B.dr_adapters(2, 129, 8, 5), B.dr_adapters(-1, 4, 8, 5), B.dr_adapters(16385, 4, 8, 5)):
            assert size(xd, bad, need) == B.DR_ERR_UNSUPPORTED
        for bad in (B.dr_adapters(2, 4, 7, 5), B.dr_adapters(2, 4, 8, 0), B.dr_adapters(2, 4, 0, 5)):
            assert size(xd, bad, need) == B.DR_ERR_SHAPE
        assert size(tensor(3, 8, 2, 2, layout=B.DR_NCHW), ad, need) == B.DR_ERR_UNSUPPORTED and "channels-last" in B.last_error()
        assert size(tensor(3, 8, layout=B.DR_NCHW), ad, need) == B.DR_OK
        assert size(tensor(1 << 20, 8), B.dr_adapters(2, 4, 8, 1 << 12), need) == B.DR_ERR_UNSUPPORTED
        assert size(tensor(3, 1 << 16), B.dr_adapters(2, 4, 1 << 16, 1 << 15), need) == B.DR_ERR_UNSUPPORTED
        assert size(tensor(3, 1 << 12), B.dr_adapters(1 << 13, 64, 1 << 12, 8), need) == B.DR_ERR_UNSUPPORTED
        assert size(tensor((1 << 26) + 1, 8), B.dr_adapters(2, 4, 8, 8), need) == B.DR_ERR_UNSUPPORTED and size(tensor(1 << 26, 8), B.dr_adapters(2, 4, 8, 8), need) == B.DR_OK
        assert size(tensor(1, 1 << 17), B.dr_adapters(1 << 12, 1, 1 << 17, 8), need) == B.DR_ERR_UNSUPPORTED
        assert size(tensor(0, 8, 1 << 20, 1 << 20), ad, need) == B.DR_OK                  # (no pixels, whatever the map)
    assert L.dr_adapter_fwd_workspace_bytes(xd, ad, need) == B.DR_OK and need.value > 0
    names = ("x", "w", "a", "b", "ids", "y")
    def fwd(xd=xd, ad=ad, yd=yd, drop=None, ws=FAKE, n=need.value, **p):
        x, w, a, b, ids = (p.get(k, FAKE) for k in names[:5])
        return L.dr_adapter_fwd(xd, x, ad, w, None, a, b, None, ids, drop, yd, p.get("y", OTHER), None, ws, n, None)
    for k in names:
        assert fwd(**{k: None}) == B.DR_ERR_NULL, k
    assert fwd(y=FAKE) == B.DR_ERR_UNSUPPORTED
    assert fwd(yd=None) == B.DR_ERR_NULL and fwd(yd=tensor(3, 6, 2, 2)) == B.DR_ERR_SHAPE and fwd(yd=tensor(3, 5, 4, 1)) == B.DR_ERR_SHAPE
    assert fwd(yd=tensor(3, 5, 2, 2, B.DR_BF16)) == B.DR_ERR_UNSUPPORTED and fwd(yd=tensor(3, 5, 2, 2, layout=B.DR_NCHW)) == B.DR_ERR_UNSUPPORTED
    assert fwd(drop=B.dr_dropout(2.0, 0, 0, None)) == B.DR_ERR_SHAPE
    assert fwd(ws=None) == B.DR_ERR_WORKSPACE and fwd(n=need.value - 1) == B.DR_ERR_WORKSPACE and fwd(ws=C.c_void_p(4096 + 8)) == B.DR_ERR_WORKSPACE
    assert fwd(xd=tensor(0, 8, 2, 2), yd=tensor(0, 5, 2, 2), x=None, y=None) == B.DR_OK
    assert L.dr_adapter_bwd_workspace_bytes(xd, ad, need) == B.DR_OK and need.value > 0
    def bwd(dx=OTHER, da=OTHER, db=OTHER, drop=None, ws=FAKE, n=need.value, **p):
        dy, x, w, a, b, ids, inner = (p.get(k, FAKE) for k in ("dy", "x", "w", "a", "b", "ids", "inner"))
        return L.dr_adapter_bwd(yd, dy, xd, x, ad, w, a, b, None, ids, drop, inner, dx, da, db, ws, n, None)
    for k in ("dy", "x", "w", "a", "b", "ids", "inner"):
        assert bwd(**{k: None}) == B.DR_ERR_NULL, k
    assert bwd(dx=FAKE) == B.DR_ERR_UNSUPPORTED and bwd(drop=B.dr_dropout(float("nan"), 0, 0, None)) == B.DR_ERR_SHAPE
    assert bwd(ws=None) == B.DR_ERR_WORKSPACE and bwd(n=need.value - 1) == B.DR_ERR_WORKSPACE


def test_binding_refuses():
    x, w, a, b = torch.zeros(3, 8), torch.zeros(5, 8), torch.zeros(2, 4, 8), torch.zeros(2, 5, 4)
    ids, y, ws = torch.zeros(3, dtype=torch.int32), torch.zeros(3, 5), torch.zeros(1 << 16, dtype=torch.uint8)
    fwd = lambda x=x, w=w, bias=None, a=a, b=b, ids=ids, y=y, **k: B.adapter_fwd(x, w, bias, a, b, ids, y, ws, **k)
    for bad in (dict(x=x.bfloat16()), dict(a=a.bfloat16()), dict(a=torch.zeros(2, 4, 8, dtype=torch.float16), b=b.half(), x=x.half())):
        with pytest.raises(TypeError):
            fwd(**bad)
    for bad in (dict(x=torch.zeros(3, 8, 1, 1)), dict(x=torch.zeros(8, 3).t()), dict(w=torch.zeros(8, 5)), dict(w=None), dict(w=w.bfloat16()), dict(b=torch.zeros(2, 5, 3)),
                dict(a=torch.zeros(3, 4, 8)), dict(y=torch.zeros(3, 6)), dict(y=B.NHWC(torch.zeros(3, 1, 1, 5))), dict(y=torch.zeros(5, 3).t()), dict(bias=torch.zeros(4)),
                dict(bias=torch.zeros(5, dtype=torch.float64)), dict(scales=torch.zeros(3)), dict(inner=torch.zeros(3, 5))):
        with pytest.raises(ValueError):
            fwd(**bad)
    with pytest.raises(ValueError, match="device"):
        fwd()                                                          # tensors of the host
    z, labels = torch.zeros(3, 5), torch.zeros(3, dtype=torch.int32)
    for bad in (dict(z=torch.zeros(3, 5, 1)), dict(dz=torch.zeros(5, 3)), dict(dz=z.bfloat16()), dict(loss=torch.zeros(2)), dict(row_loss=torch.zeros(4)), dict(z=z.t())):
        with pytest.raises(ValueError):
            B.softmax_loss_grad(**{**dict(z=z, labels=labels, dz=None, loss=None, ws=ws), **bad})
    with pytest.raises(ValueError, match="device"):
        B.softmax_loss_grad(z, labels, None, None, ws)
    with pytest.raises(TypeError):
        B._ints(labels.long(), 3, "labels")
    with pytest.raises(ValueError):
        B._ints(labels, 4, "labels")
    drop = B.dropout_desc(0.5, 1)
    for x, y in ((z, z.bfloat16()), (z, torch.zeros(5, 3)), (z, B.NHWC(torch.zeros(3, 1, 1, 5))), (z.t(), z.t()), (z, z)):
        with pytest.raises(ValueError):
            B.dropout_fwd(x, drop, y)
    for bad in (dict(seed=-1), dict(seed=2 ** 64), dict(offset=2 ** 64), dict(step=torch.zeros(1, dtype=torch.int64)), dict(step=torch.zeros(2))):
        with pytest.raises(ValueError):
            B.dropout_desc(**{**dict(p=0.5, seed=1), **bad})
