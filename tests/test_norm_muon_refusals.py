"""What dr_layernorm_*, dr_orthogonalise and dr_muon_step refuse, on the host, before anything is launched.  No GPU needed."""
import ctypes as C

import pytest
import torch

from paper_1708_04728_amd import binding as B

FAKE = C.c_void_p(4096)      # never dereferenced


def tensor(n, c, h, w, dtype=B.DR_F32, layout=B.DR_NCHW):
    return B.dr_tensor(n, c, h, w, dtype, layout)


def test_layernorm_refuses():
    L = B.lib()
    d = tensor(2, 8, 3, 3)
    fwd = lambda d=d, x=FAKE, eps=1e-5, y=FAKE: L.dr_layernorm_fwd(d, x, None, None, eps, 0, y, None, None, None)
    assert fwd(d=None) == B.DR_ERR_NULL
    assert fwd(x=None) == B.DR_ERR_NULL and fwd(y=None) == B.DR_ERR_NULL
    assert fwd(eps=-1.0) == B.DR_ERR_SHAPE and fwd(eps=float("nan")) == B.DR_ERR_SHAPE and "eps" in B.last_error()
    assert fwd(d=tensor(2, 8, -1, 3)) == B.DR_ERR_SHAPE
    assert fwd(d=tensor(2, 8, 3, 3, 7)) == B.DR_ERR_UNSUPPORTED and fwd(d=tensor(2, 8, 3, 3, 0, 5)) == B.DR_ERR_UNSUPPORTED
    assert fwd(d=tensor(1 << 11, 1 << 10, 1 << 5, 1 << 5)) == B.DR_ERR_UNSUPPORTED
    assert fwd(d=tensor(0, 8, 3, 3), x=None, y=None) == B.DR_OK
    need = C.c_size_t(0)
    assert L.dr_layernorm_bwd_workspace_bytes(d, None) == B.DR_ERR_NULL
    assert L.dr_layernorm_bwd_workspace_bytes(d, need) == B.DR_OK and need.value > 0
    bwd = lambda dy=FAKE, x=FAKE, mean=FAKE, rstd=FAKE, dx=C.c_void_p(8192), dgamma=FAKE, ws=FAKE, n=need.value: \
        L.dr_layernorm_bwd(d, dy, x, None, mean, rstd, dx, dgamma, None, ws, n, None)
    for name in ("dy", "x", "mean", "rstd"):
        assert bwd(**{name: None}) == B.DR_ERR_NULL, name
    assert bwd(ws=None) == B.DR_ERR_WORKSPACE and bwd(n=need.value - 1) == B.DR_ERR_WORKSPACE and bwd(ws=C.c_void_p(4096 + 16)) == B.DR_ERR_WORKSPACE
    assert bwd(dx=FAKE) == B.DR_ERR_UNSUPPORTED and "dx" in B.last_error()


def test_orthogonalise_refuses():
    L = B.lib()
    ms = (B.dr_matrix * 2)((3, 5), (7, 2))
    ptrs = (C.c_void_p * 2)(4096, 8192)
    need = C.c_size_t(0)
    assert L.dr_orthogonalise_workspace_bytes(2, ms, B.DR_F32, None) == B.DR_ERR_NULL
    assert L.dr_orthogonalise_workspace_bytes(2, ms, B.DR_F32, need) == B.DR_OK and need.value > 0
    ns = lambda steps=5, eps=1e-7: B.dr_newton_schulz(steps, *B.NEWTON_SCHULZ, eps)
    call = lambda count=2, ms=ms, dtype=B.DR_F32, g=ptrs, o=ptrs, p=ns(), ws=FAKE, n=need.value: L.dr_orthogonalise(count, ms, dtype, g, o, p, ws, n, None)
    assert call(count=-1) == B.DR_ERR_SHAPE and call(ms=None) == B.DR_ERR_NULL and call(dtype=3) == B.DR_ERR_UNSUPPORTED
    assert call(g=None) == B.DR_ERR_NULL and call(o=None) == B.DR_ERR_NULL and call(p=None) == B.DR_ERR_NULL
    assert call(g=(C.c_void_p * 2)(4096, None)) == B.DR_ERR_NULL and "g[1]" in B.last_error()
    assert call(p=ns(steps=0)) == B.DR_ERR_SHAPE and call(p=ns(steps=65)) == B.DR_ERR_SHAPE and call(p=ns(eps=-1.0)) == B.DR_ERR_SHAPE
    assert call(ms=(B.dr_matrix * 2)((3, 5), (-7, 2))) == B.DR_ERR_SHAPE
    assert call(ms=(B.dr_matrix * 2)((3, 5), (65536, 65536))) == B.DR_ERR_UNSUPPORTED
    assert call(ws=None) == B.DR_ERR_WORKSPACE and call(n=need.value - 1) == B.DR_ERR_WORKSPACE and call(ws=C.c_void_p(4096 + 8)) == B.DR_ERR_WORKSPACE
    assert call(count=0, ms=None, g=None, o=None, ws=None, n=0) == B.DR_OK
    empty = (B.dr_matrix * 2)((0, 5), (7, 0))
    assert L.dr_orthogonalise_workspace_bytes(2, empty, B.DR_F32, need) == B.DR_OK
    assert call(ms=empty, g=(C.c_void_p * 2)(None, None), o=(C.c_void_p * 2)(None, None), n=need.value) == B.DR_OK


def test_muon_step_refuses():
    L = B.lib()
    ps = (B.dr_muon_param * 1)((3, 5, 4096, 8192, 12288))
    need = C.c_size_t(0)
    assert L.dr_muon_step_workspace_bytes(1, ps, need) == B.DR_OK
    opt = lambda steps=5, eps=1e-7: B.dr_muon(0.02, 0.95, 0.0, B.dr_newton_schulz(steps, *B.NEWTON_SCHULZ, eps))
    call = lambda count=1, ps=ps, o=opt(), ws=FAKE, n=need.value: L.dr_muon_step(count, ps, o, ws, n, None)
    assert call(count=-1) == B.DR_ERR_SHAPE and call(ps=None) == B.DR_ERR_NULL and call(o=None) == B.DR_ERR_NULL
    assert call(o=opt(steps=0)) == B.DR_ERR_SHAPE and call(o=opt(eps=-1.0)) == B.DR_ERR_SHAPE
    for bad in ((3, 5, None, 8192, 12288), (3, 5, 4096, None, 12288), (3, 5, 4096, 8192, None)):
        assert call(ps=(B.dr_muon_param * 1)(bad)) == B.DR_ERR_NULL
    assert call(ps=(B.dr_muon_param * 1)((-3, 5, 4096, 8192, 12288))) == B.DR_ERR_SHAPE
    assert call(ps=(B.dr_muon_param * 1)((65536, 32768, 4096, 8192, 12288))) == B.DR_ERR_UNSUPPORTED
    assert call(ws=None) == B.DR_ERR_WORKSPACE and call(n=need.value - 1) == B.DR_ERR_WORKSPACE
    assert call(count=0, ps=None, ws=None, n=0) == B.DR_OK


def test_binding_refuses():
    t = torch.zeros(2, 4, 3, 3)
    with pytest.raises(ValueError):
        B.layernorm_fwd(t, None, None, 1e-5, False, torch.zeros(2, 4, 3, 2))
    with pytest.raises(ValueError):
        B.layernorm_fwd(t, None, None, 1e-5, False, B.NHWC(t))
    with pytest.raises(TypeError):
        B.layernorm_fwd(t, torch.zeros(4, dtype=torch.float64), None, 1e-5, False, t)
    for vectors in ((torch.zeros(3), None), (None, torch.zeros(5)), (torch.zeros(8)[::2], None)):
        with pytest.raises(ValueError):
            B.layernorm_fwd(t, *vectors, 1e-5, False, t)
    pixels = torch.zeros(2, 3, 3)
    for mean, rstd in ((pixels, torch.zeros(17)), (torch.zeros(19), pixels)):
        with pytest.raises(ValueError):
            B.layernorm_fwd(t, None, None, 1e-5, False, t, mean, rstd)
        with pytest.raises(ValueError):
            B.layernorm_bwd(t, t, None, mean, rstd, t.clone(), None, None, None)
    with pytest.raises(ValueError):
        B.layernorm_bwd(t, t, None, pixels, pixels, t.clone(), torch.zeros(5), None, None)
    with pytest.raises(ValueError):
        B.orthogonalise([torch.zeros(3, 4)], [torch.zeros(4, 3)], None)
    with pytest.raises(TypeError):
        B.orthogonalise([torch.zeros(3, 4), torch.zeros(3, 4, dtype=torch.bfloat16)], [], None)
    with pytest.raises(ValueError):
        B.orthogonalise_workspace_bytes([torch.zeros(3)])
    with pytest.raises(ValueError):
        B.orthogonalise_workspace_bytes([torch.zeros(4, 3).t()])
    with pytest.raises(TypeError):
        B.muon_params([(torch.zeros(3, 4), torch.zeros(3, 4, dtype=torch.bfloat16), torch.zeros(3, 4))])
    with pytest.raises(ValueError):
        B.muon_params([(torch.zeros(3, 4), torch.zeros(4, 3), torch.zeros(3, 4))])


def test_networks_with_a_layer_normalisation():
    from paper_1708_04728_amd import graph as G
    layers = [("conv", {"k": 6, "r": 3, "s": 3, "stride": 1, "pad": 1}), ("layernorm", {"eps": 1e-5}), ("relu", {}), ("maxpool", {"k": 3, "stride": 2, "pad": 0})]
    net, fused = B.Net(G.net_descs(layers, 4)), B.Net(G.net_descs(layers, 4, fuse_relu=True))
    assert net.n_layers == 4 and fused.n_layers == 3 and net.num_params() == fused.num_params() == 4
    d = net.output_desc(tensor(2, 4, 9, 9))
    assert (d.n, d.c, d.h, d.w) == (2, 6, 4, 4)
    bad = B.Net(G.net_descs([("layernorm", {"eps": -1.0})], 4))
    with pytest.raises(B.DeepRebirthError):
        bad.output_desc(tensor(2, 4, 9, 9))
