"""Learning a slim layer that keeps a normalisation: convolution, layer normalisation over the channels, ReLU.

Streamline slimming (Sec. 3.1) drops the block's LRN; the slim layer is then learned by regression on the block's output.  Here the layer keeps a normalisation
with learned weights in the place of the dropped one.  A step is

    forward     z = conv(x; w, b),  f = max(layernorm(z; gamma, beta), 0)
    loss        sum (f - y)^2                                      dr_regression_loss_grad
    backward    through the normalisation to z, gamma and beta     dr_layernorm_bwd
                through the convolution to w and b                 dr_conv2d_bwd_params
    descent     w on orthogonalised momentum                       dr_muon_step
                b, gamma, beta along their gradients               dr_sgd_step

every one of them a kernel of the library on the caller's stream, on buffers made once.  ``python -m paper_1708_04728_amd.fit`` learns the replacement of a
conv - ReLU - LRN - max-pool block on synthetic data and prints the loss.
"""
from __future__ import annotations

import math

import torch

from . import binding as B


class NormalisedSlimLayer:
    """k filters of r x r at `stride` on inputs shaped like x (fp32, NCHW), with what a step needs; parameters w, b, gamma, beta are device tensors."""

    def __init__(self, x, k, r, stride, pad, eps=1e-5, generator=None):
        n, c, h, w = x.shape
        dev = x.device
        self.eps = eps
        self.conv = B.conv_desc(k, c, r, r, stride, pad, False, B.DR_KCRS)
        p, q = B.conv_out_size(h, r, stride, pad), B.conv_out_size(w, r, stride, pad)
        self.w = torch.randn((k, c, r, r), device=dev, generator=generator) * math.sqrt(2.0 / (c * r * r))
        self.b, self.gamma, self.beta = torch.zeros(k, device=dev), torch.ones(k, device=dev), torch.zeros(k, device=dev)
        self.z, self.f = (torch.empty((n, k, p, q), device=dev) for _ in range(2))
        self.mean, self.rstd = (torch.empty((n, p, q), device=dev) for _ in range(2))
        self.dw, self.db, self.dgamma, self.dbeta = (torch.empty_like(t) for t in (self.w, self.b, self.gamma, self.beta))
        self.momentum = torch.zeros_like(self.w)
        self.loss = torch.zeros(1, device=dev)
        self.params = B.muon_params([(self.w, self.dw, self.momentum)])
        need = max(B.conv2d_workspace_bytes(x, self.conv), B.regression_loss_workspace_bytes(), B.layernorm_bwd_workspace_bytes(self.z),
                   B.conv2d_bwd_params_workspace_bytes(x, self.conv), B.muon_step_workspace_bytes(self.params), 256)
        self.ws = torch.empty(need, dtype=torch.uint8, device=dev)

    def forward(self, x, stream=None):
        """f for input x; keeps what the gradients need."""
        B.conv2d_fwd_ws(x, self.conv, self.w, self.b, self.z, self.ws, stream=stream)
        return B.layernorm_fwd(self.z, self.gamma, self.beta, self.eps, True, self.f, self.mean, self.rstd, stream=stream)

    def gradients(self, x, y, stream=None):
        """Forward, loss (self.loss) and the parameters' gradients for target y; f is overwritten."""
        f = self.forward(x, stream)
        B.regression_loss_grad(f, y, f, self.loss, self.ws, stream)
        B.layernorm_bwd(f, self.z, self.gamma, self.mean, self.rstd, f, self.dgamma, self.dbeta, self.ws, stream)
        B.conv2d_bwd_params(x, self.conv, f, self.dw, self.db, self.ws, stream)

    def step(self, x, y, lr, lr_vectors, momentum=0.95, weight_decay=0.0, stream=None):
        """One step: filters by lr on orthogonalised momentum, vectors by lr_vectors along their gradients."""
        self.gradients(x, y, stream)
        B.muon_step(self.params, self.ws, lr, momentum, weight_decay, stream=stream)
        for v, dv in ((self.b, self.db), (self.gamma, self.dgamma), (self.beta, self.dbeta)):
            B.sgd_step(v, dv, lr_vectors, stream)


def main(batch=16, c=64, k=192, size=56, steps=60):
    """Learns what replaces conv 3x3 - ReLU - LRN - max-pool 3x3/2 (the second block of GoogLeNet) from |N(0,1)| inputs."""
    from . import graph as G
    gen = torch.Generator(device="cuda").manual_seed(1)
    layers = [("conv", {"k": k, "r": 3, "s": 3, "stride": 1, "pad": 1}), ("relu", {}), ("lrn", {"n": 5, "alpha": 1e-4, "beta": 0.75, "k": 1.0}),
              ("maxpool", {"k": 3, "stride": 2, "pad": 0})]
    net = B.Net(G.net_descs(layers, c))
    x = torch.randn((batch, c, size, size), device="cuda", generator=gen).abs()
    y = G.empty_like_desc(net.output_desc(B.desc(x)))
    ws = torch.empty(max(net.workspace_bytes(B.desc(x)), 256), dtype=torch.uint8, device="cuda")
    net.fwd(x, [torch.randn((k, c, 3, 3), device="cuda", generator=gen) * math.sqrt(2.0 / (c * 9)), torch.zeros(k, device="cuda")], y, ws)
    layer = NormalisedSlimLayer(x, k, 3, 2, 1, generator=gen)
    pixels = y.shape[0] * y.shape[2] * y.shape[3]
    for i in range(steps):
        layer.step(x, y, 0.02 * (1 - i / steps), 0.1 / pixels)
        if i % 10 == 0 or i + 1 == steps:
            print("step %3d  loss per output %.4f" % (i, layer.loss.item() / y.numel()))


if __name__ == "__main__":
    main()
