"""Adapting a network's classifier to many tasks: one shared projection, a low-rank adapter per task.

A network's features (behind its average pooling) go through dropout and the classifier; the classifier's weights are shared and fixed, and each task learns a small
correction B A of them.  A step on a batch whose images belong to any of the tasks is

    forward     y = W x + b + B_a A_a drop(x)                      dr_adapter_fwd
    loss        softmax loss of the labels                         dr_softmax_loss_grad
    backward    to every task's A and B (and to x)                 dr_adapter_bwd
    descent     A and B along their gradients                      dr_sgd_step

every one of them a kernel of the library on the caller's stream, on buffers made once; a batch may have fewer rows than they were made for.  Parameters are fp32.
``python -m paper_1708_04728_amd.adapt`` learns adapters of a classifier of GoogLeNet's size (1024 features to 1000 classes, random weights) on synthetic features and
prints the loss.
"""
from __future__ import annotations

import math

import torch

from . import binding as B


class AdaptedClassifier:
    """The projection w (classes, c), bias with `tasks` adapters of rank `rank`, for batches of up to `rows` feature vectors (fp32); parameters a, b are device tensors."""

    def __init__(self, w, bias, tasks, rank, rows, p=0.0, seed=0, input_gradient=False, generator=None):
        classes, c = w.shape
        dev = w.device
        self.w, self.bias, self.rank = w, bias, rank
        self.a = torch.randn((tasks, rank, c), device=dev, generator=generator) * math.sqrt(1.0 / c)
        self.b = torch.zeros((tasks, classes, rank), device=dev)                 # an adapter starts as no correction
        self.da, self.db = torch.empty_like(self.a), torch.empty_like(self.b)
        self.y, self.inner = torch.empty((rows, classes), device=dev), torch.empty((rows, rank), device=dev)
        self.dx = torch.empty((rows, c), device=dev) if input_gradient else None
        self.loss, self.row_loss = torch.zeros(1, device=dev), torch.empty(rows, device=dev)
        self.draws = torch.zeros(1, dtype=torch.int64, device=dev)               # masks drawn so far: every step has its own, in a recorded graph too
        self.drop = B.dropout_desc(p, seed, 0, self.draws) if p else None
        x = torch.empty((rows, c), device=dev)
        need = max(B.adapter_fwd_workspace_bytes(x, self.a, self.b), B.adapter_bwd_workspace_bytes(x, self.a, self.b), B.softmax_loss_workspace_bytes(self.y), 256)
        self.ws = torch.empty(need, dtype=torch.uint8, device=dev)

    def forward(self, x, tasks, training=False, stream=None):
        """Logits of x (rows, c), each row through its task's adapter (a task outside 0 .. tasks - 1: the shared classifier alone); keeps what the gradient needs."""
        y, inner = self.y[:len(x)], self.inner[:len(x)]
        return B.adapter_fwd(x, self.w, self.bias, self.a, self.b, tasks, y, self.ws, drop=self.drop if training else None, inner=inner if training else None, stream=stream)

    def gradients(self, x, tasks, labels, smoothing=0.0, stream=None):
        """Forward with dropout, mean loss (self.loss) and the adapters' gradients; the logits are overwritten by theirs."""
        dy = self.forward(x, tasks, True, stream)
        B.softmax_loss_grad(dy, labels, dy, self.loss, self.ws, smoothing, row_loss=self.row_loss[:len(x)], stream=stream)
        B.adapter_bwd(dy, x, self.w, self.a, self.b, tasks, self.inner[:len(x)], None if self.dx is None else self.dx[:len(x)], self.da, self.db, self.ws, drop=self.drop,
                      stream=stream)

    def step(self, x, tasks, labels, lr, smoothing=0.0, stream=None):
        self.gradients(x, tasks, labels, smoothing, stream)
        B.sgd_step(self.a, self.da, lr, stream)
        B.sgd_step(self.b, self.db, lr, stream)
        if self.drop is not None:
            with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream()):
                self.draws.add_(1)


def main(batch=128, c=1024, classes=1000, tasks=4, rank=8, steps=100):
    """Learns what `tasks` corrections of a classifier do to its labels from features |N(0,1)|."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    normal = lambda *shape: torch.randn(shape, device="cuda", generator=gen)
    w, bias = normal(classes, c) * math.sqrt(2.0 / c), torch.zeros(classes, device="cuda")
    true = B.adapter_fwd_workspace_bytes(normal(batch, c), normal(tasks, rank, c), normal(tasks, classes, rank))
    a, b, ws = normal(tasks, rank, c) * math.sqrt(1.0 / c), normal(tasks, classes, rank), torch.empty(max(true, 256), dtype=torch.uint8, device="cuda")
    model = AdaptedClassifier(w, bias, tasks, rank, batch, p=0.4, seed=1, generator=gen)
    y = torch.empty((batch, classes), device="cuda")
    for i in range(steps):
        x = normal(batch, c).abs()
        ids = torch.randint(0, tasks, (batch,), device="cuda", generator=gen, dtype=torch.int32)
        labels = B.adapter_fwd(x, w, bias, a, b, ids, y, ws).argmax(1).int()
        model.step(x, ids, labels, 0.05)
        if i % 20 == 0 or i + 1 == steps:
            print("step %3d  loss %.4f" % (i, model.loss.item()))


if __name__ == "__main__":
    main()
