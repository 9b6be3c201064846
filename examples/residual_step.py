"""A training step of a residual block between features and a classifier, on the library's calls: a norm, a widening dense layer with
GELU and dropout, a narrowing one, the block's norm, gate, dropout and residual with the norm before the classifier, a linear classifier whose logits
are never kept, and the matrices updated by orthogonalised gradients.

    python examples/residual_step.py [steps]

What is kept for the backward pass are the block's input, the matrices' inputs and the two sums: no mask, no pre-activation, no
normalised row.  The step's number lies on the device, so that a captured step draws another mask each time it is replayed.  Device memory is torch's.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2409_11902_amd import binding as B  # noqa: E402

DEV = "cuda:0"
TYPES = {B.F32: torch.float32, B.BF16: torch.bfloat16}


class Block:
    """Weights, descriptors and buffers; step() is one pass forward, backward and update."""

    def __init__(self, rows=256, width=192, hidden=512, classes=100, p=0.1, alpha=0.5, dtype=B.BF16, seed=0):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.gen, self.shape, self.dtype, td = g, (rows, width, hidden, classes), dtype, TYPES[dtype]

        def normal(*shape, std, kind=td):
            return (torch.randn(*shape, generator=g, device=DEV) * std).to(kind)

        def new(*shape, kind=td):
            return torch.empty(*shape, dtype=kind, device=DEV)

        self.w = {"wide": normal(hidden, width, std=width ** -0.5), "wide_b": normal(hidden, std=0.02),
                  "narrow": normal(width, hidden, std=hidden ** -0.5), "narrow_b": normal(width, std=0.02),
                  "head": normal(classes, width, std=0.05), "in": torch.ones(width, device=DEV), "gate": torch.full((1, width), 0.5, device=DEV),
                  "post": torch.ones(width, device=DEV), "pre": torch.ones(width, device=DEV), "pre_b": torch.zeros(width, device=DEV)}
        self.grad = {k: torch.empty_like(v) for k, v in self.w.items()}
        self.rng = torch.tensor([seed, 0], dtype=torch.int64, device=DEV)
        # every place that drops has a number of its own
        self.first = B.make_block_norm_desc(rows, width, dtype=dtype, post=B.NORM_NONE, pre=B.NORM_RMS)
        self.wide = B.make_linear_desc(rows, width, hidden, dtype=dtype, has_bias=1, act=B.ACT_GELU, p=p, site=1)
        self.narrow = B.make_linear_desc(rows, hidden, width, dtype=dtype, has_bias=1)
        self.join = B.make_block_norm_desc(rows, width, dtype=dtype, post=B.NORM_RMS, pre=B.NORM_LAYER, gate_rows=rows, alpha=alpha, p=p, site=2)
        self.loss = B.make_loss_desc(rows, width, classes, dtype=dtype)
        self.update = {k: B.make_muon_desc(*self.w[k].shape, dtype=dtype, grad_dtype=dtype) for k in ("wide", "narrow", "head")}
        self.momentum = {k: torch.zeros(self.w[k].shape, device=DEV) for k in self.update}
        need = [B.cac_block_norm_workspace_size(d, B.BLOCK_NORM_BWD) for d in (self.first, self.join)]
        need += [B.cac_linear_workspace_size(d, op) for d in (self.wide, self.narrow) for op in (B.LINEAR_FWD, B.LINEAR_BWD)]
        need += [B.cac_loss_workspace_size(self.loss, op) for op in (B.LOSS_FWD, B.LOSS_BWD)]
        need += [B.cac_muon_workspace_size(d, B.MUON_STEP) for d in self.update.values()]
        self.ws = torch.empty(max(16, max(need)), dtype=torch.uint8, device=DEV)
        self.h, self.f, self.s, self.out = (new(rows, width) for _ in range(4))
        self.a = new(rows, hidden)
        self.losses, self.lse = new(rows, kind=torch.float32), new(rows, kind=torch.float32)
        self.gloss = torch.full((rows,), 1.0 / rows, device=DEV)
        self.dout, self.ds, self.df, self.dh, self.dx = (new(rows, width) for _ in range(5))
        self.da = new(rows, hidden)
        self.patterns = torch.randn(classes, width, generator=g, device=DEV)

    def batch(self):
        rows, width, _, classes = self.shape
        labels = torch.randint(0, classes, (rows,), generator=self.gen, device=DEV)
        x = self.patterns[labels] + 0.5 * torch.randn(rows, width, generator=self.gen, device=DEV)
        return x.to(TYPES[self.dtype]), labels

    def forward(self, X, labels):
        w, ws = self.w, self.ws
        B.cac_block_norm_fwd(self.first, X, None, None, None, None, w["in"], None, None, None, self.h)
        B.cac_linear_fwd(self.wide, self.h, w["wide"], w["wide_b"], None, self.rng, self.a, ws)
        B.cac_linear_fwd(self.narrow, self.a, w["narrow"], w["narrow_b"], None, None, self.f, ws)
        B.cac_block_norm_fwd(self.join, self.f, X, w["gate"], w["post"], None, w["pre"], w["pre_b"], self.rng, self.s, self.out)
        B.cac_loss_fwd(self.loss, self.out, w["head"], None, labels, self.losses, self.lse, ws)

    def backward(self, X, labels):
        w, g, ws = self.w, self.grad, self.ws
        B.cac_loss_bwd(self.loss, self.out, w["head"], None, labels, self.lse, self.gloss, self.dout, g["head"], None, ws)
        B.cac_block_norm_bwd(self.join, self.f, self.s, w["gate"], w["post"], None, w["pre"], self.dout, None, self.rng, self.ds, self.df, g["gate"],
                             g["post"], None, g["pre"], g["pre_b"], ws)
        B.cac_linear_bwd(self.narrow, self.a, w["narrow"], None, self.df, None, self.da, g["narrow"], g["narrow_b"], ws)
        B.cac_linear_bwd(self.wide, self.h, w["wide"], w["wide_b"], self.da, self.rng, self.dh, g["wide"], g["wide_b"], ws)
        # the block's input is the sum that its first norm normalises: the residual's gradient comes in beside it
        B.cac_block_norm_bwd(self.first, None, X, None, None, None, w["in"], self.dh, self.ds, None, self.dx, None, None, None, None, g["in"], None, ws)

    def step(self, X, labels, lr=0.02):
        self.forward(X, labels)
        self.backward(X, labels)
        for k, d in self.update.items():
            B.cac_muon_step(d, self.grad[k], self.momentum[k], self.w[k], 0.9, 1.0, lr * max(1.0, d.rows / d.cols) ** 0.5, self.ws)
        for k, v in self.w.items():
            if k not in self.update:
                v.sub_(lr * self.grad[k])
        self.rng[1] += 1
        return self.losses


def main(steps=60, lr=0.02, **sizes):
    block = Block(**sizes)
    history = []
    for k in range(steps):
        mean = float(block.step(*block.batch(), lr=lr).mean())
        history.append(mean)
        if k % 10 == 0 or k + 1 == steps:
            print(f"step {k:3d}  loss {mean:.4f}", flush=True)
    return history


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 60)
