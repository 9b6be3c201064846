"""A training step from end to end on the library's calls: a convolution whose saved input is pooled, batch normalisation
from its pooled record, a linear classifier whose logits are never kept, and the filters and the classifier's weights updated by
orthogonalised gradients.

    python examples/classifier_step.py [steps]

trains a network of one 3x3 convolution and a classifier on synthetic images (every class has a pattern of its own, under
noise) and prints the loss of every tenth step.  Device memory, the batch statistics and the average over the pixels are torch's.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2409_11902_amd import binding as B  # noqa: E402

DEV = "cuda:0"


class Network:
    def __init__(self, images=128, channels=16, filters=64, side=16, classes=1000, pool=2, seed=0):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.gen, self.N, self.C, self.K, self.side, self.V = g, images, channels, filters, side, classes
        self.W = torch.randn(filters, channels, 3, 3, generator=g, device=DEV) * (2.0 / (9 * channels)) ** 0.5
        self.head = torch.randn(classes, filters, generator=g, device=DEV) * 0.05
        self.gamma, self.beta, self.bias = torch.ones(filters, device=DEV), torch.zeros(filters, device=DEV), torch.zeros(classes, device=DEV)
        self.patterns = torch.randn(classes, channels, generator=g, device=DEV)
        # the descriptors of the step: the convolution, the normalisation (a 1x1 consumer of the same pooling), the loss, the updates
        self.conv = B.make_desc(images, channels, filters, side, side, 3, 3, 1, 1, 1, 1, pool, pool, dtype=B.F32, has_bias=0)
        self.norm = B.make_desc(images, filters, 1, side, side, 1, 1, 1, 1, 0, 0, pool, pool, dtype=B.F32, has_bias=0)
        self.loss = B.make_loss_desc(images, filters, classes, dtype=B.F32, has_bias=1)
        self.update = [(self.W, B.make_muon_desc(filters, channels * 9)), (self.head, B.make_muon_desc(classes, filters))]
        self.momentum = [torch.zeros_like(w) for w, _ in self.update]
        need = [B.cac_workspace_size(self.conv, op) for op in (B.OP_FWD_AND_COMPRESS, B.OP_BWD_WEIGHT_COMPRESSED)]
        need += [B.cac_workspace_size(self.norm, B.OP_BN_BWD)]
        need += [B.cac_loss_workspace_size(self.loss, op) for op in (B.LOSS_FWD, B.LOSS_BWD)]
        need += [B.cac_muon_workspace_size(d, B.MUON_STEP) for _, d in self.update]
        self.ws = torch.empty((max(need) + 15) // 16 * 16, dtype=torch.uint8, device=DEV)
        half = -(-side // pool)
        shape = (images, filters, side, side)
        self.Z, self.Zin = torch.empty(images, channels, half, half, device=DEV), torch.empty(images, filters, half, half, device=DEV)
        self.Znext = torch.empty_like(self.Zin)                      # (the next convolution's record, had the network one)
        self.Y, self.act, self.dY = torch.empty(shape, device=DEV), torch.empty(shape, device=DEV), torch.empty(shape, device=DEV)
        self.losses, self.lse = torch.empty(images, device=DEV), torch.empty(images, device=DEV)
        self.gloss = torch.full((images,), 1.0 / images, device=DEV)

    def batch(self):
        labels = torch.randint(0, self.V, (self.N,), generator=self.gen, device=DEV)
        noise = torch.randn(self.N, self.C, self.side, self.side, generator=self.gen, device=DEV)
        return self.patterns[labels][:, :, None, None] + 0.5 * noise, labels

    def step(self, X, labels, lr=0.02):
        ws, pixels = self.ws, self.side * self.side
        # forward
        B.conv_fwd_and_compress(self.conv, X, self.W, None, self.Y, self.Z, ws)          # X itself is not needed again
        mean, var = self.Y.mean(dim=(0, 2, 3)), self.Y.var(dim=(0, 2, 3), unbiased=False)
        invstd = (var + 1e-5).rsqrt()
        scale = self.gamma * invstd
        B.cac_bn_relu_fwd_compress(self.norm, self.Y, scale, self.beta - mean * scale, self.act, self.Znext, self.Zin)
        H = self.act.mean(dim=(2, 3))
        B.cac_loss_fwd(self.loss, H, self.head, self.bias, labels, self.losses, self.lse, ws)
        # backward
        dH, dhead, dbias = torch.empty_like(H), torch.empty_like(self.head), torch.empty_like(self.bias)
        B.cac_loss_bwd(self.loss, H, self.head, self.bias, labels, self.lse, self.gloss, dH, dhead, dbias, ws)
        dact = (dH / pixels)[:, :, None, None] * (self.act > 0)
        dgamma, dbeta, dW = torch.empty_like(self.gamma), torch.empty_like(self.beta), torch.empty_like(self.W)
        B.cac_bn_bwd_compressed(self.norm, self.Zin, dact, mean, invstd, self.gamma, dgamma, dbeta, self.dY, ws)
        B.conv_bwd_weight_compressed(self.conv, self.Z, self.dY, dW, ws)
        # update: matrices by orthogonalised momentum, vectors by plain steps
        for (w, d), m, grad in zip(self.update, self.momentum, (dW, dhead)):
            B.cac_muon_step(d, grad, m, w, 0.9, 1.0, lr * max(1.0, d.rows / d.cols) ** 0.5, ws)
        for v, grad in ((self.gamma, dgamma), (self.beta, dbeta), (self.bias, dbias)):
            v.sub_(lr * grad)
        return self.losses


def main(steps=60, lr=0.06, **sizes):
    net = Network(**sizes)
    history = []
    for k in range(steps):
        mean = float(net.step(*net.batch(), lr=lr).mean())
        history.append(mean)
        if k % 10 == 0 or k + 1 == steps:
            print(f"step {k:3d}  loss {mean:.4f}", flush=True)
    return history


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 60)
