"""A block of a model around a layer of experts: the layer norm before it, the sum with what came in, the balance loss of its router, the clipping of its
gradients; answers in microscaled 4-bit floating point.

    python -m paper_2006_02230_amd.expert_block      # trains one on a synthetic map, then answers with its weights in 4 bits
"""
import collections

import torch

from . import training as Y
from .expert_layer import ExpertLayer

BlockGradients = collections.namedtuple("BlockGradients", "x gamma beta router w1 w2")


class ExpertBlock:
    """out = x + layer(layernorm(x)), x [T][D] bfloat16, gamma and beta [D] float32, layer an ExpertLayer.  What the norm and the layer give is bfloat16, as
    by themselves, and so is their sum with x.

    `forward` leaves what `backward` needs in `kept`; with several forwards before their backwards, take it from there after each and give it to its
    backward."""

    def __init__(self, gamma, beta, layer, eps=1e-5):
        self.gamma, self.beta, self.layer, self.eps = gamma, beta, layer, eps
        self.kept = None

    def forward(self, x, keep=True):
        """out [T][D] bfloat16.  keep=False: an answer without a backward, of which nothing is kept."""
        norm = Y.layernorm_fwd(x, self.gamma, self.beta, self.eps)
        out = x + self.layer.forward(norm.y, keep)
        if keep:
            self.kept = x, norm, self.layer.kept
        return out

    def backward(self, dout, kept=None):
        """BlockGradients(x bfloat16, the others float32) of the forward that left `kept` (None: the only one since the last backward), from the
        gradient of what it gave; the layer's balance loss, times its share, belongs to the loss."""
        if kept is None:
            self.layer._only(self.kept and self.kept[2])
            kept = self.kept
        x, norm, layer = kept
        inner = self.layer.backward(dout, layer)
        # The norm's gradient in float32, so that its sum with what comes past the layer is rounded once.  A sum of two bfloat16 values has 1.28 times the error
        # (2.1e-3 of the sum's norm where it is 1.65e-3); the whole backward takes 2404 us with one and 2464 so (8192 rows of 2048, 4 of 16 experts of 4096).
        d = Y.layernorm_bwd(inner.x, x.float(), norm.mean, norm.rstd, self.gamma)
        return BlockGradients(torch.add(d.dx, dout, out=torch.empty_like(x)), d.dgamma, d.dbeta, inner.router, inner.w1, inner.w2)

    def microscaled(self):
        """The same block with its experts' products in microscaled 4-bit floating point; it answers."""
        return MicroscaledExpertBlock(self)


class MicroscaledExpertBlock:
    def __init__(self, block):
        self.gamma, self.beta, self.eps, self.layer = block.gamma, block.beta, block.eps, block.layer.microscaled()

    def forward(self, x):
        return x + self.layer.forward(Y.layernorm_fwd(x, self.gamma, self.beta, self.eps).y)


def main(steps=60, T=2048, D=256, F=512, E=16, k=2, balance=0.01, max_norm=0.1, seed=0):
    """Fits a block to the answers of another one; returns the losses, balance losses and gradient norms of the steps, and the loss in 4 bits."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s, scale=1.0: torch.randn(*s, generator=g, device="cuda") * scale   # noqa: E731
    make = lambda: [1 + randn(D, scale=0.1), randn(D, scale=0.1), randn(D, E, scale=D ** -0.5), randn(E, F, D, scale=D ** -0.5),    # noqa: E731
                    randn(E, D, F, scale=F ** -0.5)]
    build = lambda m: ExpertBlock(m[0], m[1], ExpertLayer(m[2], m[3].bfloat16(), m[4].bfloat16(), k, balance))   # noqa: E731
    true = make()
    goal = build(true)
    master = [a + 0.3 * b for a, b in zip(true, make())]
    moments = [torch.zeros_like(m) for m in master], [torch.zeros_like(m) for m in master]
    losses, balances, norms = [], [], []
    for step in range(steps):
        x = (randn(T, D) + 0.5).bfloat16()
        block = build(master)
        error = block.forward(x).float() - goal.forward(x, keep=False).float()
        losses.append(error.square().mean())
        balances.append(block.layer.used.loss)
        grads = block.backward((error * (2.0 / error.numel())).bfloat16())[1:]
        norms.append(Y.clip_grads(grads, max_norm))
        for m, grad, a, b in zip(master, grads, *moments):
            a.mul_(0.9).add_(grad, alpha=0.1)
            b.mul_(0.99).addcmul_(grad, grad, value=0.01)
            m.sub_(3e-3 * (a / (1 - 0.9 ** (step + 1))) / ((b / (1 - 0.99 ** (step + 1))).sqrt() + 1e-12))
    x = (randn(T, D) + 0.5).bfloat16()
    coded = (block.microscaled().forward(x).float() - goal.forward(x, keep=False).float()).square().mean()
    return [[float(v) for v in values] for values in (losses, balances, norms)] + [float(coded)]


if __name__ == "__main__":
    _losses, _balances, _norms, _coded = main()
    print("loss: %.4f at first, %.4f after training, %.4f with the trained weights in 4 bits; balance loss %.3f, then %.3f; gradients' norm %.3f, then %.3f"
          % (_losses[0], _losses[-1], _coded, _balances[0], _balances[-1], _norms[0], _norms[-1]))
