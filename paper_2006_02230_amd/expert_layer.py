"""A layer of experts from the library's operators: the router's product (sgemm), the choice and plan (route), two products grouped by
expert with ReLU between them, the weighted sum, and all their gradients; answers from 4-bit weights.

    python -m paper_2006_02230_amd.expert_layer      # trains one on a synthetic map, then answers with its weights in 4 bits
"""
import collections

import torch

from . import binding as B
from . import experts as X

Gradients = collections.namedtuple("Gradients", "x router w1 w2")


def _logits(x, router):
    logits = x.new_empty(x.shape[0], router.shape[1])
    return B.sgemm(x, router, logits, alpha=1.0, beta=0.0) if len(x) else logits           # sgemm has no empty matrices


class ExpertLayer:
    """out[t] = sum over the k chosen experts e of weight[t][e] * w2[e] relu(w1[e] x[t]), weights softmax(x[t] router) over the chosen.

    router [D][E] float32, w1 [E][F][D] and w2 [E][D][F] bfloat16, x [T][D] bfloat16.  `forward` leaves what `backward` needs in `kept`;
    with several forwards before their backwards, take it from there after each and give it to its backward."""

    def __init__(self, router, w1, w2, k):
        self.router, self.w1, self.w2, self.k = router, w1, w2, k
        self.kept, self.waiting = None, 0

    def forward(self, x, keep=True):
        """out [T][D] bfloat16.  keep=False: an answer without a backward, of which nothing is kept."""
        xf = x.float()
        logits = _logits(xf, self.router)
        r = X.route(logits, self.k)
        h = X.grouped_gemm_bf16(x, self.w1, r.offsets, rows=r.tokens, act="relu")
        y = X.grouped_gemm_bf16(h, self.w2, r.offsets)
        if keep:
            self.kept, self.waiting = (x, xf, logits, r, h, y), self.waiting + 1
        return X.combine_bf16(y, r.slots, r.weights)

    def backward(self, dout, kept=None):
        """Gradients(x bfloat16, router, w1, w2 float32) of the forward that left `kept` (None: the only one since the last backward), from the
        gradient of what it gave."""
        if kept is None:
            if self.kept is None:
                raise RuntimeError("backward needs a forward that keeps")
            if self.waiting > 1:
                raise RuntimeError("%d forwards wait for their backward: give backward the one's `kept`, and keep=False to a forward without "
                                   "a backward" % self.waiting)
            kept = self.kept
        self.waiting = max(self.waiting - 1, 0)
        x, xf, logits, r, h, y = kept
        dy, dweights = X.combine_bwd_bf16(dout, y, r.slots, r.weights)
        dh = X.grouped_gemm_dx_bf16(dy, self.w2, r.offsets, h=h, act="relu")
        dw2 = X.grouped_gemm_dw_bf16(dy, h, r.offsets)
        dw1 = X.grouped_gemm_dw_bf16(dh, x, r.offsets, rows=r.tokens)
        dx = X.combine_bf16(X.grouped_gemm_dx_bf16(dh, self.w1, r.offsets, out_dtype=torch.bfloat16), r.slots, out_dtype=torch.float32)
        dlogits = X.route_bwd(logits, r.ids, r.weights, dweights)
        if not len(x):
            return Gradients(dx.bfloat16(), torch.zeros_like(self.router), dw1, dw2)
        drouter = B.sgemm(xf.t().contiguous(), dlogits, torch.empty_like(self.router), alpha=1.0, beta=0.0)
        B.sgemm(dlogits, self.router.t().contiguous(), dx)                     # added to what came through the experts
        return Gradients(dx.bfloat16(), drouter, dw1, dw2)

    def coded(self, group=128, asymmetric=False):
        """The same layer with its experts' weights in 4 bits."""
        return CodedExpertLayer(self, group, asymmetric)


class CodedExpertLayer:
    """An ExpertLayer that answers: weights in 4 bits, read once for every 16, 32 or 64 rows of an expert, by the experts' mean."""

    def __init__(self, layer, group, asymmetric):
        self.router, self.k, self.group = layer.router, layer.k, group
        _, self.width, _ = layer.w1.shape
        self.w1, self.w2 = (X.w4_pack_bf16(w, group, asymmetric) for w in (layer.w1, layer.w2))

    def forward(self, x):
        F, D = self.width, self.router.shape[0]
        r = X.route(_logits(x.float(), self.router), self.k)
        h = X.w4_gemm_bf16(x, self.w1.q, self.w1.scales, F, self.group, zeros=self.w1.zeros, offsets=r.offsets, rows=r.tokens, act="relu")
        y = X.w4_gemm_bf16(h, self.w2.q, self.w2.scales, D, self.group, zeros=self.w2.zeros, offsets=r.offsets)
        return X.combine_bf16(y, r.slots, r.weights)


def main(steps=60, T=2048, D=256, F=512, E=16, k=2, seed=0):
    """Fits a layer to the answers of another one; returns the first and last loss and the loss with 4-bit weights."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s, scale=1.0: torch.randn(*s, generator=g, device="cuda") * scale   # noqa: E731
    make = lambda: (randn(D, E, scale=D ** -0.5), randn(E, F, D, scale=D ** -0.5), randn(E, D, F, scale=F ** -0.5))   # noqa: E731
    router, w1, w2 = make()
    goal = ExpertLayer(router, w1.bfloat16(), w2.bfloat16(), k)
    start = make()
    master = [router + 0.3 * start[0], w1 + 0.3 * start[1], w2 + 0.3 * start[2]]
    moments = [torch.zeros_like(m) for m in master], [torch.zeros_like(m) for m in master]
    losses = []
    for step in range(steps):
        x = randn(T, D).bfloat16()
        want = goal.forward(x, keep=False).float()
        layer = ExpertLayer(master[0], master[1].bfloat16(), master[2].bfloat16(), k)
        error = layer.forward(x).float() - want
        losses.append(error.square().mean())
        grads = layer.backward((error * (2.0 / error.numel())).bfloat16())
        for m, grad, a, b in zip(master, grads[1:], *moments):
            a.mul_(0.9).add_(grad, alpha=0.1)
            b.mul_(0.99).addcmul_(grad, grad, value=0.01)
            m.sub_(3e-3 * (a / (1 - 0.9 ** (step + 1))) / ((b / (1 - 0.99 ** (step + 1))).sqrt() + 1e-12))
    x = randn(T, D).bfloat16()
    coded = (layer.coded(32, True).forward(x).float() - goal.forward(x, keep=False).float()).square().mean()
    return float(losses[0]), float(losses[-1]), float(coded)


if __name__ == "__main__":
    print("loss: %.4f at first, %.4f after training, %.4f with the trained weights in 4 bits" % main())
