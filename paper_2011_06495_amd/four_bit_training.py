"""Training with the vote step and 4-bit numerics around it, on one GPU: an example.

  python -m paper_2011_06495_amd.four_bit_training [--steps 40] [--workers 8] [--eight-bit] [--norm] [--teacher 4]

N workers train one two-layer network on a synthetic classification task.  One step is

  products      mv_mx_linear, mv_mx_linear_grad   every worker's forward and backward pass, all products in microscaled
                                                  4-bit floating point
  clipping      mv_clip_grads                     every worker's gradients scaled to a global norm of at most MAX_NORM and
                                                  packed into its row of the N x d matrix
  vote          mv_vote_step                      error compensation, votes, the mask, error update
  sending       mv_mx_encode, mv_mx_aggregate     the workers' masked values in 4 bits; what 4 bits lose goes back into
                                                  the error buffers; the server's mean moves the parameters

The parameters are kept in fp32 and quantised after every step.  The softmax and its gradient, the gather of the
masked values and the update are plain torch.  Options change what a worker's pass is made of:

  --eight-bit   mv_f8_linear, mv_f8_linear_grad              products in 8-bit floating point by blocks of 128
  --norm        mv_layernorm_forward, mv_layernorm_backward  a layer norm between the two layers, with weights that are trained
  --teacher K   mv_distill_loss                              half of the loss is distillation from a teacher's best K logits,
                                                             and loss and gradient are one call
"""
from __future__ import annotations

import argparse
import math
from typing import List

import torch

from . import binding as B

INPUTS, HIDDEN, CLASSES, BATCH = 200, 330, 10, 96
MAX_NORM = 1.0
EPS, TEMPERATURE = 1e-5, 2.0


def up(x: int, m: int) -> int:
    return (x + m - 1) // m * m


class Weights:
    """A layer's weights in 4 bits, along the inputs for the forward pass and along the outputs for the backward pass."""

    words, row_words, row_scales = torch.int32, staticmethod(B.mv_mx_row_words), staticmethod(B.mv_mx_row_scales)
    encode, encode_t = staticmethod(B.mv_mx_encode), staticmethod(B.mv_mx_encode_t)
    linear, linear_grad = staticmethod(B.mv_mx_linear), staticmethod(B.mv_mx_linear_grad)
    scratch_bytes = (B.mv_mx_linear_scratch_bytes, B.mv_mx_linear_grad_scratch_bytes)

    def __init__(self, w):
        self.n, self.k = w.shape
        dev = w.device
        self.codes = torch.zeros((self.n, self.row_words(self.k)), dtype=self.words, device=dev)
        self.scales = torch.zeros((self.n, self.row_scales(self.k)), dtype=torch.uint8, device=dev)
        self.codes_t = torch.zeros((self.k, self.row_words(self.n)), dtype=self.words, device=dev)
        self.scales_t = torch.zeros((self.k, self.row_scales(self.n)), dtype=torch.uint8, device=dev)

    def hold(self, w) -> None:
        self.encode(w, self.codes, self.scales)
        self.encode_t(w, self.codes_t, self.scales_t)


class EightBitWeights(Weights):
    """The same in 8 bits."""

    words, row_words, row_scales = torch.uint8, staticmethod(B.mv_f8_row_bytes), staticmethod(B.mv_f8_row_scales)
    encode, encode_t = staticmethod(B.mv_f8_encode), staticmethod(B.mv_f8_encode_t)
    linear, linear_grad = staticmethod(B.mv_f8_linear), staticmethod(B.mv_f8_linear_grad)
    scratch_bytes = (B.mv_f8_linear_scratch_bytes, B.mv_f8_linear_grad_scratch_bytes)


class Trainer:
    def __init__(self, workers: int, seed: int = 0, share: int = 50, eight_bit: bool = False, norm: bool = False, teacher: int = 0):
        dev = torch.device("cuda:0")
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.n, self.gen, self.dev = workers, gen, dev
        shapes = [(HIDDEN, INPUTS), (CLASSES, HIDDEN)]
        layers = len(shapes)
        if norm:
            shapes += [(HIDDEN,), (HIDDEN,)]         # its weight and its bias
        self.sizes = [math.prod(shape) for shape in shapes]
        self.d = sum(self.sizes)
        self.k = self.d // share
        self.flat = torch.empty(self.d, device=dev)
        self.params = [p.view(s) for p, s in zip(self.flat.split(self.sizes), shapes)]
        for p in self.params[:layers]:
            p.copy_(torch.randn(p.shape, generator=gen, device=dev) / p.shape[1] ** 0.5)
        self.norm = self.params[layers:]
        if norm:
            self.norm[0].fill_(1.0)
            self.norm[1].zero_()
        held = EightBitWeights if eight_bit else Weights
        self.weights = [held(p) for p in self.params[:layers]]
        self.teacher = teacher
        self.centres = 0.4 * torch.randn((CLASSES, INPUTS), generator=gen, device=dev)
        # a worker's gradients as its backward pass leaves them, and the matrix that the vote step takes
        self.grads = [[torch.zeros(s, device=dev) for s in shapes] for _ in range(workers)]
        ld = up(self.d, 8)
        self.rows = torch.zeros((workers, ld), device=dev)[:, : self.d]
        self.err = torch.zeros((workers, ld), device=dev)[:, : self.d]
        self.sent = torch.zeros((workers, ld), device=dev)[:, : self.d]
        self.norms, self.coefs = torch.zeros(workers, device=dev), torch.zeros(workers, device=dev)
        places = [t.view(s) for row in self.rows for t, s in zip(row.split(self.sizes), shapes)]
        self.clip = B.mv_clip_begin([g for worker in self.grads for g in worker], out=places,
                                    groups=[r for r in range(workers) for _ in shapes])
        self.ctx = B.mv_begin(B.make_config(workers, self.d, self.k))
        self.mask = torch.zeros(self.k, dtype=torch.int32, device=dev)
        self.mean = torch.zeros(self.k, device=dev)
        self.codes = torch.zeros((workers, B.mv_mx_row_words(self.k)), dtype=torch.int32, device=dev)
        self.scales = torch.zeros((workers, B.mv_mx_row_scales(self.k)), dtype=torch.uint8, device=dev)
        need = max(size(BATCH, *s) for size in held.scratch_bytes for s in shapes[:layers])
        if norm:
            need = max(need, B.mv_layernorm_scratch_bytes(BATCH, HIDDEN))
            self.h_mean, self.h_rstd = torch.zeros(BATCH, device=dev), torch.zeros(BATCH, device=dev)
        if teacher:
            need = max(need, B.mv_distill_scratch_bytes(BATCH, CLASSES))
            self.share = torch.full((BATCH,), 1.0 / BATCH, device=dev)
        self.scratch = torch.empty(need, dtype=torch.uint8, device=dev)

    def batch(self):
        y = torch.randint(0, CLASSES, (BATCH,), generator=self.gen, device=self.dev)
        return self.centres[y] + torch.randn((BATCH, INPUTS), generator=self.gen, device=self.dev), y

    def loss(self, x, y, out):
        """The losses of a batch and their mean's gradient."""
        if self.teacher:
            # what a teacher knows who has seen where the inputs come from: their classes' log densities
            logits = x @ self.centres.t() - 0.5 * self.centres.square().sum(1)
            top, idx = logits.topk(self.teacher)
            losses, dy = torch.empty(BATCH, device=self.dev), torch.empty_like(out)
            B.mv_distill_loss(out, idx.to(torch.int32), top, y.to(torch.int32), TEMPERATURE, 0.5, 0.5, losses, self.scratch, dz=dy,
                              grad=self.share)
            return losses, dy
        log_p = torch.log_softmax(out, 1)
        dy = torch.exp(log_p)
        dy[torch.arange(BATCH, device=self.dev), y] -= 1.0
        dy /= BATCH
        return -log_p[torch.arange(BATCH, device=self.dev), y], dy

    def gradients(self, x, y, grads) -> torch.Tensor:
        """One worker's pass: its gradients into `grads`; returns its loss."""
        w1, w2 = self.weights
        h, out = torch.empty((BATCH, HIDDEN), device=self.dev), torch.empty((BATCH, CLASSES), device=self.dev)
        w1.linear(x, w1.codes, w1.scales, h, self.scratch)
        live = h > 0
        h *= live
        h2 = h
        if self.norm:
            h2 = torch.empty_like(h)
            B.mv_layernorm_forward(h, *self.norm, EPS, h2, self.h_mean, self.h_rstd)
        w2.linear(h2, w2.codes, w2.scales, out, self.scratch)
        losses, dy = self.loss(x, y, out)
        dh = torch.empty_like(h)
        w2.linear_grad(h2, dy, w2.codes_t, w2.scales_t, dh, grads[1], self.scratch)
        if self.norm:
            B.mv_layernorm_backward(h, dh, self.norm[0], self.h_mean, self.h_rstd, dh, grads[2], grads[3], self.scratch)
        dh *= live
        w1.linear_grad(x, dh, None, None, None, grads[0], self.scratch)
        return losses.mean()

    def step(self, rate: float) -> torch.Tensor:
        for w, p in zip(self.weights, self.params):
            w.hold(p)
        losses = [self.gradients(*self.batch(), grads) for grads in self.grads]
        B.mv_clip_grads(self.clip, MAX_NORM, self.norms, self.coefs)
        # the step's own sum g + e is wanted on the mask below, so it is formed here and e starts it at zero
        torch.add(self.rows, self.err, out=self.sent)
        self.err.zero_()
        B.mv_vote_step(self.ctx, self.sent, self.err, None, None, self.mask, self.mean)
        at = self.mask.long()
        vals = self.sent[:, at]
        B.mv_mx_encode(vals, self.codes, self.scales, resid=vals)
        B.mv_mx_aggregate(self.codes, self.scales, None, self.mean)
        self.err[:, at] = vals
        self.flat[at] -= rate * self.mean
        return torch.stack(losses).mean()

    def close(self) -> None:
        B.mv_clip_end(self.clip)
        B.mv_clip_release(self.clip)
        B.mv_end(self.ctx)
        B.mv_release(self.ctx)


def train(steps: int, workers: int = 8, rate: float = 0.5, seed: int = 0, **options) -> List[float]:
    """The mean loss of each step."""
    t = Trainer(workers, seed, **options)
    try:
        return [float(t.step(rate)) for _ in range(steps)]
    finally:
        t.close()


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--workers", type=int, default=8)
    ap.add_argument("--eight-bit", action="store_true", help="products in 8 bits")
    ap.add_argument("--norm", action="store_true", help="a layer norm between the layers")
    ap.add_argument("--teacher", type=int, default=0, metavar="K", help="learn from a teacher's best K logits, too")
    a = ap.parse_args()
    if not 0 <= a.teacher <= CLASSES:
        ap.error("a teacher has 1 to %d logits" % CLASSES)
    for i, loss in enumerate(train(a.steps, a.workers, eight_bit=a.eight_bit, norm=a.norm, teacher=a.teacher)):
        if i % 5 == 0 or i == a.steps - 1:
            print("step %3d  loss %.4f" % (i, loss), flush=True)


if __name__ == "__main__":
    main()
