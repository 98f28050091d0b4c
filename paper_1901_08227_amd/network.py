"""A network trained by M simulated workers: its layers run on 8-bit codes (lowbit), its gradients go through the coder (tng_step).

    x [M, rows, width] -> linear 1 -> relu, dropout -> linear 2 -> dropout, + x -> linear 3 -> classes, softmax cross-entropy

One iteration is forward and backward of every worker's minibatch side by side, each worker's gradient in its row of g[M][d], and
tng_step: normalise against the trajectory, code, decode, average, step.  The weights' codes are laid out once an iteration.

    python -m paper_1901_08227_amd.network [--workers 4] [--rows 256] [--width 256] [--hidden 1024] [--classes 10] [--steps 100]
"""
from __future__ import annotations

import argparse

import torch

from . import binding as B
from . import lowbit, synth


class Network:
    """The parameters as one vector w, as tng_step takes it, and views of its pieces."""

    def __init__(self, *, workers, width, hidden, classes, p=0.1, lr=0.1, seed=0, bits=4, device="cuda:0", dtype=torch.bfloat16):
        self.shapes = [(hidden, width), (width, hidden), (classes, width)]
        self.M, self.p, self.seed, self.dtype = workers, p, seed, dtype
        self.device = torch.device(device)
        self.d = sum(n * (k + 1) for n, k in self.shapes)
        gen = torch.Generator(device=self.device)
        gen.manual_seed(seed)
        self.w = torch.zeros(self.d, device=self.device)
        self.g = torch.zeros((workers, self.d), device=self.device)
        for w, _ in self.layers(self.w):
            w.copy_(torch.randn(w.shape, generator=gen, device=self.device) * w.shape[-1] ** -0.5)
        self.ctx = B.Context(d=self.d, M=workers, bits=bits, norm=B.NORM_SUB, ref_policy=B.REF_LAST_AVG, ref_period=1, seed=seed, lr=lr,
                             problem=B.PROB_EXTERNAL, device=device)
        self.gref = torch.zeros(self.d, device=self.device)
        self.vbar = torch.empty(self.d, device=self.device)
        self.codes = torch.empty((workers, self.ctx.words), dtype=torch.int32, device=self.device)
        self.scales = torch.empty(workers, device=self.device)

    def layers(self, flat):
        """(weights, bias) of each layer in a vector [d], or in each row of [M, d]."""
        at, out = 0, []
        for n, k in self.shapes:
            w, b = flat[..., at:at + n * k], flat[..., at + n * k:at + n * (k + 1)]
            out.append((w.unflatten(-1, (n, k)), b))
            at += n * (k + 1)
        return out

    def forward(self, x, it, keep=False):
        """Logits [M, rows, classes]; keep: and what backward reads again."""
        (w1, b1), (w2, b2), (w3, b3) = self.layers(self.w)
        weights = [lowbit.weight(w, turned=keep) for w in (w1, w2, w3)]
        p = self.p if keep else 0.0
        inner, outer = lowbit.Drop(self.seed, it, 0, p, True), lowbit.Drop(self.seed, it, 1, p, False)
        if not keep:
            h = lowbit.linear(lowbit.linear(x, weights[0], b1), weights[1], b2, inner)
            return lowbit.linear(lowbit.dropout(h, outer, x), weights[2], b3)
        h, s1 = lowbit.linear(x, weights[0], b1, keep=True)
        h, s2 = lowbit.linear(h, weights[1], b2, inner, keep=True)
        logits, s3 = lowbit.linear(lowbit.dropout(h, outer, x), weights[2], b3, keep=True)
        return logits, (weights, (s1, s2, s3), outer)

    def backward(self, dlogits, kept, it):
        """Every worker's gradient, into g."""
        weights, saved, outer = kept
        grads = self.layers(self.g)

        def layer(k, dy):
            dx, _, db = lowbit.linear_grad(dy, saved[k], weights[k], seed=self.seed, iter=it, site=2 + k, out=grads[k][0])
            grads[k][1].copy_(db)
            return dx

        layer(0, layer(1, lowbit.dropout_grad(layer(2, dlogits), outer)))

    def step(self, it, x, labels):
        """One iteration on minibatches x [M, rows, width], labels [M, rows]; the workers' mean losses."""
        logits, kept = self.forward(x, it, keep=True)
        log_p = torch.log_softmax(logits.float(), -1)
        loss = -log_p.gather(-1, labels[..., None]).mean((1, 2))
        d = log_p.exp()
        d.scatter_add_(-1, labels[..., None], torch.full_like(log_p[..., :1], -1.0))
        self.backward((d / labels.shape[1]).to(self.dtype), kept, it)
        self.ctx.step(it, self.w, self.gref, self.g, self.codes, self.scales, self.vbar)
        return loss

    def close(self):
        self.ctx.close()


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("workers", 4), ("rows", 256), ("width", 256), ("hidden", 1024), ("classes", 10), ("steps", 100), ("seed", 0)):
        ap.add_argument(f"--{name}", type=int, default=default)
    a = ap.parse_args()
    net = Network(workers=a.workers, width=a.width, hidden=a.hidden, classes=a.classes, seed=a.seed)
    for it in range(a.steps):
        x, labels = synth.class_mixture(a.workers, a.rows, a.width, a.classes, a.seed, it, spread=0.2, device=net.device)
        loss = net.step(it, x.to(net.dtype), labels)
        if it % 10 == 0 or it == a.steps - 1:
            print(f"iteration {it}: loss {loss.mean().item():.4f}", flush=True)
    net.close()


if __name__ == "__main__":
    main()
