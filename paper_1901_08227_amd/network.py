"""A network trained by M simulated workers: its layers run on 8-bit codes (lowbit), its gradients go through the coder (tng_step).

    x [M, rows, width] -> linear 1 -> relu, dropout -> linear 2 -> dropout, + x -> linear 3 -> classes, softmax cross-entropy

TokenNetwork takes tokens in x's place, and norms its layers' inputs:

    tokens [M, rows] -> embedding e -> norm -> linear 1 -> relu, dropout -> linear 2 -> + e, norm -> linear 3 -> classes

One iteration is forward and backward of every worker's minibatch side by side, each worker's gradient in its row of g[M][d], and
tng_step: normalise against the trajectory, code, decode, average, step.  With orthogonal=True the decoded average of each layer's weights is
orthogonalised before the step.  The weights' codes are laid out once an iteration.

    python -m paper_1901_08227_amd.network [--workers 4] [--rows 256] [--width 256] [--hidden 1024] [--classes 10] [--steps 100]
        [--vocabulary 0] [--orthogonal]
"""
from __future__ import annotations

import argparse

import torch

from . import binding as B
from . import lowbit, synth, update


class Network:
    """The parameters as one vector w, as tng_step takes it, and views of its pieces."""

    def __init__(self, *, workers, width, hidden, classes, p=0.1, lr=0.1, seed=0, bits=4, device="cuda:0", dtype=torch.bfloat16, orthogonal=False,
                 more=0):
        """more: parameters behind those of the layers (a subclass's)."""
        self.shapes = [(hidden, width), (width, hidden), (classes, width)]
        self.M, self.p, self.seed, self.dtype, self.orthogonal, self.lr = workers, p, seed, dtype, orthogonal, lr
        self.device = torch.device(device)
        self.d = sum(n * (k + 1) for n, k in self.shapes) + more
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
        if self.orthogonal:
            self.orthogonal_step(it)
        else:
            self.ctx.step(it, self.w, self.gref, self.g, self.codes, self.scales, self.vbar)
        return loss

    def orthogonal_step(self, it):
        """What tng_step does, but w goes along the decoded averages of the layers' weights orthogonalised, and along the others as they are."""
        self.ctx.normalize_encode(it, self.g, self.gref, self.codes, self.scales)
        self.ctx.decode_aggregate(self.codes, self.scales, self.gref, self.vbar)
        along = self.vbar.clone()
        for w, _ in self.layers(along):
            update.orthogonalize(w, scale=max(1.0, w.shape[0] / w.shape[1]) ** 0.5, out=w)
        self.w.sub_(along, alpha=self.lr)
        self.ctx.update_reference(it, self.vbar, self.gref)

    def close(self):
        self.ctx.close()


class TokenNetwork(Network):
    """A network of tokens: an embedding table [vocabulary, width] and the two norms' weights lie behind the layers' parameters in w."""

    def __init__(self, *, vocabulary, width, **kw):
        self.vocabulary, self.width = vocabulary, width
        super().__init__(width=width, more=(vocabulary + 2) * width, **kw)
        gen = torch.Generator(device=self.device)
        gen.manual_seed(self.seed + 1)
        table, *gains = self.embedding(self.w)
        table.copy_(torch.randn(table.shape, generator=gen, device=self.device) * self.width ** -0.5)
        for gain in gains:
            gain.fill_(1.0)

    def embedding(self, flat):
        """(table, weights of the first norm, of the second) in a vector [d], or in each row of [M, d]."""
        at = self.d - (self.vocabulary + 2) * self.width
        table, gains = flat[..., at:self.d - 2 * self.width], flat[..., self.d - 2 * self.width:]
        return table.unflatten(-1, (self.vocabulary, self.width)), gains[..., :self.width], gains[..., self.width:]

    def forward(self, tokens, it, keep=False):
        (w1, b1), (w2, b2), (w3, b3) = self.layers(self.w)
        table, gain1, gain2 = self.embedding(self.w)
        weights = [lowbit.weight(w, turned=keep) for w in (w1, w2, w3)]
        inner = lowbit.Drop(self.seed, it, 0, self.p if keep else 0.0, True)
        e = lowbit.embed(tokens, table, scale=self.width ** 0.5, dtype=self.dtype)
        n1 = lowbit.rms_norm_codes(e, gain1, turned=keep)
        h = lowbit.matmul_i8(n1.q, weights[0].q, n1.scale, weights[0].scale, b1, dtype=self.dtype)
        h, saved = lowbit.linear(h, weights[1], b2, inner, keep=True) if keep else (lowbit.linear(h, weights[1], b2, inner), None)
        n2 = lowbit.rms_norm_codes(h, gain2, residual=e, turned=keep)
        logits = lowbit.matmul_i8(n2.q, weights[2].q, n2.scale, weights[2].scale, b3, dtype=self.dtype)
        return (logits, (tokens, weights, n1, saved, n2)) if keep else logits

    def backward(self, dlogits, kept, it):
        tokens, weights, n1, saved, n2 = kept
        grads, (dtable, dgain1, dgain2) = self.layers(self.g), self.embedding(self.g)
        _, gain1, gain2 = self.embedding(self.w)

        def layer(k, dy, saved):
            dx, _, db = lowbit.linear_grad(dy, saved, weights[k], seed=self.seed, iter=it, site=2 + k, out=grads[k][0])
            grads[k][1].copy_(db)
            return dx

        dh, dgain = lowbit.rms_norm_grad(layer(2, dlogits, lowbit.Saved(None, None, n2.scale, n2.qt)), n2.h, gain2)
        dgain2.copy_(dgain)
        d = layer(0, layer(1, dh, saved), lowbit.Saved(None, None, n1.scale, n1.qt))
        de, dgain = lowbit.rms_norm_grad(d, n1.h, gain1, dresidual=dh)
        dgain1.copy_(dgain)
        lowbit.embed_grad(tokens, de, self.vocabulary, scale=self.width ** 0.5, out=dtable)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("workers", 4), ("rows", 256), ("width", 256), ("hidden", 1024), ("classes", 10), ("steps", 100), ("seed", 0),
                          ("vocabulary", 0)):
        ap.add_argument(f"--{name}", type=int, default=default)
    ap.add_argument("--orthogonal", action="store_true")
    a = ap.parse_args()
    args = dict(workers=a.workers, width=a.width, hidden=a.hidden, classes=a.classes, seed=a.seed, orthogonal=a.orthogonal)
    if a.orthogonal:
        args["lr"] = 0.01  # (of an update whose singular values are about 1)
    net = TokenNetwork(vocabulary=a.vocabulary, **args) if a.vocabulary else Network(**args)
    for it in range(a.steps):
        if a.vocabulary:
            x, labels = synth.token_classes(a.workers, a.rows, a.vocabulary, a.classes, a.seed, it, device=net.device)
        else:
            x, labels = synth.class_mixture(a.workers, a.rows, a.width, a.classes, a.seed, it, spread=0.2, device=net.device)
            x = x.to(net.dtype)
        loss = net.step(it, x, labels)
        if it % 10 == 0 or it == a.steps - 1:
            print(f"iteration {it}: loss {loss.mean().item():.4f}", flush=True)
    net.close()


if __name__ == "__main__":
    main()
