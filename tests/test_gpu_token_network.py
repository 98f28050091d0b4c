"""Embeddings, norms, 8-bit layers and orthogonalised updates as a network of tokens puts them together: its gradients against those of the same
network in binary64, and its steps."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, say
from oracle import token_oracle as T
from oracle import update_oracle as U
from paper_1901_08227_amd import lowbit, network, synth

pytestmark = pytest.mark.gpu


def make(**kw):
    args = dict(vocabulary=50, workers=3, width=64, hidden=160, classes=7, p=0.0, lr=0.1, seed=5, device=DEV, dtype=torch.float32)
    args.update(kw)
    return network.TokenNetwork(**args)


def batch(net, it, rows=40):
    return synth.token_classes(net.M, rows, net.vocabulary, net.shapes[2][0], 5, it, device=DEV)


def exact_gradients(net, tokens, labels):
    """Each worker's gradient, of no codes, by autograd in binary64 on the host."""
    out = []
    for m in range(net.M):
        w = net.w.double().cpu().requires_grad_()
        (w1, b1), (w2, b2), (w3, b3) = net.layers(w)
        table, gain1, gain2 = net.embedding(w)
        e = table[tokens[m].cpu()] * net.width ** 0.5
        norm = lambda h, gain: h * torch.rsqrt((h * h).mean(-1, keepdim=True) + 1e-6) * gain  # noqa: E731
        h = torch.relu(norm(e, gain1) @ w1.t() + b1) @ w2.t() + b2
        logits = norm(h + e, gain2) @ w3.t() + b3
        torch.nn.functional.cross_entropy(logits, labels[m].cpu()).backward()
        out.append(w.grad)
    return torch.stack(out)


def test_gradients_are_those_of_the_network():
    # What the codes take: a rounding is off by step / sqrt(12) in the mean, and the largest of 64 to 160 numbers is 2.5 to 3.5 of their root mean square, so
    # an operand is off by 3.5 / 127 / sqrt(12) = 0.8 % of itself, by twice that where draws round it.  A gradient comes by way of at most six products,
    # of two operands each: sqrt(6 (0.8^2 + 1.6^2)) = 4.4 %.  A term left out or doubled is off by far more than three times that.
    net = make()
    tokens, labels = batch(net, 0)
    want = exact_gradients(net, tokens, labels)
    net.step(0, tokens, labels)
    got = net.g.double().cpu()
    for a, b in zip([t for pair in net.layers(got) for t in pair] + list(net.embedding(got)), [t for pair in net.layers(want) for t in pair] + list(net.embedding(want))):
        for m in range(net.M):
            assert (a[m] - b[m]).norm() <= 0.13 * b[m].norm()
    net.close()


def test_calls_hand_on_what_the_next_ones_take(monkeypatch):
    seen = {}

    def kept(name):
        f = getattr(lowbit, name)

        def call(*args, **kw):
            seen.setdefault(name, []).append((args, kw, f(*args, **kw)))
            return seen[name][-1][2]
        monkeypatch.setattr(lowbit, name, call)

    for name in ("embed", "rms_norm_codes", "rms_norm_grad", "embed_grad", "linear_grad"):
        kept(name)
    net = make(dtype=torch.bfloat16, p=0.1)
    tokens, labels = batch(net, 1)
    table, gain1, gain2 = (t.clone() for t in net.embedding(net.w))
    net.step(1, tokens, labels)
    e = seen["embed"][0][2]
    assert torch.equal(e, (table[tokens] * torch.tensor(net.width ** 0.5, device=DEV)).bfloat16())
    (n1, n2), ((a2, k2, (dh, dgain2)), (a1, k1, (de, dgain1))) = [s[2] for s in seen["rms_norm_codes"]], seen["rms_norm_grad"]
    assert n1.h is e and seen["rms_norm_codes"][1][1]["residual"] is e
    assert a2[1] is n2.h and a1[1] is e and k1["dresidual"] is dh and "dresidual" not in k2
    assert a2[0] is seen["linear_grad"][0][2][0] and seen["linear_grad"][1][0][0] is dh and a1[0] is seen["linear_grad"][2][2][0]
    dtable, g1, g2 = net.embedding(net.g)
    assert torch.equal(g1, dgain1) and torch.equal(g2, dgain2) and seen["embed_grad"][0][0][1] is de
    for m in range(net.M):
        want, size = T.embed_grad(tokens[m].cpu().numpy(), de[m].float().cpu().numpy(), net.vocabulary, net.width ** 0.5)
        count = np.bincount(tokens[m].cpu().numpy(), minlength=net.vocabulary)[:, None]
        assert np.all(np.abs(dtable[m].double().cpu().numpy() - want) <= (count + 1) * 2.0 ** -24 * size)
    net.close()


def test_an_orthogonal_step():
    net, plain = make(orthogonal=True, lr=0.02), make(lr=0.02)
    tokens, labels = batch(net, 0)
    before = net.w.clone()
    net.step(0, tokens, labels)
    plain.step(0, tokens, labels)
    assert torch.equal(net.vbar, plain.vbar) and torch.equal(net.gref, plain.gref) and torch.equal(net.codes, plain.codes)
    # the layers' weights go along the orthogonalised average, the others as tng_step has them (a product and a difference, one rounding each, or one of both)
    for (w, b), (w0, b0), (v, vb) in zip(net.layers(net.w), net.layers(before), net.layers(net.vbar)):
        scale = max(1.0, w.shape[0] / w.shape[1]) ** 0.5
        want, error = U.orthogonalize(v.cpu().numpy(), ((3.4445, -4.775, 2.0315),) * 5, 1e-7, scale, (2.0 ** -21, 2.0 ** -39, lambda k: (3 * k / 32 + 8) * 2.0 ** -23 + 3 * 2.0 ** -21))
        step = (w0.double() - w.double()).cpu().numpy() / 0.02
        assert np.linalg.norm(step - want) <= error + 2.0 ** -24 * (np.linalg.norm(want) + 2 * w0.double().norm().item() / 0.02)
        assert torch.allclose(b, b0 - 0.02 * vb, rtol=2.0 ** -22, atol=1e-9)
    for a, a0, v in zip(net.embedding(net.w), net.embedding(before), net.embedding(net.vbar)):
        assert torch.allclose(a, a0 - 0.02 * v, rtol=2.0 ** -22, atol=1e-9)
    net.close()
    plain.close()


@pytest.mark.parametrize("orthogonal", [False, True])
def test_runs_repeat_bit_for_bit(orthogonal):
    runs = []
    for _ in range(2):
        net = make(dtype=torch.bfloat16, p=0.1, orthogonal=orthogonal, lr=0.02)
        losses = [net.step(it, *batch(net, it)).mean().item() for it in range(12)]
        x, _ = batch(net, 100, rows=5)
        runs.append((losses, net.w.clone(), net.forward(x, 0)))
        assert np.all(np.isfinite(losses)) and net.w.isfinite().all()
        net.close()
    say(f"token network: loss {losses[0]:.3f} -> {losses[-1]:.3f}")
    assert runs[0][0] == runs[1][0] and torch.equal(runs[0][1], runs[1][1]) and torch.equal(runs[0][2], runs[1][2])
