"""A network on 8-bit layers whose gradients go through the coder: the whole of an iteration, as network.py puts it together."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, say
from oracle import lowbit_oracle as L
from oracle import tng_oracle as O
from paper_1901_08227_amd import network, synth

pytestmark = pytest.mark.gpu


def make(**kw):
    args = dict(workers=3, width=64, hidden=200, classes=7, p=0.1, lr=0.2, seed=5, device=DEV, dtype=torch.float32)
    args.update(kw)
    return network.Network(**args)


def batch(net, it, rows=40):
    return synth.class_mixture(net.M, rows, net.shapes[0][1], net.shapes[2][0], 5, it, device=DEV)


def test_loss_falls_and_runs_repeat_bit_for_bit():
    runs = []
    for _ in range(2):
        net = make(dtype=torch.bfloat16)
        losses = []
        for it in range(40):
            x, labels = batch(net, it)
            losses.append(net.step(it, x.to(net.dtype), labels).mean().item())
        say(f"network: loss {losses[0]:.3f} -> {losses[-1]:.3f}")
        runs.append((losses, net.w.clone(), net.gref.clone()))
        x, labels = batch(net, 1000, rows=200)
        right = (net.forward(x.to(net.dtype), 0).argmax(-1) == labels).float().mean().item()
        net.close()
    # classes 8 deviations apart on average: a working iteration separates them, one that only shrinks weights stays at ln 7
    assert losses[-1] < 0.5 * losses[0] and right > 0.8
    assert runs[0][0] == runs[1][0] and torch.equal(runs[0][1], runs[1][1]) and torch.equal(runs[0][2], runs[1][2])


def test_an_iteration_against_the_oracle():
    net = make()
    it = 3
    x, labels = batch(net, it)
    w0 = net.w.clone()
    logits, kept = net.forward(x, it, keep=True)
    (w1, b1), (w2, b2), (w3, b3) = [(w.cpu().numpy(), b.cpu().numpy()) for w, b in net.layers(w0)]

    # forward: the oracle's codes of what the layer before handed on (teacher-forced: float32 sums of other orders move codes)
    def codes(v):
        q, s = L.codes(np.ascontiguousarray(v, dtype=np.float32), 2)
        return q, s[..., 0]

    M, rows = labels.shape
    shape1, shape2 = (M, rows, w1.shape[0]), (M, rows, w2.shape[0])
    xh = x.cpu().numpy()
    q1, s1 = codes(xh)
    assert np.array_equal(kept[1][0].qt.cpu().numpy(), np.swapaxes(q1, 1, 2))
    c1, t1 = codes(w1[None])
    h1 = L.product(q1, c1[0], s1, t1[0], b1).astype(np.float32)
    keep1 = L.kept(net.seed, it, 0, net.p, shape1)
    keep2 = L.kept(net.seed, it, 1, net.p, shape2)
    h1_device = kept[1][1].x.cpu().numpy()
    assert np.all(np.abs(h1_device - h1) <= 2.0 ** -20 * (np.abs(h1) + np.abs(b1)))
    q2, s2 = codes(L.dropped(h1_device, keep1, net.p, True))
    assert np.array_equal(kept[1][1].qt.cpu().numpy(), np.swapaxes(q2, 1, 2))
    c2, t2 = codes(w2[None])
    h2 = L.dropout(L.product(q2, c2[0], s2, t2[0], b2).astype(np.float32), keep2, net.p, False, xh)
    q3 = np.swapaxes(kept[1][2].qt.cpu().numpy(), 1, 2)
    s3 = kept[1][2].scale.cpu().numpy()
    assert np.all(np.abs(q3 * s3[..., None].astype(np.float64) - h2) <= s3[..., None] * (0.5 + 1e-3) + 2.0 ** -18 * np.abs(h2))
    c3, t3 = codes(w3[None])
    want = L.product(q3, c3[0], s3, t3[0], b3)
    assert np.all(np.abs(logits.cpu().numpy() - want) <= 2.0 ** -20 * (np.abs(want) + np.abs(b3)))

    # backward of the last layer from the device's own logits, and the coder's step from the device's own gradients
    loss = net.step(it, x, labels)
    z = logits.double().cpu().numpy()
    pr = np.exp(z - z.max(-1, keepdims=True))
    pr /= pr.sum(-1, keepdims=True)
    picked = np.take_along_axis(pr, labels.cpu().numpy()[..., None], -1)[..., 0]
    assert np.allclose(loss.cpu().numpy(), -np.log(picked).mean(1), rtol=1e-5)
    dl = pr.copy()
    np.put_along_axis(dl, labels.cpu().numpy()[..., None], picked[..., None] - 1, -1)
    dl /= rows
    dw3, db3 = (t.cpu().numpy().astype(np.float64) for t in net.layers(net.g)[2])
    exact = np.swapaxes(dl * s3[..., None], 1, 2) @ q3
    step = np.abs(dl * s3[..., None]).max(1)[..., None] / 127  # a drawn code is less than a step off
    assert np.all(np.abs(dw3 - exact) <= step * np.abs(q3.astype(np.float64)).sum(1)[:, None, :] * 1.001 + 1e-7)
    assert np.allclose(db3, dl.sum(1), atol=1e-6)
    cfg = O.Config(d=net.d, M=M, bits=4, norm=O.NORM_SUB, ref_policy=O.REF_LAST_AVG, ref_period=1, seed=net.seed, lr=0.2, batch=0)
    w, ref, c, s, v = O.step(cfg, it, w0.cpu().numpy(), np.zeros(net.d, np.float32), net.g.cpu().numpy())
    assert np.array_equal(net.w.cpu().numpy(), w) and np.array_equal(net.gref.cpu().numpy(), ref) and np.array_equal(net.scales.cpu().numpy(), s)
    net.close()
