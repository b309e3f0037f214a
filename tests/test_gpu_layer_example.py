"""The layer operators together with the store: examples/layer_training_step.py learns, and its gradients are those
of the quantised layer in 64 bits."""
import os
import sys

import numpy as np
import pytest
import torch

import mx_reference as mx

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))


def test_training_reduces_the_loss():
    """The target has variance 1 per output and the layer starts at random, so the loss starts near 2.  Four bits leave an
    error of a few per cent of the product; 40 rounds of gradient descent have to bring it below a quarter of the start."""
    import layer_training_step as ex
    losses, layer, x = ex.train(rounds=40, frames=1000, width_in=256, width_out=320)
    assert np.isfinite(losses).all()
    assert losses[-1] < 0.25 * losses[0], losses
    assert int(layer.status[0]) == 0 and layer.plan.status() == 0
    layer.load()
    batch = layer.forward(x)
    for i in (0, 7, 999):
        # one frame alone: the same quantised operands, exact products; the sums may be taken in another order
        one = layer.frame(x[i:i + 1])[0].double()
        assert float((one - batch[i].double()).abs().max()) <= 2.0 ** -7 * float(batch[i].double().abs().max())


def test_gradients_reach_the_arena():
    import layer_training_step as ex
    frames, k, n = 300, 200, 144
    layer = ex.Layer(k, n, frames, seed=3)
    rng = np.random.default_rng(3)
    x = torch.from_numpy(rng.standard_normal((frames, k))).to(torch.bfloat16).cuda()
    dy = torch.from_numpy(rng.standard_normal((frames, n))).to(torch.bfloat16).cuda()
    layer.load()
    y = layer.forward(x).double().cpu().numpy()
    layer.backward(x, dy)
    torch.cuda.synchronize()
    host = lambda t: t.double().cpu().numpy()
    w, normed, d = host(layer.view(layer.full, 0)).reshape(n, k), host(layer.normed), host(dy)
    # products of quantised operands: K 2^-23 of the sums of magnitudes, and BF16's half unit
    for got, a, b, unit in ((y, mx.quantised(normed), mx.quantised(w).T, 2.0 ** -8),
                            (host(layer.dnormed), mx.quantised(d), mx.quantised(w.T).T, 2.0 ** -8),
                            (host(layer.view(layer.grads, 0)).reshape(n, k), mx.quantised(d.T), mx.quantised(normed.T).T, 2.0 ** -24)):
        want, size = a @ b, np.abs(a) @ np.abs(b)
        assert (np.abs(got - want) <= a.shape[1] * 2.0 ** -23 * size + unit * np.abs(want) + 1e-30).all()
    xhat = (host(x) - host(layer.mean[:frames])[:, None]) * host(layer.rstd[:frames])[:, None]
    dn = host(layer.dnormed)
    deep = (148 + frames / 16 + 100) * 2.0 ** -24
    assert (np.abs(host(layer.view(layer.grads, 1)) - (dn * xhat).sum(0)) <= deep * np.abs(dn * xhat).sum(0)).all()
    assert (np.abs(host(layer.view(layer.grads, 2)) - dn.sum(0)) <= deep * np.abs(dn).sum(0)).all()
