"""The example that runs the lookup, its gradient, the averaging, Muon and LAMB
together: the model learns, and its gradients in the accumulator are
autograd's."""

import importlib.util
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_lm.py")


def example():
    spec = importlib.util.spec_from_file_location("train_lm", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_loss_falls():
    losses = example().train(rounds=60, peers=3)
    # a uniform guess is log(500) = 6.2; the next token is a function of the last
    assert losses[0] > 5.5 and np.mean(losses[-5:]) < 0.5 * losses[0]


def test_accumulated_gradients_are_autograds():
    """fp32 sums of at most 2048 terms in two orders: 2048 * 2^-24 of their magnitudes, here of the largest."""
    ex = example()
    model = ex.Model("cuda")
    acc = torch.zeros_like(model.x)
    batches = [ex.text(200, torch.Generator(device="cuda").manual_seed(k)) for k in range(3)]
    want = torch.zeros_like(model.x, dtype=torch.float64)
    for ids, target in batches:
        model.gradients(ids, target, acc)
        w1, w2, table, gain = (p.detach().double().requires_grad_() for p in model.views(model.x))
        rows = torch.where((ids >= 0)[..., None], table[ids.clamp(min=0)] * ex.SCALE, 0.0)
        hidden = torch.tanh(rows.view(len(ids), -1) @ w1.t()) * gain
        loss = torch.nn.functional.cross_entropy(hidden @ w2.t(), target)
        grads = torch.autograd.grad(loss, [w1, w2, table, gain])
        for a, g in zip(model.views(want), grads):
            a += len(ids) * g
    for a, w in zip(model.views(acc), model.views(want)):
        assert float((a.double() - w).abs().max()) <= 2048 * 2.0 ** -24 * float(w.abs().max())
