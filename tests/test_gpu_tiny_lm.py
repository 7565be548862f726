"""The operators and the layer together, as examples/tiny_lm.py uses them: the gradient of the whole against differences, and a loss
that falls."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import tiny_lm  # noqa: E402

pytestmark = pytest.mark.gpu


def test_the_gradient_of_the_whole_is_that_of_differences():
    """float32, along directions that leave the routing alone.  A directional derivative from two losses that are right to 2^-18 of
    log V each, over 2 step, and the third derivative over a step of 2^-6 of weights' own size."""
    m = tiny_lm.TinyLM(vocab=200, d_model=64, d_ff=(32, 96, 64, 64), dtype="f32", batch=96)
    gen = torch.Generator(device="cuda").manual_seed(3)
    tokens, targets = tiny_lm.text(96, 200, gen)
    targets[5] = -1
    m.loss_and_gradients(tokens, targets)
    grads = {"Wout": m.dWout.clone(), "W1": m.dW1.clone(), "W3": m.dW3.clone(), "W2": m.dW2.clone(), "gamma2": m.dgamma2.clone()}
    for name, g in grads.items():
        w = getattr(m, name)
        way = torch.randn(w.shape, generator=gen, device="cuda") * w.float().std().clamp_min(0.05)
        before, step = w.clone(), 2.0 ** -6
        sides = []
        for sign in (1, -1):
            w.copy_(before + sign * step * way)
            sides.append(float(m.loss_and_gradients(tokens, targets)))
        w.copy_(before)
        quotient, along = (sides[0] - sides[1]) / (2 * step), float((g.view(w.shape).double() * way.double()).sum())
        tol = 2.0 ** -18 * 6 / step + 6 * step ** 2
        assert abs(quotient - along) <= tol, (name, quotient, along, tol)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_model_learns(dtype):
    m = tiny_lm.TinyLM(dtype=dtype)
    gen = torch.Generator(device="cuda").manual_seed(1)
    losses = [float(m.step(*tiny_lm.text(m.T, m.V, gen))) for _ in range(40)]
    assert abs(losses[0] - 6.24) < 0.5          # log 512: it knows nothing
    assert losses[-1] < losses[0] - 1.0, losses
    idx, logp, entropy = m.alternatives(torch.arange(64, device="cuda"), 5)
    assert (logp.diff(dim=1) <= 0).all() and (entropy > 0).all()
    right = (idx[:, 0].long() == (5 * torch.arange(64, device="cuda") + 3) % m.V).float().mean()
    assert right > 0.5
