"""Gradients against differences, along the gradient itself, where a wrong one cannot hide: a gradient that is zero, or turned, or
lacks a term is off by as much as the slope.

Q(s) = (f(x + s d) - f(x - s d)) / 2s with d = g / |g| should be |g|.  Its error is that of the two values over s, and c s^2 of the
curvature, which Q(s/2) has a quarter of: (4 Q(s/2) - Q(s)) / 3 is without it, and what is left of it is below their difference, as long as
that is small.  With values right to e the tolerance is 3 e / s + |Q(s) - Q(s/2)|, and every slope has to be ten times its tolerance."""
import os
import sys

import pytest
import torch

import paper_2409_12210_amd as m
from test_gpu_logprobs import logits_of, run, targets_for

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import tiny_lm  # noqa: E402

pytestmark = pytest.mark.gpu


def holds(along, s, wide, narrow, e, what):
    tol = 3 * e / s + abs(wide - narrow)
    assert abs(along) > 10 * tol, (what, "no power", along, wide, narrow, tol)
    assert abs((4 * narrow - wide) / 3 - along) <= tol, (what, along, wide, narrow, tol)


@pytest.mark.parametrize("name", ["Wout", "W1", "W3", "W2", "gamma2", "E"])
def test_weights_of_a_routed_model(name):
    """float32.  The mean loss of 96 tokens is right to 2^-20 of log V, 6.  Where the weight is in front of the router the step is the largest
    one (of halves) that leaves the routing alone."""
    slope_of_the_model(name, tiny_lm.TinyLM(vocab=200, d_model=64, d_ff=(32, 96, 64, 64), dtype="f32", batch=96))


@pytest.mark.parametrize("name", ["Wout", "W1", "W3", "W2", "gamma2", "gamma1", "E", "W_gate"])
def test_weights_of_a_model_whose_tokens_go_to_all_experts(name):
    """Both experts of two: nothing jumps, whatever happens in front of the router.  The experts are large enough to be heard beside the
    embeddings."""
    model = tiny_lm.TinyLM(vocab=200, d_model=64, d_ff=(96, 64), dtype="f32", batch=96)
    for w in (model.W1, model.W3, model.W2):
        w *= 4
    slope_of_the_model(name, model)


def slope_of_the_model(name, model):
    gen = torch.Generator(device="cuda").manual_seed(3)
    tokens, targets = tiny_lm.text(96, 200, gen)
    targets[5] = -1
    model.loss_and_gradients(tokens, targets)
    w, g = getattr(model, name), getattr(model, "d" + name).clone()
    g = g.view(w.shape)
    size = float(g.double().norm())
    assert size > 0

    def routes():
        return model.routing.topk_idx.sort(1).values
    before, there, way = w.clone(), routes(), g / size
    for halves in range(9, 15):
        s = 2.0 ** -halves / size                  # the loss changes by 2^-halves, about
        found, same = [], True
        for step in (s, s / 2):
            values = []
            for sign in (1, -1):
                w.copy_(before + sign * step * way)
                values.append(float(model.loss_and_gradients(tokens, targets)))
                same = same and torch.equal(routes(), there)
            found.append((values[0] - values[1]) / (2 * step))
        w.copy_(before)
        if same:
            break
    assert same
    holds(size, s, *found, 6 * 2.0 ** -20, name)


@pytest.mark.parametrize("part", ["logp", "entropy", "both"])
@pytest.mark.parametrize("T,V", [(5, 333), (3, 20011)])
def test_log_probabilities_and_entropy(T, V, part):
    """A row's outputs are right to 2^-20 of their size and of the logits', 16 in all at the most."""
    x, targets = logits_of(T, V, "f32", 1), targets_for(T, V, 3)
    gen = torch.Generator(device="cuda").manual_seed(2)
    w, dE = torch.rand(T, generator=gen, device="cuda") + 0.5, torch.rand(T, generator=gen, device="cuda") + 0.5
    if part == "logp":
        dE = None
    if part == "entropy":
        w = torch.zeros(T, device="cuda")
    g = run(x, "f32", targets, d_logp=w, d_entropy=dE)["d_logits"]
    size = float(g.double().norm())
    way = g / size

    def value(at):
        o = run(at, "f32", targets)
        return float((w.double() * o["logp"].double()).sum() + (0 if dE is None else (dE.double() * o["entropy"].double()).sum()))
    s = 2.0 ** -4
    found = [(value(x + step * way) - value(x - step * way)) / (2 * step) for step in (s, s / 2)]
    holds(size, s, *found, T * 16 * 2.0 ** -20, part)


@pytest.mark.parametrize("wrt", ["x", "gamma"])
@pytest.mark.parametrize("T,d", [(8, 264), (600, 40), (3, 4104)])
def test_norm(T, d, wrt):
    """<dY, y> of T d values of size 1 with roundings of 2^-22 in the mean: right to 2^-22 of the root of their number, four times that."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    x, gamma, dY = rand(T, d), 1 + 0.1 * rand(d), rand(T, d)
    rstd, y, dX, dgamma = torch.empty(T, device="cuda"), torch.empty_like(x), torch.empty_like(x), torch.empty(d, device="cuda")
    m.modse_norm_fwd(T, d, "f32", x, None, gamma, 1e-5, y, None, rstd)
    ws = torch.empty(m.modse_norm_bwd_workspace_size(T, d, "f32"), dtype=torch.uint8, device="cuda")
    m.modse_norm_bwd(T, d, "f32", x, gamma, rstd, dY, None, dX, dgamma, False, ws)
    g = dX if wrt == "x" else dgamma
    size = float(g.double().norm())
    way = g / size

    def value(step):
        at = (x + step * way, gamma) if wrt == "x" else (x, gamma + step * way)
        m.modse_norm_fwd(T, d, "f32", at[0], None, at[1], 1e-5, y, None, None)
        return float((y.double() * dY.double()).sum())
    s = 2.0 ** -2
    found = [(value(step) - value(-step)) / (2 * step) for step in (s, s / 2)]
    holds(size, s, *found, 4 * 2.0 ** -22 * (T * d) ** 0.5, wrt)
