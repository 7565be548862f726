"""The operators at both ends of a model and the dropout together with the layer, the norm and the update, as examples/tiny_lm.py uses
them: its gradients against the ones without them, and against differences."""
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))
import tiny_lm  # noqa: E402

pytestmark = pytest.mark.gpu

SMALL = dict(vocab=200, d_model=64, d_ff=(32, 96, 64, 64), batch=96)
NAMES = ("E", "Wout", "W1", "W3", "W2", "gamma1", "gamma2", "W_gate")


def data(seed, batch=96, vocab=200):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    tokens, targets = tiny_lm.text(batch, vocab, gen)
    targets[5] = -1
    return tokens, targets, gen


def gradients(m):
    return {n: getattr(m, "d" + n).double().reshape(-1).clone() for n in NAMES}


def test_gradients_are_those_of_the_model_without_them():
    """float32.  The two models differ in the order of sums alone: of 64 and 200 terms in the products at the end, of 200 exponentials and
    of a token's rows; what comes out goes through the layer, whose own products sum up to 96 terms.  2^-14 of a gradient's norm
    is 2^10 roundings."""
    tokens, targets, _ = data(3)
    a, b = tiny_lm.TinyLM(dtype="f32", **SMALL), tiny_lm.TinyLM(dtype="f32", ends=True, **SMALL)
    la, lb = float(a.loss_and_gradients(tokens, targets)), float(b.loss_and_gradients(tokens, targets))
    assert abs(la - lb) <= 2.0 ** -14 * la
    ga, gb = gradients(a), gradients(b)
    for n in NAMES:
        assert float((ga[n] - gb[n]).norm()) <= 2.0 ** -14 * float(ga[n].norm()), n
    # and the rows that no token chose have none
    chosen = torch.zeros(200, dtype=torch.bool, device="cuda").index_fill_(0, tokens, True)
    assert (b.dE[~chosen] == 0).all() and (b.dE[chosen] != 0).any(1).all()


@pytest.mark.parametrize("p", [0.0, 0.3])
def test_the_gradient_of_the_whole_is_that_of_differences(p):
    """float32, along directions that leave the routing alone, with one mask.  As for the model without them: two losses that are right to
    2^-18 of log V each, over 2 step, and the third derivative over a step of 2^-6 of the weights' own size, which the scale of
    what is kept makes 1 / (1 - p)^3 as large."""
    m = tiny_lm.TinyLM(dtype="f32", ends=True, dropout=p, **SMALL)
    tokens, targets, gen = data(4)
    m.loss_and_gradients(tokens, targets)
    grads = {n: g for n, g in gradients(m).items() if n in ("Wout", "W1", "W3", "W2", "gamma2")}
    for name, g in grads.items():
        w = getattr(m, name)
        way = torch.randn(w.shape, generator=gen, device="cuda") * w.float().std().clamp_min(0.05)
        before, step = w.clone(), 2.0 ** -6
        sides = []
        for sign in (1, -1):
            w.copy_(before + sign * step * way)
            sides.append(float(m.loss_and_gradients(tokens, targets)))
        w.copy_(before)
        quotient, along = (sides[0] - sides[1]) / (2 * step), float((g.view(w.shape) * way.double()).sum())
        tol = 2.0 ** -18 * 6 / step + 6 * step ** 2 / (1 - p) ** 3
        assert abs(quotient - along) <= tol, (name, quotient, along, tol)


def test_a_step_makes_another_mask_and_changes_the_weights():
    m = tiny_lm.TinyLM(dtype="bf16", ends=True, dropout=0.5, **SMALL)
    tokens, targets, _ = data(5)
    before = {n: getattr(m, n).clone() for n in NAMES}
    first = float(m.loss_and_gradients(tokens, targets))
    assert float(m.loss_and_gradients(tokens, targets)) == first            # the same mask
    m.step(tokens, targets)
    for n in NAMES:
        # (of a bf16 gamma at 1 a step of less than 2^-9 is nothing)
        assert getattr(m, n).isfinite().all() and (n in ("gamma1", "gamma2") or not torch.equal(getattr(m, n), before[n])), n
        getattr(m, n).copy_(before[n])
    assert float(m.loss_and_gradients(tokens, targets)) != first
    # serving: nothing is dropped, and fewer tokens than a batch
    idx, logp, entropy = m.alternatives(tokens[:7], 3)
    again = m.alternatives(tokens[:7], 3)
    assert torch.equal(logp, again[1]) and torch.equal(idx, again[0]) and logp.isfinite().all()


def test_a_captured_training_pass_gives_the_eager_gradients_with_every_offset():
    m = tiny_lm.TinyLM(dtype="bf16", ends=True, dropout=0.2, **SMALL)
    tokens, targets, _ = data(6)
    m.loss_and_gradients(tokens, targets)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.loss_and_gradients(tokens, targets)
    for offset in range(4):
        t, u, _ = data(10 + offset)
        tokens.copy_(t)
        targets.copy_(u)
        m.rng[1] = offset
        graph.replay()
        torch.cuda.synchronize()
        got, logp = gradients(m), m.logp.clone()
        m.loss_and_gradients(tokens, targets)
        torch.cuda.synchronize()
        want = gradients(m)
        assert torch.equal(logp, m.logp) and all(torch.equal(got[n], want[n]) for n in NAMES)


def test_tied_matrices_take_both_gradients_in_one_buffer():
    m = tiny_lm.TinyLM(dtype="f32", ends=True, **SMALL)
    modse = tiny_lm.modse
    tokens, targets, _ = data(7)
    m.loss_and_gradients(tokens, targets)
    both = m.dWout.clone()
    modse.modse_embed_bwd(m.T, m.d, m.V, "f32", tokens.int(), m.dh1, 1.0, both, True, m.ws)
    want = m.dWout.double() + m.dE.double()
    # a rounding of the sum, and those of the sums of up to 96 rows in another place
    assert ((both.double() - want).abs() <= 2.0 ** -24 * (want.abs() + 98 * 2 * m.dh1.abs().double().sum(0))).all()


def test_the_command_runs():
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "tiny_lm.py"), "--steps", "3", "--ends", "--dropout", "0.1"],
                       capture_output=True, text=True, timeout=110)
    assert r.returncode == 0 and "after 3" in r.stdout, r.stdout + r.stderr
