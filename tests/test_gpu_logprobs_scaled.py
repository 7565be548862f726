"""Gradients of the entropy under a large loss scale, at entries of probability 0: masked ones, and ones far below the largest.
Tolerances as in test_gpu_logprobs.py, all of which are relative to the incoming gradients."""
import pytest
import torch

from test_gpu_logprobs import INF, check, logits_of, targets_for

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [2.0 ** 30, 2.0 ** 60, 2.0 ** 100])
def test_entries_of_probability_zero_have_no_gradient(scale, dtype):
    T, V = 6, 5000
    x = logits_of(T, V, dtype, 1, masked=0.3)
    x[1, :100] = -1e4                                  # no mask, but e^-1e4
    x[2, 5:] = torch.finfo(x.dtype).min
    x[3] = -INF
    targets = targets_for(T, V, 2)
    gen = torch.Generator(device="cuda").manual_seed(3)
    w, dE = (torch.randn((T,), generator=gen, device="cuda") * scale for _ in range(2))
    o = check(x, dtype, targets, d_logp=w, d_entropy=dE)
    d = o["d_logits"]
    assert d.isfinite().all()
    at = torch.zeros_like(x, dtype=torch.bool)
    rows = torch.nonzero(targets >= 0)[:, 0]
    at[rows, targets[rows].long()] = True              # (a masked target has the gradient of its own probability)
    assert (d[(x <= -1e4) & ~at] == 0).all()
