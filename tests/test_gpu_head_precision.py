"""What the gradients of log probabilities from hidden rows keep of G, where no single entry of it decides.  Tolerances as derived at the head of
test_gpu_head.py; G of bf16 layers is two bf16 numbers for dX, each off by at most half a step of what the one before it leaves: 2^-16 of an entry."""
import pytest
import torch
from test_gpu_head import HALF, TYPE, backward, near, reference

pytestmark = pytest.mark.gpu


def wrong_tokens(T, d, V, dtype, n, seed):
    """Rows whose probability lies on n tokens that are not the target: whole numbers, exact logits."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    W = (torch.randint(-4, 5, (V, d), generator=gen, device="cuda") / 8.0).to(TYPE[dtype])
    likely = torch.randint(0, V, (T, n), generator=gen, device="cuda")
    x = torch.zeros((T, d), device="cuda")
    for k in range(n):
        x += 2 * (W[likely[:, k]].float() * 8).sign()       # each of them gets about d |w| out of it
    x = x.to(TYPE[dtype])
    targets = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    targets[T // 2] = -1
    return x, W, targets, torch.randn(T, generator=gen, device="cuda")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 5])
@pytest.mark.parametrize("T,d,V", [(7, 64, 500), (100, 64, 1003), (129, 96, 5000), (256, 128, 700), (300, 64, 9001), (700, 320, 5003), (1500, 256, 3001)])
def test_dX_where_the_probability_lies_on_other_tokens_than_the_target(T, d, V, n, dtype):
    print("wrong tokens", T, d, V, n, dtype, flush=True)
    x, W, targets, w = wrong_tokens(T, d, V, dtype, n, T + V + n)
    logp, _, G, tol, _, tol_G = reference(x, W, targets, w, exact=True)
    at = targets.clamp_min(0).long()[:, None]
    elsewhere = G.scatter(1, at, 0.0).abs().amax(1) > 0.1 * G.gather(1, at)[:, 0].abs()
    assert elsewhere[targets >= 0].double().mean() > 0.9      # it is what the test is about
    lp, dX, _ = backward(x, W, targets, w, dtype)
    near(lp, logp, tol, "logp")
    W64 = W.double()
    size = (G.abs() + tol_G) @ W64.abs()
    most = w[targets >= 0].double().abs().max()
    kept = 2.0 ** -16 * size if dtype == "bf16" else 2.0 ** -19 * size + 2.0 ** -38 * V * most * W64.abs().max()
    # (numbers below 2^-126, of G, its parts and the result, may be taken for 0: each of a term's three by that much of W)
    bound = tol_G @ W64.abs() + kept + (2 * V + 2) * 2.0 ** -23 * size + 2.0 ** -126 * (3 * V * W64.abs().max() + 1)
    want = G @ W64
    near(dX, want, bound + HALF[dtype] * (want.abs() + bound), "dX")
