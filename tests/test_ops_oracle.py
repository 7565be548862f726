"""Pins of oracle/ops_oracle.py: against torch's own functions in float64, autograd, central differences and closed forms."""
import numpy as np
import pytest
import torch

from oracle import ops_oracle as orc

RNG = np.random.default_rng(7)


def t64(a):
    return torch.tensor(a, dtype=torch.float64)


def differences(f, x, step=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        hi, lo = x.copy(), x.copy()
        hi[i] += step
        lo[i] -= step
        g[i] = (f(hi) - f(lo)) / (2 * step)
    return g


@pytest.mark.parametrize("with_residual", [False, True])
def test_norm_is_torch_rms_norm_and_its_gradient_is_autograd(with_residual):
    x, gamma, dY, dH = RNG.normal(size=(5, 13)), RNG.normal(size=13), RNG.normal(size=(5, 13)), RNG.normal(size=(5, 13))
    res = RNG.normal(size=(5, 13)) if with_residual else None
    h, y, rstd = orc.norm_fwd(x, res, gamma, 1e-5)
    th = t64(h).requires_grad_()
    tg = t64(gamma).requires_grad_()
    ty = torch.nn.functional.rms_norm(th, (13,), tg, 1e-5)
    assert np.allclose(y, ty.detach().numpy(), rtol=1e-13, atol=1e-13)
    ((ty * t64(dY)).sum() + (th * t64(dH)).sum()).backward()
    dX, dgamma = orc.norm_bwd(h, gamma, rstd, dY, dH)
    assert np.allclose(dX, th.grad.numpy(), rtol=1e-11, atol=1e-12)
    assert np.allclose(dgamma, tg.grad.numpy(), rtol=1e-11, atol=1e-12)


def test_norm_gradient_is_that_of_differences():
    x, gamma, dY = RNG.normal(size=(2, 6)), RNG.normal(size=6), RNG.normal(size=(2, 6))
    h, _, rstd = orc.norm_fwd(x, None, gamma, 1e-3)
    dX, dgamma = orc.norm_bwd(h, gamma, rstd, dY)
    assert np.allclose(dX, differences(lambda v: (orc.norm_fwd(v, None, gamma, 1e-3)[1] * dY).sum(), x), atol=1e-8)
    assert np.allclose(dgamma, differences(lambda v: (orc.norm_fwd(x, None, v, 1e-3)[1] * dY).sum(), gamma), atol=1e-8)


def test_e4m3_values_are_those_of_the_type():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(orc.e4m3_values(codes), want, equal_nan=True)
    s, wide = orc.scales(np.array([[448.0, 1.0, -896.0, 0.0, 0.0]]), 2)
    assert np.array_equal(s, [[1.0, 2.0, 2.0 ** -126]]) and np.array_equal(wide[0, :4], [1, 1, 2, 2])


def test_logprobs_are_torch_log_softmax_entropy_topk_and_autograd():
    x = RNG.normal(size=(6, 31)) * 3
    x[1, :20] = -np.inf
    targets = np.array([3, 25, -1, 0, 30, 12])
    w, dE = RNG.normal(size=6), RNG.normal(size=6)
    logp, entropy, idx, value = orc.logprobs_fwd(x, targets, 5)
    tx = t64(x).requires_grad_()
    lp = torch.log_softmax(tx, 1)
    p = lp.exp()
    ent = -torch.where(p > 0, p * lp.masked_fill(p == 0, 0.0), 0.0).sum(1)
    want = torch.where(t64(targets) >= 0, lp[torch.arange(6), t64(targets).clamp_min(0).long()], 0.0)
    assert np.allclose(logp, want.detach().numpy(), atol=1e-13)
    assert np.allclose(entropy, ent.detach().numpy(), atol=1e-13)
    top = lp.topk(5, dim=1)
    assert np.array_equal(idx, top.indices.numpy()) and np.allclose(value, top.values.detach().numpy(), atol=1e-13)
    ((want * t64(w)).sum() + (ent * t64(dE)).sum()).backward()
    got = orc.logprobs_bwd(x, targets, w, dE)
    seen = np.isfinite(x)
    assert np.allclose(got[seen], np.nan_to_num(tx.grad.numpy())[seen], atol=1e-12) and (got[~seen] == 0).all()


def test_logprobs_gradient_is_that_of_differences():
    x, targets, w, dE = RNG.normal(size=(3, 7)), np.array([2, -1, 6]), RNG.normal(size=3), RNG.normal(size=3)

    def loss(v):
        logp, entropy, _, _ = orc.logprobs_fwd(v, targets)
        return (w * logp + dE * entropy).sum()
    assert np.allclose(orc.logprobs_bwd(x, targets, w, dE), differences(loss, x), atol=1e-8)


def test_logprobs_at_the_edges():
    none = -np.inf
    x = np.array([[none, none, none], [none, 2.0, none], [1.0, 1.0, 1.0], [0.0, -0.0, 5.0]])
    logp, entropy, idx, value = orc.logprobs_fwd(x, np.array([1, 1, 2, 3]), 4)
    assert logp[0] == none and logp[1] == 0 and np.isclose(logp[2], -np.log(3)) and np.isnan(logp[3])
    assert entropy[0] == 0 and entropy[1] == 0 and np.isclose(entropy[2], np.log(3))
    assert idx.tolist() == [[-1] * 4, [1, -1, -1, -1], [0, 1, 2, -1], [2, 0, 1, -1]]
    assert (value[0] == none).all() and value[2, 3] == none
    g = orc.logprobs_bwd(x[:3], np.array([1, 1, 2]), np.ones(3), np.ones(3))
    assert (g[:2] == 0).all() and np.allclose(g[2], [-1 / 3, -1 / 3, 2 / 3])


def test_orthogonalize_maps_singular_values_by_the_polynomials():
    u, _ = np.linalg.qr(RNG.normal(size=(9, 9)))
    v, _ = np.linalg.qr(RNG.normal(size=(14, 14)))
    s = np.linspace(0.1, 2.0, 9)
    G = (u * s) @ v[:9]
    coeffs = [(3.4445, -4.7750, 2.0315), (2.0, -1.5, 0.5), (1.875, -1.25, 0.375)]
    want = s / (np.sqrt((s * s).sum()) + 1e-3)
    for a, b, c in coeffs:
        want = a * want + b * want ** 3 + c * want ** 5
    for M, U, V in ((G, u, v[:9]), (G.T, v[:9].T, u.T)):
        assert np.allclose(orc.orthogonalize(M, coeffs, 1e-3), (U * want) @ V, atol=1e-12)
    # the quintic with p(1) = 1, p'(1) = p''(1) = 0 settles on the nearest matrix of orthonormal rows
    assert np.allclose(orc.orthogonalize(G, [(1.875, -1.25, 0.375)] * 40, 0.0), u @ v[:9], atol=1e-9)
    assert (orc.orthogonalize(np.zeros((3, 4)), coeffs, 1e-7) == 0).all()
