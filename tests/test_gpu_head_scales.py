"""Rows of sizes far apart in log probabilities from hidden rows and their gradients.  What is held in float16 numbers goes by powers of two of each row's own, so a
row's log probabilities and dX do not depend on what stands in the others, and dW, which sums over them, loses what lies below 2^-39 of the largest |w_t| max|x_t|.
Tolerances as derived at the head of test_gpu_head.py, with a row's own weight and largest values in the place of all rows'."""
import pytest
import torch
from test_gpu_head import HALF, backward, forward, inputs, near, reference

pytestmark = pytest.mark.gpu

# stream, tiles of 128 and of 256, several pieces; float32: products in float32, pairs of float16 numbers (tiles of 128 and 256, several pieces)
SHAPES = [(60, 64, 700), (330, 64, 6401), (700, 320, 5003), (5000, 64, 4097), (900, 1024, 8001), (600, 32, 1 << 20)]


def bounds(x, W, targets, w, dtype, T):
    """What dX and dW may be off by, before they are rounded."""
    logp, log_z, G, tol, tol_z, tol_G = reference(x, W, targets, w)
    x64, W64, V = x.double(), W.double(), len(W)
    own = torch.where(targets >= 0, w.double().abs(), 0.0)[:, None]
    size = G.abs() + tol_G
    terms = size @ W64.abs()
    if dtype == "bf16":
        off = (tol_G + 2.0 ** -16 * size) @ W64.abs()
    else:       # by pairs: G in 22 bits and 2^-39 of the row's weight, W in 22 and 2^-39 of its largest, 2^-20 of each product in all
        off = tol_G @ W64.abs() + 2.0 ** -19 * terms + own * 2.0 ** -39 * (W64.abs().sum(0, keepdim=True) + V * W64.abs().max())
    off_dX = off + (2 * V + 2) * 2.0 ** -23 * terms
    most = float((own * x64.abs().amax(1, keepdim=True)).max())
    St, Et = size.t().contiguous(), tol_G.t().contiguous()
    off_dW = Et @ x64.abs() + ((2 * T + 2) * 2.0 ** -23 + 2.0 ** -19) * (St @ x64.abs()) + T * 2.0 ** -38 * most
    return logp, log_z, tol, tol_z, G @ W64, off_dX, G.t().contiguous() @ x64, off_dW


def check(x, W, targets, w, dtype, dW_too=True):
    T = len(x)
    logp, log_z, tol, tol_z, dX, off_dX, dW, off_dW = bounds(x, W, targets, w, dtype, T)
    a, b = forward(x, W, targets, dtype)
    near(a, logp, tol, "logp")
    near(b, log_z, tol_z, "log_z")
    lp, gx, gw = backward(x, W, targets, w, dtype)
    near(lp, logp, tol, "logp of the gradient's call")
    # (the weights' smallest here are 2^-40: all that underflows lies below 2^-100)
    near(gx, dX, off_dX + HALF[dtype] * (dX.abs() + off_dX) + 2.0 ** -100, "dX")
    if dW_too:
        near(gw, dW, off_dW + 2.0 ** -24 * (dW.abs() + off_dW) + 2.0 ** -100, "dW")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,V", SHAPES)
def test_weights_far_apart(T, d, V, dtype):
    print("weights far apart", T, d, V, dtype, flush=True)
    x, W, targets, w = inputs(T, d, V, dtype, T + V)
    check(x, W, targets, w * 2.0 ** torch.linspace(-40, 0, T, device="cuda"), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,V", SHAPES)
def test_rows_far_apart_whose_gradients_are_not(T, d, V, dtype):
    """Rows of 2^-30 under weights of 2^30, and back: all of them count in dW."""
    print("rows far apart", T, d, V, dtype, flush=True)
    x, W, targets, w = inputs(T, d, V, dtype, T + V + 1)
    by = (2.0 ** torch.linspace(0, 30, T, device="cuda").round())
    check((x.float() / by[:, None]).to(x.dtype), W, targets, w * by, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,V", SHAPES)
def test_one_large_row_with_a_target(T, d, V, dtype):
    """2^26 times the others, whose log probabilities and dX are what they are without it."""
    print("one large row", T, d, V, dtype, flush=True)
    x, W, targets, w = inputs(T, d, V, dtype, T + V + 2)
    targets[3] = 5
    others = torch.arange(T, device="cuda") != 3
    logp, _, tol, _, dX, off, _, _ = bounds(x, W, targets, w, dtype, T)
    was = forward(x, W, targets, dtype) + backward(x, W, targets, w, dtype)[:2]
    for large in (2.0 ** 26, 1e30):
        filled = x.clone()
        filled[3] = (x[3].float() * large).to(x.dtype)
        now = forward(filled, W, targets, dtype) + backward(filled, W, targets, w, dtype)[:2]
        assert all(torch.equal(p[others], q[others]) for p, q in zip(was, now))
        assert now[0][3].isfinite() and now[2][3].isfinite()
    near(now[2][others], logp[others], tol[others], "logp")
    near(now[3][others], dX[others], (off + HALF[dtype] * (dX.abs() + off))[others], "dX")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weights_of_nothing(dtype):
    """Rows with a target whose weight is 0 have no gradient and no part in dW, also where all of them are such."""
    for T, d, V in SHAPES[:4]:
        x, W, targets, w = inputs(T, d, V, dtype, T + V + 3)
        w[::3] = 0.0
        _, dX, dW = backward(x, W, targets, w, dtype)
        assert (dX[::3] == 0).all()
        large = x.clone()
        large[::3] *= 2.0 ** 60
        assert all(torch.equal(p, q) for p, q in zip((dX, dW), backward(large, W, targets, w, dtype)[1:]))
        _, dX, dW = backward(x, W, targets, torch.zeros_like(w), dtype)
        assert (dX == 0).all() and (dW == 0).all()
