"""Logits that overflow to -infinity where rows and matrix are finite: probability 0, and nothing for the other columns, whatever the columns that
are summed together.  Tolerances as derived at the head of test_gpu_head.py, of the matrix without the column that overflows."""
import pytest
import torch
from test_gpu_head import HALF, backward, forward, inputs, near, reference

pytestmark = pytest.mark.gpu


# Columns are summed in groups of 16 and 64 (stream over the matrix), 64 (bf16: tiles of 128, float32: of 128), 128 (tiles of 256) and 32 (float32: tiles of
# 64): the last group has one column, the one that overflows.
@pytest.mark.parametrize("T,d,V,dtype", [(20, 64, 65, "bf16"), (20, 64, 65, "f32"), (1, 256, 4097, "bf16"), (60, 96, 641, "f32"), (1, 32, 1 + 1024, "f32"),
                                         (330, 64, 6401, "bf16"), (520, 512, 16001, "bf16"), (200, 512, 16001, "f32"), (249, 64, 131073, "f32")])
def test_a_last_column_that_overflows(T, d, V, dtype):
    print("overflow", T, d, V, dtype, flush=True)
    x, W, targets, w = inputs(T, d, V, dtype, T + V)
    x[:, 0] = 4.0
    W[V - 1] = 0.0
    W[V - 1, 0] = -3e38
    targets = torch.where(targets == V - 1, 0, targets)
    rest = W[:V - 1].contiguous()
    logp, log_z, G, tol, tol_z, tol_G = reference(x, rest, targets, w)
    a, b = forward(x, W, targets, dtype)
    near(a, logp, tol, "logp")
    near(b, log_z, tol_z, "log_z")
    lp, dX, dW = backward(x, W, targets, w, dtype)
    near(lp, logp, tol, "logp of the gradient's call")
    x64, W64 = x.double(), rest.double()
    size = G.abs() + tol_G
    kept = 2.0 ** -16 if dtype == "bf16" else 0.0
    bound = (tol_G + kept * size) @ W64.abs() + (2 * V + 2) * 2.0 ** -23 * (size @ W64.abs())
    want = G @ W64
    near(dX, want, bound + HALF[dtype] * (want.abs() + bound), "dX")
    assert (dW[V - 1] == 0).all()
    most = w[targets >= 0].double().abs().max() if (targets >= 0).any() else 0.0
    held = (2.0 ** -21 * size + 2.0 ** -39 * most) * (dtype == "bf16")
    St, Et = size.t().contiguous(), (tol_G + held).t().contiguous()
    tol_dW = Et @ x64.abs() + (dtype == "bf16") * St.sum(1, keepdim=True) * 2.0 ** -39 * x64.abs().max() + (2 * T + 2) * 2.0 ** -23 * (St @ x64.abs())
    want = G.t().contiguous() @ x64
    near(dW[:V - 1], want, tol_dW + 2.0 ** -24 * (want.abs() + tol_dW), "dW")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,V", [(20, 64, 320), (330, 64, 6400), (520, 512, 16000)])
def test_whole_groups_and_targets_that_overflow(T, d, V, dtype):
    """256 columns in a row; a target among them has log probability -infinity, all others are as without these columns."""
    if dtype == "f32" and T > 250:
        T = 250
    x, W, targets, w = inputs(T, d, V, dtype, T + V)
    x[:, 0] = 4.0
    W[:256, 1:], W[:256, 0] = 0.0, -3e38
    targets[(targets >= 0) & (targets < 256)] = 256
    logp, log_z, _, tol, tol_z, _ = reference(x, W[256:].contiguous(), torch.where(targets >= 0, targets - 256, targets), w)
    targets[0] = 17
    others = torch.arange(T, device="cuda") != 0
    a, b = forward(x, W, targets, dtype)
    lp, dX, dW = backward(x, W, targets, w, dtype)
    assert a[0] == -float("inf") and lp[0] == -float("inf")
    near(a[others], logp[others], tol[others], "logp")
    near(lp[others], logp[others], tol[others], "logp of the gradient's call")
    near(b, log_z, tol_z, "log_z")
    assert dX[others].isfinite().all() and not dW.isnan().any()
