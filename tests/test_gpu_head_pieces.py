"""Log probabilities from hidden rows and their gradients of more rows than the workspace holds logits of: the batch goes by in pieces.  (The vocabulary
says how many rows a piece has: 256 at 2^20 columns, 2048 at 131072, 8192 at 32000; up to 65536 when scored.)"""
import pytest
import test_gpu_head as head
import torch

pytestmark = pytest.mark.gpu


# bf16, float32 by pairs of float16 numbers (a few hundred rows and more), and in float32 (more than 2^28 elements of W)
@pytest.mark.parametrize("T,d,V,dtype", [(600, 32, 1 << 20, "bf16"), (600, 32, 1 << 20, "f32"), (520, 288, 1 << 20, "f32"), (290, 32, 1 << 20, "f32"),
                                         (4200, 32, 131072, "bf16"), (4200, 32, 131072, "f32"), (2049, 64, 131001, "bf16"), (8193, 64, 31999, "bf16")])
def test_gradients_in_pieces(T, d, V, dtype):
    """Two and three of them, the last one shorter: against float64, added to what there is, dX in the buffer of x, either gradient alone, and the same
    bits again."""
    head.test_sums_are_added_to_and_results_are_the_same_bits_again(T, d, V, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_in_pieces(dtype):
    """Three pieces of 16384 rows at the most, against the rows by themselves."""
    T, d, V = 33000, 32, 1 << 20
    print("scores in pieces", dtype, flush=True)
    x, W, targets, _ = head.inputs(T, d, V, dtype, 3)
    logp, log_z = head.forward(x, W, targets, dtype)
    for first in (0, 11000, 16300, 22300, 32760):
        at = slice(first, first + 240)
        want = head.reference(x[at], W, targets[at], torch.ones(240, device="cuda"))
        head.near(logp[at], want[0], want[3], "logp", first)
        head.near(log_z[at], want[1], want[4], "log_z", first)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_pieces_than_there_are_tables_for(dtype):
    """Eighteen pieces; the tables of sixteen are there at a time."""
    T, d, V = 17 * 256 + 44, 32, 1 << 20
    print("many pieces", dtype, flush=True)
    x, W, targets, w = head.inputs(T, d, V, dtype, 5)
    lp, dX, dW = head.backward(x, W, targets, w, dtype)
    want_dW, tol_dW = (torch.zeros((V, d), dtype=torch.float64, device="cuda") for _ in range(2))
    W64, most_w = W.double(), w[targets >= 0].double().abs().max()
    for first in range(0, T, 256):
        at = slice(first, min(first + 256, T))
        logp, _, G, tol, _, tol_G = head.reference(x[at], W, targets[at], w[at])
        head.near(lp[at], logp, tol, "logp", first)
        size, x64 = G.abs() + tol_G, x[at].double()
        in_parts = 2.0 ** -21 * size + 2.0 ** -39 * most_w
        terms = size @ W64.abs()
        kept = in_parts if dtype == "f32" else 2.0 ** -16 * size
        bound = (tol_G + kept) @ W64.abs() + (2 * V + 2) * 2.0 ** -23 * terms
        if dtype == "f32":
            bound += 2.0 ** -20 * terms + size.sum(1, keepdim=True) * 2.0 ** -39 * W64.abs().max()
        want = G @ W64
        head.near(dX[at], want, bound + head.HALF[dtype] * (want.abs() + bound), "dX", first)
        St = size.t().contiguous()
        want_dW += G.t().contiguous() @ x64
        tol_dW += (tol_G + in_parts).t().contiguous() @ x64.abs() + St.sum(1, keepdim=True) * 2.0 ** -39 * x.double().abs().max()
        tol_dW += ((2 * T + 2) * 2.0 ** -23 + 2.0 ** -20 * (dtype == "f32")) * (St @ x64.abs())
    head.near(dW, want_dW, tol_dW + 2.0 ** -24 * (want_dW.abs() + tol_dW), "dW")
