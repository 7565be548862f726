"""Output matrices of float32 layers whose values lie far apart: a few rows that are far larger than the others, most values zeros, infinities.  Where parts in float16
numbers would lose the smaller ones the products are in float32.  Tolerances as derived at the head of test_gpu_head.py."""
import pytest
import torch
from test_gpu_head import backward, forward, inputs, near, reference

pytestmark = pytest.mark.gpu

# more rows than those from which on pairs of float16 numbers are taken; the last two: tiles of 256, several pieces
SHAPES = [(5000, 64, 4097), (300, 256, 50257), (450, 512, 20001), (900, 1024, 8001), (9000, 512, 1000), (70000, 256, 256), (4200, 32, 131072)]


def check(x, W, targets, w, without=0):
    """Against the matrix less its last `without` rows, whose logits have to be so low that they count for nothing."""
    T, V = len(x), len(W)
    rest = W[:V - without].contiguous()
    logp, log_z, G, tol, tol_z, tol_G = reference(x, rest, targets, w)
    a, b = forward(x, W, targets, "f32")
    near(a, logp, tol, "logp")
    near(b, log_z, tol_z, "log_z")
    lp, dX, dW = backward(x, W, targets, w, "f32")
    near(lp, logp, tol, "logp of the gradient's call")
    x64, W64 = x.double(), rest.double()
    size = G.abs() + tol_G
    terms = size @ W64.abs()
    want = G @ W64
    off = tol_G @ W64.abs() + ((2 * V + 2) * 2.0 ** -23 + 2.0 ** -19) * terms
    near(dX, want, off + 2.0 ** -24 * (want.abs() + off) + 2.0 ** -100, "dX")
    most = w[targets >= 0].double().abs().max()
    St = size.t().contiguous()
    off = tol_G.t().contiguous() @ x64.abs() + ((2 * T + 2) * 2.0 ** -23 + 2.0 ** -19) * (St @ x64.abs()) + T * 2.0 ** -38 * most * x64.abs().max()
    want = G.t().contiguous() @ x64
    near(dW[:V - without], want, off + 2.0 ** -24 * (want.abs() + off), "dW")
    assert (dW[V - without:] == 0).all()


@pytest.mark.parametrize("low", [-1e30, -3e38, -float("inf")])
@pytest.mark.parametrize("T,d,V", SHAPES)
def test_rows_that_mask_their_columns(T, d, V, low):
    """A column of x that is 1 and rows of W with a very low value there: what pads a vocabulary, say."""
    print("masked rows", T, d, V, low, flush=True)
    x, W, targets, w = inputs(T, d, V, "f32", T + V)
    x[:, 5] = 1.0
    W[V - 9:] = 0.0
    W[V - 9:, 5] = low
    targets = torch.where(targets >= V - 9, 1, targets)
    if low == -float("inf"):      # (0 times infinity: dX of such a column is NaN, as in float32)
        rest = W[:V - 9].contiguous()
        logp, log_z, _, tol, tol_z, _ = reference(x, rest, targets, w)
        a, b = forward(x, W, targets, "f32")
        near(a, logp, tol, "logp")
        near(b, log_z, tol_z, "log_z")
    else:
        check(x, W, targets, w, without=9)


@pytest.mark.parametrize("T,d,V", SHAPES)
def test_a_matrix_of_zeros_but_for_one_row(T, d, V):
    print("one row", T, d, V, flush=True)
    x, W, targets, w = inputs(T, d, V, "f32", T + V + 1)
    row = W[7].clone()
    W.zero_()
    W[7] = row
    check(x, W, targets, w)


@pytest.mark.parametrize("large", [2.0 ** 22, 2.0 ** 40, 2.0 ** 100])
@pytest.mark.parametrize("T,d,V", SHAPES)
def test_one_far_larger_row(T, d, V, large):
    """In columns that no row of x has, so that its own logit is 0, as are the other rows' values there."""
    print("larger row", T, d, V, large, flush=True)
    x, W, targets, w = inputs(T, d, V, "f32", T + V + 2)
    x[:, d // 2:] = 0.0
    W[:, d // 2:] = 0.0
    W[3] = 0.0
    W[3, d // 2:] = large
    check(x, W, targets, w)


def test_replays_with_ordinary_and_other_matrices():
    """A captured graph takes what the matrix asks for at each replay."""
    T, d, V = 450, 512, 20001
    import paper_2409_12210_amd as m
    x, W, targets, w = inputs(T, d, V, "f32", 9)
    ws = torch.empty(m.modse_head_workspace_size(T, d, V, "f32", m.WS_BWD), dtype=torch.uint8, device="cuda")
    lp, dX, dW = torch.empty(T, device="cuda"), torch.empty_like(x), torch.empty((V, d), device="cuda")
    call = lambda: m.modse_head_bwd(T, d, V, "f32", x, W, targets, w, lp, dX, dW, False, ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    ordinary, other = W.clone(), W.clone()
    x[:, 5] = 1.0
    other[V - 3:] = 0.0
    other[V - 3:, 5] = -1e30
    targets[targets >= V - 3] = 0
    for matrix in (ordinary, other, ordinary, other):
        W.copy_(matrix)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (lp, dX, dW)]
        for t in (lp, dX, dW):
            t.fill_(float("nan"))
        call()
        assert all(torch.equal(p, q) for p, q in zip(got, (lp, dX, dW)))
        want = reference(x, W[:V - 3].contiguous() if matrix is other else W, targets, w)
        near(lp, want[0], want[3], "logp")
