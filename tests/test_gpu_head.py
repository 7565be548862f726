"""Log probabilities from hidden rows and the output matrix, and their gradients, against the formulas in float64.

Tolerances.  A logit is a sum of d products in float32, whose instructions drop what lies 2^-23 below a partial sum: off by at most
e = (d + 6) 2^-23 sum |x W| (0 where the inputs are whole numbers whose sums float32 holds); four of these stand for float32 matrices that are
held as pairs of float16 ones: 2^-23 of each factor, and 2^-22 of the product of the second parts, which is left out.  Sums of exponentials: V terms of one sign,
joined in groups, under 2^9 roundings each with an exponential of relative error 2 u + |z| u whose weight falls as e^z: 2^-14 at the
worst.  So log Z and log p are off by a = e_max + e_target + 2^-14 + 2^-22 (|l| + |log p|), and p relatively by as much (and 2^-21 |log p|).
G = w (1[target] - p) adds 2^-22 |w| at the target.  For dX of bf16 layers it is rounded to half a step of bf16, but for the target's
entry, and all of them up to 128 rows, which are held to 2^-16.  For dW of bf16 layers it is held to
2^-22 of each value (2^-21 with the product by its scale) and 2^-39 of the largest weight, and x to 2^-39 of its largest value; so are, of
many rows of float32 layers, G, x and W, and to 2^-22 of each value.  The products sum in float32: (terms + 2) 2^-23 of the sum of the absolute values; a result is rounded to its type."""
import numpy as np
import pytest
import torch

import paper_2409_12210_amd as m
from oracle import ends_oracle as orc

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
NAN = float("nan")


def inputs(T, d, V, dtype, seed, sigma=2.5, whole=False):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if whole:   # sums of whole numbers, in steps of 2^-3: exact in float32
        x = torch.randint(-2, 3, (T, d), generator=gen, device="cuda").to(TYPE[dtype])
        W = (torch.randint(-2, 3, (V, d), generator=gen, device="cuda") / 8.0).to(TYPE[dtype])
    else:
        x = torch.empty((T, d), dtype=TYPE[dtype], device="cuda").normal_(0.0, 1.0, generator=gen)
        W = torch.empty((V, d), dtype=TYPE[dtype], device="cuda").normal_(0.0, sigma / d ** 0.5, generator=gen)
    targets = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    if T > 2:
        targets[T // 2] = -1
        targets[T - 1] = V - 1
    w = torch.randn(T, generator=gen, device="cuda")
    return x, W, targets, w


def workspace(T, d, V, dtype, which, shift=0):
    n = m.modse_head_workspace_size(T, d, V, dtype, which)
    ws = torch.empty(n + shift + 64, dtype=torch.uint8, device="cuda").fill_(255)
    return ws[shift:shift + n], ws[shift + n:]


def forward(x, W, targets, dtype, logp=True, log_z=True):
    (T, d), V = x.shape, len(W)
    ws, behind = workspace(T, d, V, dtype, m.WS_FWD, 16)
    a, b = (torch.full((T + 3,), NAN, device="cuda") if on else None for on in (logp, log_z))
    m.modse_head_fwd(T, d, V, dtype, x, W, targets, a[:T] if logp else None, b[:T] if log_z else None, ws)
    assert (behind == 255).all() and all(t is None or t[T:].isnan().all() for t in (a, b))
    return a[:T] if logp else None, b[:T] if log_z else None


def backward(x, W, targets, w, dtype, dX=True, dW=True, old=None, inplace=False):
    (T, d), V = x.shape, len(W)
    ws, behind = workspace(T, d, V, dtype, m.WS_BWD, 16)
    logp = torch.full((T,), NAN, device="cuda")
    gx = torch.full((T + 1, d), 3.0, dtype=x.dtype, device="cuda") if dX else None
    gw = torch.full((V + 2, d), 3.0, device="cuda") if dW else None
    if old is not None:
        gw[:V] = old
    if inplace:
        gx[:T] = x
        x = gx[:T]
    m.modse_head_bwd(T, d, V, dtype, x, W, targets, w, logp, gx[:T] if dX else None, gw[:V] if dW else None, old is not None, ws)
    assert (behind == 255).all() and (gx is None or (gx[T:] == 3.0).all()) and (gw is None or (gw[V:] == 3.0).all())
    return logp, gx[:T] if dX else None, gw[:V] if dW else None


def reference(x, W, targets, w, exact=False):
    """logp, log Z, G and the bounds of logp, log Z, and of G as it is computed."""
    x, W, w = x.double(), W.double(), w.double()
    d = x.shape[1]
    logits = x @ W.t().contiguous()
    e = 0.0 if exact else ((d + 6) * 2.0 ** -23) * (x.abs() @ W.abs().t().contiguous())
    at, has = targets.clamp_min(0).long()[:, None], targets >= 0
    log_z = logits.logsumexp(1)
    logp = logits.gather(1, at)[:, 0] - log_z
    most = 0.0 if exact else e.amax(1)
    size = 2.0 ** -14 + 2.0 ** -22 * logits.abs().amax(1)
    tol_z = most + size
    tol = 2 * most + size + 2.0 ** -22 * logp.abs()
    lp = logits - log_z[:, None]
    p = lp.exp()
    ww = torch.where(has, w, 0.0)[:, None]
    G = -ww * p
    G.scatter_add_(1, at, ww)
    rel = (2 * most + size)[:, None] + 2.0 ** -21 * lp.abs()
    tol_G = ww.abs() * p * rel.expm1()
    tol_G.scatter_add_(1, at, 2.0 ** -22 * ww.abs())
    return torch.where(has, logp, 0.0), log_z, G, torch.where(has, tol, 0.0), tol_z, tol_G


def near(got, want, tol, what, *tag):
    err = (got.double() - want).abs()
    ok = err <= tol
    assert ok.all(), (what,) + tag + (int((~ok).sum()), float(err[~ok].max()) if err[~ok].numel() else NAN, torch.nonzero(~ok)[:3].tolist())


def check(T, d, V, dtype, seed=0, whole=False, sigma=2.5, times_x=1.0, times_w=1.0):
    print("head", T, d, V, dtype, whole, times_x, times_w, flush=True)
    x, W, targets, w = inputs(T, d, V, dtype, seed, sigma, whole)
    x, W, w = x * times_x, W / times_x, w * times_w
    logp, log_z, G, tol, tol_z, tol_G = reference(x, W, targets, w, whole)
    got = forward(x, W, targets, dtype)
    near(got[0], logp, tol, "logp", T, d, V, dtype)
    near(got[1], log_z, tol_z, "log_z", T, d, V, dtype)
    assert torch.equal(forward(x, W, targets, dtype, log_z=False)[0], got[0]) and torch.equal(forward(x, W, targets, dtype, logp=False)[1], got[1])

    lp, dX, dW = backward(x, W, targets, w, dtype)
    near(lp, logp, tol, "logp of the gradient's call", T, d, V, dtype)
    x64, W64 = x.double(), W.double()
    size = G.abs() + tol_G
    rounded = torch.zeros_like(size)
    most_w = w[targets >= 0].double().abs().max() if (targets >= 0).any() else 0.0
    in_parts = 2.0 ** -21 * size + 2.0 ** -39 * most_w
    pairs = dtype == "f32" and T > 128
    if dtype == "bf16":
        rounded = size * (2.0 ** -16 if T <= 128 else HALF[dtype])
        at = targets.clamp_min(0).long()[:, None]
        rounded.scatter_(1, at, 2.0 ** -16 * size.gather(1, at))
    elif pairs:
        rounded = in_parts
    terms = size @ W64.abs()
    tol_dX = (tol_G + rounded) @ W64.abs() + (V + 2) * 2.0 ** -23 * terms
    if pairs:
        tol_dX += 2.0 ** -20 * terms + size.sum(1, keepdim=True) * 2.0 ** -39 * W64.abs().max()
    want = G @ W64
    near(dX, want, tol_dX + HALF[dtype] * (want.abs() + tol_dX), "dX", T, d, V, dtype)
    held = dtype == "bf16" or pairs
    Gt, St, Et = G.t().contiguous(), size.t().contiguous(), (tol_G + held * in_parts).t().contiguous()
    terms = St @ x64.abs()
    tol_dW = Et @ x64.abs() + held * St.sum(1, keepdim=True) * 2.0 ** -39 * x64.abs().max() + (2 * T + 2) * 2.0 ** -23 * terms
    if pairs:
        tol_dW += 2.0 ** -20 * terms
    want = Gt @ x64
    near(dW, want, tol_dW + 2.0 ** -24 * (want.abs() + tol_dW), "dW", T, d, V, dtype)
    return x, W, targets, w, dX, dW, want, tol_dW


# A stream over W where a few rows or a small vocabulary make few blocks, tiles of 128 x 128 or 256 x 256 (float32: 64 or 128) beyond; dX in two parts up to 128
# rows; dW's sum in parts where the vocabulary is small
SHAPES = [(1, 32, 1), (1, 64, 7), (2, 32, 31), (3, 96, 32), (5, 64, 33), (16, 128, 100), (17, 32, 255), (33, 96, 257), (64, 2048, 700),
          (65, 512, 1023), (63, 64, 8191), (49, 256, 64), (32, 32, 65), (129, 64, 1500), (255, 64, 300), (257, 128, 1000), (300, 256, 5003),
          (1000, 64, 4097), (40, 96, 50257), (4, 4096, 9001), (128, 96, 513), (192, 64, 777), (520, 96, 31), (70, 64, 40000), (65, 512, 33000),
          (128, 32, 16500), (129, 96, 20011), (200, 64, 12345), (257, 128, 9001), (520, 32, 5003), (700, 160, 3333), (2100, 64, 1001),
          (3000, 256, 256), (4100, 32, 32), (700, 320, 5003), (1000, 288, 20011), (1025, 256, 4099), (1024, 256, 4099)]
# float32 by pairs of float16 numbers, from the rows on where that is faster
PAIRS = [(5000, 64, 4097), (2600, 160, 3333), (10001, 64, 4097), (300, 256, 50257), (300, 2048, 32000), (520, 96, 131073), (9000, 512, 1000),
         (70000, 256, 256), (450, 512, 20001), (900, 1024, 8001)]


@pytest.mark.parametrize("T,d,V", PAIRS)
def test_float32_by_pairs(T, d, V):
    check(T, d, V, "f32", seed=T + V)
    check(T, d, V, "f32", seed=T + V + 1, whole=d <= 512)
    check(T, d, V, "bf16", seed=T + V)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,V", SHAPES)
def test_log_probabilities_and_gradients(T, d, V, dtype):
    check(T, d, V, dtype, seed=T + V)
    check(T, d, V, dtype, seed=T + V + 1, whole=d <= 512)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,V", [(1, 32, 5), (70, 64, 333), (300, 256, 2000), (9001, 32, 100), (700, 96, 5003), (5001, 64, 4097), (40, 64, 9000)])
def test_sums_are_added_to_and_results_are_the_same_bits_again(T, d, V, dtype):
    """Also more rows than a piece has; also dX in the buffer of x, and either gradient alone."""
    x, W, targets, w, dX, dW, want, tol = check(T, d, V, dtype, seed=7)
    old = torch.randn((V, d), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    got = backward(x, W, targets, w, dtype, old=old)
    near(got[2], want + old, tol + 2.0 ** -23 * ((want + old).abs() + tol + old.abs() + want.abs()), "dW added", T, d, V, dtype)
    again = backward(x, W, targets, w, dtype, old=old)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    assert torch.equal(got[1], dX)
    alone = backward(x, W, targets, w, dtype, dX=False)[2], backward(x, W, targets, w, dtype, dW=False)[1]
    assert torch.equal(alone[0], dW) and torch.equal(alone[1], dX)
    there = backward(x, W, targets, w, dtype, inplace=True)
    assert torch.equal(there[1], dX) and torch.equal(there[2], dW)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("times_x,times_w", [(2.0 ** -40, 1.0), (2.0 ** 40, 1.0), (1.0, 2.0 ** -60), (1.0, 2.0 ** 60), (2.0 ** -40, 2.0 ** 60),
                                             (2.0 ** 40, 2.0 ** -60), (2.0 ** -60, 2.0 ** -30), (2.0 ** 30, 2.0 ** 60), (1.0, 0.0)])
def test_rows_and_gradients_of_any_size(times_x, times_w, dtype):
    """Powers of two leave the logits as they are."""
    check(70, 64, 300, dtype, seed=13, times_x=times_x, times_w=times_w)
    check(200, 64, 300, dtype, seed=14, times_x=times_x, times_w=times_w)
    check(4800, 96, 2900, dtype, seed=15, times_x=times_x, times_w=times_w)


@pytest.mark.parametrize("dtype,T", [("bf16", 64), ("bf16", 200), ("f32", 200), ("f32", 5000), ("bf16", 5000)])
def test_weights_and_rows_of_sizes_far_apart(dtype, T):
    d, V = 64, 300 if T < 1000 else 4097
    x, W, targets, w = inputs(T, d, V, dtype, 14)
    w = w * 2.0 ** torch.linspace(-30, 0, T, device="cuda")
    x[::3] *= 2.0 ** -12
    logp, log_z, G, tol, tol_z, tol_G = reference(x, W, targets, w)
    lp, dX, dW = backward(x, W, targets, w, dtype)
    x64, size = x.double(), G.abs() + tol_G
    tol_dW = 2.0 ** -20 * (size.t().contiguous() @ x64.abs()) + (tol_G + 2.0 ** -21 * size + 2.0 ** -39 * w.abs().max()).t().contiguous() @ x64.abs() + (
        size.t().sum(1, keepdim=True) * 2.0 ** -39 * x64.abs().max()) + (2 * T + 3) * 2.0 ** -23 * (size.t().contiguous() @ x64.abs())
    near(dW, G.t().contiguous() @ x64, tol_dW, "dW")
    want = G @ W.double()
    half = HALF[dtype] if dtype == "bf16" else 2.0 ** -20
    near(dX, want, (tol_G + half * size + 2.0 ** -39 * w.abs().max()) @ W.double().abs() * 1.01 + half * want.abs() * 1.01 + (V + 2) * 2.0 ** -23 * (size @ W.double().abs()), "dX")


def test_the_largest_vocabulary_in_pieces_of_few_rows():
    check(300, 32, 1 << 20, "bf16", seed=3)
    check(3, 32, (1 << 20) - 1, "f32", seed=4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_matrix_of_more_elements_than_a_kernel_counts(dtype):
    """2^30 and more: the product of more than a few rows is cut along the vocabulary."""
    check(70, 16384, 65537 + 300, dtype, seed=5, sigma=2.0)
    check(5, 16384, 65537 + 300, dtype, seed=6, sigma=2.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [20, 200])
def test_rows_that_are_all_but_sure(dtype, T):
    """Whole logits, the target's 14 above the others, which are equal: 1 - p is (V - 1) e^-14 / Z, 2.5e-4, and right to the roundings of a
    sum near 1 and of p: 2^-21 of the weight, a thousandth of it.  Large logits beside it: log Z alone is rounded to 2^-18."""
    d, V = 64, 300
    x = torch.zeros((T, d), dtype=TYPE[dtype], device="cuda")
    W = torch.zeros((V, d), dtype=TYPE[dtype], device="cuda")
    targets = (torch.arange(T, device="cuda") * 7 % 16).int()
    x[torch.arange(T, device="cuda"), targets.long()] = 1.0      # column k tells target k
    x[:, 40] = 1.0
    W[torch.arange(16, device="cuda"), torch.arange(16, device="cuda")] = 14.0
    W[:, 40] = -112.0                                            # of all logits
    w = torch.linspace(0.5, 2.0, T, device="cuda")
    logp, log_z, G, _, _, _ = reference(x, W, targets, w, exact=True)
    lp, dX, dW = backward(x, W, targets, w, dtype)
    near(lp, logp, 2.0 ** -21, "logp")
    # dX's column of the target: 14 G_target and nothing else; dW's: the sum of its rows' G_target
    rows = torch.arange(T, device="cuda")
    got, want = dX[rows, targets.long()].double() / 14, G[rows, targets.long()]
    near(got, want, (2.0 ** -21 * w.double()) + (HALF[dtype] + 2.0 ** -16) * want.abs(), "G at the target, by dX")
    sums = torch.zeros(16, dtype=torch.float64, device="cuda").index_add_(0, targets.long(), want)
    sizes = torch.zeros(16, dtype=torch.float64, device="cuda").index_add_(0, targets.long(), w.double())
    at = torch.arange(16, device="cuda")
    near(dW[at, at], sums, 2.0 ** -20 * sizes, "G at the target, by dW")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_small_calls_are_the_numpy_oracles(dtype):
    x, W, targets, w = inputs(9, 32, 21, dtype, 2, whole=True)
    host = lambda t: t.double().cpu().numpy()  # noqa: E731
    logp, log_z, dX, dW, _ = orc.head(host(x), host(W), targets.cpu().numpy(), host(w))
    got = forward(x, W, targets, dtype) + backward(x, W, targets, w, dtype)[1:]
    for g, want in zip(got, (logp, log_z, dX, dW)):
        # 2^-14 of the sums of exponentials, and a rounding of each value of G to the type
        assert np.abs(host(g) - want).max() <= (2.0 ** -13 + 2 * (HALF[dtype] if g is got[2] else 2.0 ** -17)) * max(1.0, 9 * 2 * np.abs(host(w)).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_apart_and_equal_logits(dtype):
    T, d, V = 50, 64, 777
    x, W, targets, w = inputs(T, d, V, dtype, 11)
    W = (W.float() * 400).to(W.dtype)                # logits of a thousand: all but one probability are 0
    logp, log_z, G, tol, tol_z, tol_G = reference(x, W, targets, w)
    a, b = forward(x, W, targets, dtype)
    near(a, logp, tol, "logp")
    near(b, log_z, tol_z, "log_z")
    lp, dX, dW = backward(x, W, targets, w, dtype)
    near(lp, logp, tol, "logp of the gradient's call")
    assert dX.isfinite().all() and dW.isfinite().all()
    zero = torch.zeros_like(x)
    a, b = forward(zero, W, targets, dtype)
    none = targets < 0
    assert (a[none] == 0).all() and ((a[~none] + np.log(V)).abs() <= 2.0 ** -14).all() and ((b - np.log(V)).abs() <= 2.0 ** -14).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,V", [(40, 64, 300), (300, 64, 9001), (5000, 64, 4097)])
def test_targets_that_are_none_and_targets_beyond(dtype, T, d, V):
    x, W, targets, w = inputs(T, d, V, dtype, 12)
    w[3] = NAN                                        # of a row without a target: not used
    targets[3] = np.iinfo(np.int32).min
    lp, dX, dW = backward(x, W, targets, w, dtype)
    assert lp[3] == 0 and (dX[3] == 0).all() and dW.isfinite().all() and dX.isfinite().all()
    lp, dX, dW = backward(x, W, torch.full_like(targets, -5), w, dtype)
    assert (lp == 0).all() and (dX == 0).all() and (dW == 0).all()
    targets[7] = V
    a, b = forward(x, W, targets, dtype)
    assert a[7].isnan() and b.isfinite().all() and a[torch.arange(T, device="cuda") != 7].isfinite().all()
    w[3] = 1.0
    lp, dX, dW = backward(x, W, targets, w, dtype)
    others = torch.arange(T, device="cuda") != 7
    assert lp[7].isnan() and dX[7].isnan().all() and dX[others].isfinite().all() and dW.isnan().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,V", [(40, 64, 300), (200, 64, 12345), (700, 96, 5003), (5000, 64, 4097)])
def test_what_stands_in_one_row_touches_no_other(T, d, V, dtype):
    """Rows without a target may hold anything; infinities and NaN in a row with one are that row's, and dW's.  The same bits elsewhere."""
    x, W, targets, w = inputs(T, d, V, dtype, T + V)
    rows = [1, 5, T // 2, T - 1]
    targets[rows] = torch.tensor([-1, -7, -1, -2], dtype=torch.int32, device="cuda")
    others = torch.ones(T, dtype=torch.bool, device="cuda")
    others[rows] = False
    for no_target in (True, False):
        x[rows] = 0.0
        filled = x.clone()
        for row, value in zip(rows, (NAN, float("inf"), 1e30, -float("inf"))):
            filled[row] = value
        if not no_target:
            targets[rows] = 3
            x[rows[2]] = filled[rows[2]] = 1.0      # (a large number is one like others)
        (a, b), (c, e) = forward(x, W, targets, dtype), forward(filled, W, targets, dtype)
        assert torch.equal(a[others], c[others]) and torch.equal(b[others], e[others]) and a.isfinite().all()
        was, now = backward(x, W, targets, w, dtype), backward(filled, W, targets, w, dtype)
        assert torch.equal(was[0][others], now[0][others]) and torch.equal(was[1][others], now[1][others])
        if no_target:
            assert (c[rows] == 0).all() and torch.equal(was[0], now[0]) and torch.equal(was[1], now[1]) and torch.equal(was[2], now[2])
        else:
            wrong = [rows[0], rows[1], rows[3]]
            assert c[wrong].isnan().all() and now[0][wrong].isnan().all() and now[1][wrong].isnan().all() and now[2].isnan().all()


@pytest.mark.parametrize("dtype,T,d,V", [("bf16", 100, 128, 1000), ("f32", 33, 64, 500), ("bf16", 5, 256, 3000), ("bf16", 1, 64, 2000), ("bf16", 300, 64, 7001), ("f32", 300, 64, 7001),
                                          ("f32", 4800, 96, 2900)])
def test_capture_replay_and_another_stream(dtype, T, d, V):
    x, W, targets, w = inputs(T, d, V, dtype, 1)
    ws = workspace(T, d, V, dtype, m.WS_BWD)[0]
    logp, log_z, lp, dX, dW = (torch.zeros(s, dtype=t, device="cuda") for s, t in (
        ((T,), torch.float32), ((T,), torch.float32), ((T,), torch.float32), ((T, d), TYPE[dtype]), ((V, d), torch.float32)))

    def both(stream=None):
        m.modse_head_fwd(T, d, V, dtype, x, W, targets, logp, log_z, ws, stream=stream)
        m.modse_head_bwd(T, d, V, dtype, x, W, targets, w, lp, dX, dW, False, ws, stream=stream)
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in range(4):
        for dst, src in zip((x, W, targets, w), inputs(T, d, V, dtype, seed + 20)):
            dst.copy_(src)
        ws.fill_(seed * 85)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (logp, log_z, lp, dX, dW)]
        for t in (logp, log_z, lp, dX, dW):
            t.fill_(NAN)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        both(s)
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (logp, log_z, lp, dX, dW)))
        want = reference(x, W, targets, w)
        near(logp, want[0], want[3], "logp")


def test_gradients_against_differences():
    """float32, along each gradient: the loss's slope from values on both sides, each right to 2^-14 + e of a log probability, over 2
    steps of h, and the third derivative, whose size is that of x W cubed."""
    T, d, V = 24, 64, 200
    x, W, targets, w = inputs(T, d, V, "f32", 31)
    _, dX, dW = backward(x, W, targets, w, "f32")

    def loss(a, b):
        return float((forward(a, b, targets, "f32")[0].double() * w.double()).sum())
    noise = float(w.abs().sum()) * (2.0 ** -14)
    for a, g, other in ((x, dX, False), (W, dW, True)):
        way = g / g.norm()
        h = 2.0 ** -2 if other else 2.0 ** -1
        sides = [loss(x, W + s * h * way) if other else loss(x + s * h * way, W) for s in (1, -1)]
        slope, along = (sides[0] - sides[1]) / (2 * h), float((g.double() * way.double()).sum())
        # (the step moves a logit by at most r: its third differences by r^3 of the weights)
        r = float(((x @ way.t()) if other else (way @ W.t())).abs().max())
        curve = float(w.abs().sum()) * (2 * r) ** 3 * h ** 2 / 6
        assert abs(slope - along) <= noise / h + min(curve, 0.1 * along), (slope, along, noise / h, curve)
        assert along > 4 * noise / h       # there is a slope to see
