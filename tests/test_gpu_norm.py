"""The norm in front of a layer against its float64 oracle, element by element.

Tolerances, in roundings: of float32 arithmetic u = 2^-24 each, of the last step half a step of the output's type.  The sum of
squares adds at most 8 * 4 values in a thread, then over 6 steps of a wave and up to 16 waves: under 64 roundings of terms of
one sign; the root halves that, and six more operations follow: under 2^6 u = 2^-18 relative for y and rstd.  The gradient's
dot product has terms of both signs: its error is under 2^-17 of the sum of their magnitudes."""
import numpy as np
import pytest
import torch

import paper_2409_12210_amd as m
from oracle import ops_oracle as orc

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5
NAN = float("nan")


def host(t):
    return t.detach().double().cpu().numpy()


def made(shape, dtype, seed, mean=0.0, sigma=1.0, pad=0):
    """A tensor that starts `pad` elements behind an aligned address."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = int(np.prod(shape))
    t = torch.empty(n + pad, dtype=TYPE[dtype], device="cuda")[pad:].view(shape)
    return t.normal_(mean, sigma, generator=gen)


def blank(shape, dtype=torch.float32, pad=0):
    t = torch.empty(int(np.prod(shape)) + pad, dtype=dtype, device="cuda")[pad:].view(shape)
    return t.view(torch.uint8).fill_(0x7f).view(dtype).view(shape) if dtype == torch.float8_e4m3fn else t.fill_(NAN)


def assert_within(got, want, tol, what):
    err = np.abs(host(got) - want)
    bad = ~(err <= tol)
    assert not bad.any(), (what, int(bad.sum()), float(np.nanmax(err - tol)), np.argwhere(bad)[:3].tolist())


# widths: one element, less than a chunk, a chunk and one, every choice of waves and chunks per row and both sides of its edges
WIDTHS = (1, 7, 8, 9, 96, 511, 512, 513, 1024, 1025, 1535, 2047, 2048, 2056, 4096, 4104, 5632, 8192, 8200, 16384)
ROWS = (1, 3, 4, 5, 130)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", WIDTHS)
def test_norm_forward_and_backward(d, dtype):
    for T in ROWS + ((1100,) if d <= 2056 else ()):
        for with_residual in (True, False):
            pad = 1 if T % 2 else 0       # rows that start at the alignment of an element
            x, gamma = made((T, d), dtype, d, pad=pad), made((d,), dtype, d + 1, 1.0, 0.1, pad=pad)
            res = made((T, d), dtype, d + 2, pad=pad) if with_residual else None
            y, h = blank((T, d), TYPE[dtype], pad), blank((T, d), TYPE[dtype], pad) if with_residual else None
            rstd = blank((T,))
            m.modse_norm_fwd(T, d, dtype, x, res, gamma, EPS, y, h, rstd)
            h64, y64, r64 = orc.norm_fwd(host(x), None if res is None else host(res), host(gamma), EPS)
            tag = (T, d, dtype, with_residual)
            assert_within(rstd, r64, 2.0 ** -18 * r64, tag + ("rstd",))
            assert_within(y, y64, (HALF[dtype] + 2.0 ** -17) * np.abs(y64), tag + ("y",))
            if with_residual:
                assert_within(h, h64, (HALF[dtype] + 2.0 ** -23) * np.abs(h64), tag + ("h",))
            stored = h if with_residual else x
            dY, dH = made((T, d), dtype, d + 3, pad=pad), made((T, d), dtype, d + 4, pad=pad) if with_residual else None
            dX, dgamma = blank((T, d), TYPE[dtype], pad), blank((d,))
            ws = torch.empty(m.modse_norm_bwd_workspace_size(T, d, dtype), dtype=torch.uint8, device="cuda").fill_(255)
            m.modse_norm_bwd(T, d, dtype, stored, gamma, rstd, dY, dH, dX, dgamma, False, ws)
            check_backward(tag, dtype, stored, gamma, rstd, dY, dH, dX, dgamma, 0.0)
            m.modse_norm_bwd(T, d, dtype, stored, gamma, rstd, dY, dH, dX, dgamma.fill_(2.0), True, ws)
            check_backward(tag, dtype, stored, gamma, rstd, dY, dH, dX, dgamma, 2.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [40, 513, 1535, 2056, 4104, 8200, 16384])
def test_backward_around_512_tokens(d, dtype):
    for T in (257, 511, 512, 513, 1200):
        pad = T % 2
        h, gamma = made((T, d), dtype, d, pad=pad), made((d,), dtype, d + 1, 1.0, 0.1)
        dY, dH, rstd = made((T, d), dtype, d + 2), made((T, d), dtype, d + 3, pad=pad), blank((T,))
        m.modse_norm_fwd(T, d, dtype, h, None, gamma, EPS, blank((T, d), TYPE[dtype]), None, rstd)
        ws = torch.empty(m.modse_norm_bwd_workspace_size(T, d, dtype), dtype=torch.uint8, device="cuda").fill_(255)
        tag = (T, d, dtype)
        dX, dgamma = blank((T, d), TYPE[dtype], pad=pad), blank((d,))
        m.modse_norm_bwd(T, d, dtype, h, gamma, rstd, dY, dH, dX, dgamma, False, ws)
        check_backward(tag, dtype, h, gamma, rstd, dY, dH, dX, dgamma, 0.0)
        # in the buffers of the inputs: the same bits, added to what is there
        for place in range(3):
            a = [h.clone(), dY.clone(), dH.clone()]
            more = torch.full((d,), 2.0, device="cuda")
            m.modse_norm_bwd(T, d, dtype, a[0], gamma, rstd, a[1], a[2], a[place], more, True, ws)
            assert torch.equal(a[place], dX) and torch.equal(more, dgamma + 2.0), tag


def check_backward(tag, dtype, h, gamma, rstd, dY, dH, dX, dgamma, before):
    h64, g64, r64, dy64 = host(h), host(gamma), host(rstd)[:, None], host(dY)
    want, dg = orc.norm_bwd(h64, g64, host(rstd), dy64, None if dH is None else host(dH))
    g, hat = dy64 * g64, h64 * r64
    size = r64 * (np.abs(g) + np.abs(hat) * np.abs(g * hat).mean(1, keepdims=True)) + (0 if dH is None else np.abs(host(dH)))
    assert_within(dX, want, HALF[dtype] * np.abs(want) + 2.0 ** -17 * size, tag + ("dX",))
    # (at most 1100 / 4 rows in a sequence, then 4 waves and 16 + 32 shares: under 2^9 roundings)
    assert_within(dgamma, dg + before, 2.0 ** -15 * (np.abs(dy64 * hat).sum(0) + before), tag + ("dgamma",))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("d", [1, 31, 128, 200, 1535, 2048, 4104, 8200, 16384])
def test_norm_in_8_bits(d, group, dtype):
    for T in (1, 6, 1030 if d <= 2048 else 9):
        x, res, gamma = made((T, d), dtype, 1), made((T, d), dtype, 2, sigma=3.0), made((d,), dtype, 3, 1.0, 0.2)
        if T > 2:
            x[1], res[1] = 0.0, 0.0                      # a row of zeros
            x[2, : d // 2] = 0.0
            res[2, : d // 2] = 0.0                       # whole groups of zeros
        n = -(-d // group) if group else 1
        for keep in (True, False):
            y, h = blank((T, d), TYPE[dtype]) if keep else None, blank((T, d), TYPE[dtype])
            q, scale = blank((T, d), torch.float8_e4m3fn), blank((T, n))
            m.modse_norm_fwd(T, d, dtype, x, res, gamma, EPS, y, h, None, q, scale, group)
            _, y64, _ = orc.norm_fwd(host(x), host(res), host(gamma), EPS)
            s64, wide = orc.scales(y64, group)
            assert_within(scale, s64, 2.0 ** -17 * s64, (T, d, group, "scale"))
            values = orc.e4m3_values(q.view(torch.uint8).cpu().numpy())
            assert np.isfinite(values).all()
            # half a step: 2^-4 of a normal value, 2^-10 below 2^-6; float32 in front of it moves the scaled value by 2^-16
            tol = (2.0 ** -4 + 2.0 ** -15) * np.abs(y64) + 2.0 ** -10 * wide
            assert (np.abs(values * wide - y64) <= tol).all(), (T, d, group)
            if keep:
                assert_within(y, y64, (HALF[dtype] + 2.0 ** -17) * np.abs(y64), (T, d, group, "y"))


def test_e4m3_roundings_are_to_nearest_even():
    # rows whose largest value is 448 times a power of two: the scale is exact, and every quotient a given number
    grid = orc.e4m3_values(np.arange(0, 127, dtype=np.uint8))
    ties = (grid[:-1] + grid[1:]) / 2
    vals = np.concatenate([grid, ties, -ties, ties * (1 + 2.0 ** -12), ties * (1 - 2.0 ** -12)])
    vals = vals[np.abs(vals) <= 448]
    d = 1024
    row = np.zeros(d)
    row[: len(vals)] = vals
    row[-1] = 448.0
    # y = gamma h rstd with h = 1, eps = 0: y = gamma exactly
    x, gamma = torch.ones((1, d), device="cuda"), torch.tensor(row, dtype=torch.float32, device="cuda")
    q, scale = blank((1, d), torch.float8_e4m3fn), blank((1, 1))
    m.modse_norm_fwd(1, d, "f32", x, None, gamma, 0.0, None, None, None, q, scale)
    assert float(scale) == 1.0
    want = gamma.to(torch.float8_e4m3fn)
    assert torch.equal(q[0].view(torch.uint8), want.view(torch.uint8))


@pytest.mark.parametrize("group", [0, 64])
@pytest.mark.parametrize("d", [200, 2048, 4096])
def test_every_8_bit_value_is_the_nearest_to_the_exact_quotient(d, group):
    # y / scale = 448 h gamma / max|h gamma|.  h = i / 32 with |i| <= 254 and gamma = j / 128 with j <= 255: h gamma and 448 h gamma
    # are exact in float32, the quotient is rounded to float32 once, and float64 in between moves no tie of e4m3
    T = 97
    gen = torch.Generator(device="cuda").manual_seed(d + group)
    x, res = (torch.randint(-127, 128, (T, d), generator=gen, device="cuda").div(32).bfloat16() for _ in range(2))
    gamma = torch.randint(64, 256, (d,), generator=gen, device="cuda").div(128).bfloat16()
    q, scale = blank((T, d), torch.float8_e4m3fn), blank((T, -(-d // group) if group else 1))
    m.modse_norm_fwd(T, d, "bf16", x, res, gamma, EPS, None, blank((T, d), torch.bfloat16), None, q, scale, group)
    v = (x.double() + res.double()) * gamma.double()
    amax = torch.cat([p.abs().amax(1, keepdim=True).expand_as(p) for p in v.split(group or d, 1)], 1)
    want = (448.0 * v / amax).float().to(torch.float8_e4m3fn)
    assert torch.equal(q.view(torch.uint8), want.view(torch.uint8))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [200, 2048, 5000])
def test_outputs_in_the_buffers_of_inputs(d, dtype):
    T = 70
    x, res, gamma = made((T, d), dtype, 1), made((T, d), dtype, 2), made((d,), dtype, 3, 1.0, 0.1)
    y, h, rstd = blank((T, d), TYPE[dtype]), blank((T, d), TYPE[dtype]), blank((T,))
    m.modse_norm_fwd(T, d, dtype, x, res, gamma, EPS, y, h, rstd)
    x2, res2 = x.clone(), res.clone()
    m.modse_norm_fwd(T, d, dtype, x2, res2, gamma, EPS, x2, res2, None)
    assert torch.equal(x2, y) and torch.equal(res2, h)
    dY, dH = made((T, d), dtype, 4), made((T, d), dtype, 5)
    ws = torch.empty(m.modse_norm_bwd_workspace_size(T, d, dtype), dtype=torch.uint8, device="cuda")
    outs = []
    for place in (None, "dY", "dH", "h"):
        a = {"dY": dY.clone(), "dH": dH.clone(), "h": h.clone()}
        dX, dgamma = a.get(place, blank((T, d), TYPE[dtype])), blank((d,))
        m.modse_norm_bwd(T, d, dtype, a["h"], gamma, rstd, a["dY"], a["dH"], dX, dgamma, False, ws)
        outs.append((dX, dgamma))
    for dX, dgamma in outs[1:]:
        assert torch.equal(dX, outs[0][0]) and torch.equal(dgamma, outs[0][1])


def test_a_row_with_nan_or_infinity_leaves_the_others_alone():
    T, d = 9, 1000
    x, gamma = made((T, d), "f32", 1), made((d,), "f32", 2, 1.0, 0.1)
    clean = blank((T, d))
    m.modse_norm_fwd(T, d, "f32", x, None, gamma, EPS, clean, None, None)
    x[4, 17], x[6, 3] = NAN, float("inf")
    y = blank((T, d)).fill_(0.0)
    m.modse_norm_fwd(T, d, "f32", x, None, gamma, EPS, y, None, None)
    keep = [0, 1, 2, 3, 5, 7, 8]
    assert torch.equal(y[keep], clean[keep]) and y[4].isnan().all() and y[6, 3].isnan()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_gradient_is_that_of_differences(dtype):
    """The loss's change along a direction against <gradient, direction>, both from the kernels, float32 outputs of
    float32 inputs: the quotient's error is half a step's curvature and 2^-17 of the sums that are subtracted."""
    T, d, step = 8, 264, 2.0 ** -6
    x, gamma, dY, way = (made((T, d), "f32", 1), made((d,), "f32", 2, 1.0, 0.1), made((T, d), "f32", 3), made((T, d), "f32", 4))
    if dtype == "bf16":       # values that both types hold; the forward pass is the float32 one
        x, gamma, dY = x.bfloat16().float(), gamma.bfloat16().float(), dY.bfloat16().float()

    def loss(v):
        y = blank((T, d))
        m.modse_norm_fwd(T, d, "f32", v, None, gamma, EPS, y, None, None)
        return float((y.double() * dY.double()).sum())
    rstd, dX, dgamma = blank((T,)), blank((T, d), TYPE[dtype]), blank((d,))
    m.modse_norm_fwd(T, d, "f32", x, None, gamma, EPS, blank((T, d)), None, rstd)
    ws = torch.empty(m.modse_norm_bwd_workspace_size(T, d, dtype), dtype=torch.uint8, device="cuda")
    m.modse_norm_bwd(T, d, dtype, x.to(TYPE[dtype]), gamma.to(TYPE[dtype]), rstd, dY.to(TYPE[dtype]), None, dX, dgamma, False, ws)
    along = float((dX.double() * way.double()).sum())
    quotient = (loss(x + step * way) - loss(x - step * way)) / (2 * step)
    size = float((dX.double() * way.double()).abs().sum())
    # third derivatives of y are of the size of y (rows of unit mean square): step^2 of sum |dY| at most
    tol = HALF[dtype] * size + 2.0 ** -17 * float(dY.abs().sum()) / step + step ** 2 * float(dY.abs().sum())
    assert abs(along - quotient) <= tol


def test_runs_are_the_same_bits_and_other_streams_order_with_events():
    T, d = 3000, 2048
    x, gamma, dY = made((T, d), "bf16", 1), made((d,), "bf16", 2, 1.0, 0.1), made((T, d), "bf16", 3)
    rstd = blank((T,))
    m.modse_norm_fwd(T, d, "bf16", x, None, gamma, EPS, blank((T, d), torch.bfloat16), None, rstd)
    outs = []
    side = torch.cuda.Stream()
    for stream in (None, None, side):
        ws = torch.empty(m.modse_norm_bwd_workspace_size(T, d, "bf16"), dtype=torch.uint8, device="cuda")
        dX, dgamma = blank((T, d), torch.bfloat16), blank((d,))
        torch.cuda.synchronize()
        m.modse_norm_bwd(T, d, "bf16", x, gamma, rstd, dY, None, dX, dgamma, False, ws, stream=stream)
        torch.cuda.synchronize()
        outs.append((dX, dgamma))
    for dX, dgamma in outs[1:]:
        assert torch.equal(dX, outs[0][0]) and torch.equal(dgamma, outs[0][1])


def test_no_tokens_leave_everything_as_it_is():
    dgamma = torch.full((8,), 3.0, device="cuda")
    m.modse_norm_fwd(0, 8, "f32", None, None, None, EPS, None, None, None)
    m.modse_norm_bwd(0, 8, "f32", None, None, None, None, None, None, dgamma, False, None)
    torch.cuda.synchronize()
    assert (dgamma == 3.0).all()


def test_a_captured_step_replays():
    T, d = 65, 1000
    x, gamma, dY = made((T, d), "f32", 1), made((d,), "f32", 2, 1.0, 0.1), made((T, d), "f32", 3)
    y, rstd, dX, dgamma = blank((T, d)), blank((T,)), blank((T, d)), blank((d,))
    ws = torch.empty(m.modse_norm_bwd_workspace_size(T, d, "f32"), dtype=torch.uint8, device="cuda")

    def step():
        m.modse_norm_fwd(T, d, "f32", x, None, gamma, EPS, y, None, rstd)
        m.modse_norm_bwd(T, d, "f32", x, gamma, rstd, dY, None, dX, dgamma, False, ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (10, 11, 12, 13):
        x.copy_(made((T, d), "f32", seed))
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (y, rstd, dX, dgamma)]
        for t in (y, rstd, dX, dgamma):
            t.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (y, rstd, dX, dgamma)))
