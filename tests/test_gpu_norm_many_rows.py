"""The forward pass around and beyond 2048 rows, where rows of 1025 to 2048 values go from four waves to one, and beyond 65536 blocks,
where a block takes several rows.  Tolerances as in test_gpu_norm.py."""
import numpy as np
import pytest
import torch

import paper_2409_12210_amd as m
from oracle import ops_oracle as orc
from test_gpu_norm import EPS, HALF, TYPE, assert_within, blank, host, made

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [1024, 1025, 1535, 2047, 2048, 2049])
def test_rows_of_one_wave_and_of_four(d, dtype):
    for T in (2047, 2048, 2101):
        x, res, gamma = made((T, d), dtype, d), made((T, d), dtype, d + 2), made((d,), dtype, d + 1, 1.0, 0.1)
        y, h, rstd = blank((T, d), TYPE[dtype]), blank((T, d), TYPE[dtype]), blank((T,))
        q, scale = blank((T, d), torch.float8_e4m3fn), blank((T, 1))
        m.modse_norm_fwd(T, d, dtype, x, res, gamma, EPS, y, h, rstd, q, scale)
        h64, y64, r64 = orc.norm_fwd(host(x), host(res), host(gamma), EPS)
        tag = (T, d, dtype)
        assert_within(rstd, r64, 2.0 ** -18 * r64, tag + ("rstd",))
        assert_within(y, y64, (HALF[dtype] + 2.0 ** -17) * np.abs(y64), tag + ("y",))
        assert_within(h, h64, (HALF[dtype] + 2.0 ** -23) * np.abs(h64), tag + ("h",))
        s64, wide = orc.scales(y64, 0)
        assert_within(scale, s64, 2.0 ** -17 * s64, tag + ("scale",))
        values = orc.e4m3_values(q.view(torch.uint8).cpu().numpy())
        assert (np.abs(values * wide - y64) <= (2.0 ** -4 + 2.0 ** -15) * np.abs(y64) + 2.0 ** -10 * wide).all(), tag


@pytest.mark.parametrize("T,d", [(4 * 65536 + 9, 24), (65536 + 5, 2056)])
def test_more_rows_than_a_grid_has(T, d):
    x, gamma = made((T, d), "bf16", 1), made((d,), "bf16", 2, 1.0, 0.1)
    y, rstd = blank((T, d), torch.bfloat16), blank((T,))
    m.modse_norm_fwd(T, d, "bf16", x, None, gamma, EPS, y, None, rstd)
    want = 1.0 / (x.double().square().mean(1) + EPS).sqrt()
    assert ((rstd.double() - want).abs() <= 2.0 ** -18 * want).all()
    rows = torch.tensor([0, 1, T // 2, 65535, 65536, T - 6, T - 1], device="cuda")
    y64 = x[rows].double() * want[rows, None] * gamma.double()
    assert ((y[rows].double() - y64).abs() <= (2.0 ** -8 + 2.0 ** -17) * y64.abs()).all() and not y.isnan().any()
