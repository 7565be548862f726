"""Lookup and dropout of more work than a launch has blocks for (2^20 at the most), so that blocks take more than one share of it."""
import numpy as np
import pytest
import torch

import paper_2409_12210_amd as m
from oracle import ends_oracle as orc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_lookup_of_more_than_four_million_rows(dtype):
    """A wave takes a row, four of them are a block: 2^22 rows are a launch.  Times 2: exact."""
    T, d, V = (1 << 23) + 1029, 8, 1000
    print("lookup", T, d, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(1)
    E = torch.randn((V, d), generator=gen, device="cuda").to(dtype)
    tokens = torch.randint(-1, V + 1, (T,), generator=gen, device="cuda", dtype=torch.int32)
    x = torch.full((T + 1, d), 7.0, dtype=dtype, device="cuda")
    m.modse_embed_fwd(T, d, V, "bf16" if dtype == torch.bfloat16 else "f32", tokens, E, 2.0, x[:T])
    want = (2.0 * E)[tokens.clamp(0, V - 1).long()]
    want[tokens < 0] = 0.0
    beyond = tokens == V
    assert torch.equal(x[:T][~beyond], want[~beyond]) and x[:T][beyond].isnan().all() and (x[T] == 7.0).all()


@pytest.mark.parametrize("residual", [False, True])
def test_dropout_of_more_than_two_thousand_million_elements(residual):
    """2048 elements are a block's share; the second one begins at 2^31.  Against the counters of places on both sides of it, and as many kept as there have to be."""
    T, d, p, seed, offset, call = 524288 + 777, 4099, 0.25, 0x123456789ABCDEF, (3 << 32) + 9, 5
    n, limit = T * d, 16384
    assert n > 1 << 31
    print("dropout", T, d, residual, flush=True)
    x = torch.full((T, d), 1.5, dtype=torch.bfloat16, device="cuda")
    res = torch.full((T, d), 0.25, dtype=torch.bfloat16, device="cuda") if residual else None
    y = torch.full((n + 8,), 7.0, dtype=torch.bfloat16, device="cuda")
    rng = torch.tensor([seed, offset], dtype=torch.int64, device="cuda")
    m.modse_dropout_fwd(T, d, "bf16", x, res, p, rng, call, y[:n].view(T, d))
    kept, dropped = 2.0 + (0.25 if residual else 0.0), 0.25 if residual else 0.0      # 1.5 / 0.75 is 2
    assert (y[n:] == 7.0).all()
    counts = [0, 0]
    for part in y[:n].split(1 << 28):
        counts[0] += int((part == kept).sum())
        counts[1] += int((part == dropped).sum())
    assert sum(counts) == n and abs(counts[0] - 0.75 * n) <= 6 * (0.75 * 0.25 * n) ** 0.5       # six standard deviations
    second = (1 << 31) // 8
    for first in (0, second - 40, second, second + 100000, (n - 1) // 8 - 40):
        want = []
        for i in range(first, first + 40):
            words = orc.philox4x32((i, call, offset & 0xFFFFFFFF, offset >> 32), (seed & 0xFFFFFFFF, seed >> 32), 7)
            want += [kept if w >> s & 0xFFFF >= limit else dropped for w in words for s in (0, 16)]
        assert np.array_equal(y[first * 8:first * 8 + 320].float().cpu().numpy(), np.array(want, np.float32)), first
    if not residual:
        dX = torch.empty_like(y)
        m.modse_dropout_bwd(T, d, "bf16", x, p, rng, call, dX[:n].view(T, d))
        assert torch.equal(dX[:n], y[:n])
