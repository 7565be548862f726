"""A row's log probability, statistics and entropy are the same bits whichever outputs are asked for.

With top entries few rows of 16385 entries and more are shared by several blocks, without them from 32769 on, and both have to add up in
the same order.  The logits are small: many terms count, and log S has bits to differ in.  With more than 8 entries rows of more
than 512 / top groups of 8192 are cut otherwise; log S is right to 2^-14 there as everywhere, see test_gpu_logprobs.py."""
import pytest
import torch

from test_gpu_logprobs import logits_of, run, targets_for

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [16384, 16385, 20011, 24576, 30000, 32768, 32769, 50257])
@pytest.mark.parametrize("T", [1, 37, 256, 257])
def test_sums_do_not_depend_on_the_top_entries(T, V, dtype):
    for seed in range(3):
        x, targets = logits_of(T, V, dtype, 100 * seed + T, sigma=0.2 + seed, masked=0.4 * (seed == 2)), targets_for(T, V, seed)
        a = run(x, dtype, targets, 0)
        bare = run(x, dtype, targets, 0, entropy=False)
        assert torch.equal(a["logp"], bare["logp"]) and torch.equal(a["stats"], bare["stats"])
        for top in (1, 8, 64):
            b = run(x, dtype, targets, top)
            for k in ("logp", "stats", "entropy"):
                assert torch.equal(a[k], b[k]), (k, top, float((a[k] - b[k]).abs().max()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_other_cuts_are_within_rounding(dtype):
    for T, V, top in ((3, 131072, 64), (2, 160001, 40), (256, 80000, 64)):
        x, targets = logits_of(T, V, dtype, V, sigma=0.5), targets_for(T, V, 1)
        a, b = run(x, dtype, targets, 0), run(x, dtype, targets, top)
        for k, size in (("logp", 2.0 ** -13 + 2.0 ** -21 * 20), ("entropy", 2.0 ** -13 * 14)):
            assert ((a[k] - b[k]).abs() <= size).all()


def test_rows_of_nothing_and_of_nan_where_the_sums_are_held_apart():
    T, V, inf = 5, 30000, float("inf")
    x = logits_of(T, V, "f32", 1)
    x[0] = -inf
    x[1, :V - 1] = -inf                          # only the last group has an entry
    x[2, 9000] = float("nan")
    x[3, 8192:16384] = -inf                      # a group of nothing
    x[4, 17] = inf
    targets = torch.tensor([3, V - 1, 5, 8200, 17], dtype=torch.int32, device="cuda")
    a, b = run(x, "f32", targets, 0), run(x, "f32", targets, 5)
    for k in ("logp", "stats", "entropy"):
        same = (a[k] == b[k]) | (a[k].isnan() & b[k].isnan())
        assert same.all(), k
    assert a["logp"][0] == -inf and a["logp"][1] == 0 and a["logp"][2].isnan() and a["logp"][3] == -inf and a["logp"][4].isnan()
