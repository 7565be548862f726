"""The workspace of log probabilities from hidden rows stops growing with the batch."""
import pytest

import paper_2409_12210_amd as m


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,V", [(32, 1), (64, 100), (2048, 32000), (256, 50257), (4096, 131072), (32, 1 << 20), (16384, 1 << 20)])
def test_it_has_a_bound(d, V, dtype):
    """A piece has 65536 rows at the most, and the tables of sixteen pieces are there at a time: beyond that it is one size, at these shapes less than 4 GiB.
    (The most is 10 GiB, for gradients of rows of 16384 and a vocabulary of 4096.)"""
    for which in (m.WS_FWD, m.WS_BWD):
        sizes = [m.modse_head_workspace_size(T, d, V, dtype, which) for T in (1 << 20, (1 << 20) + 1, 1 << 22, 1 << 24)]
        assert len(set(sizes)) == 1 and sizes[0] < 4 << 30, sizes
