"""Which tensors of logits are rows of a matrix, and at what distance: seen without a device."""
import pytest
import torch

import paper_2409_12210_amd as m
from paper_2409_12210_amd.binding import _row_distance

INVALID = 1


def test_outer_dimensions_are_rows_only_where_they_could_be_flattened():
    x = torch.zeros((4, 8, 16))
    assert _row_distance(x, None, 16) == 16 and _row_distance(x[:, :, :11], None, 11) == 16
    assert _row_distance(x[:, :-1], None, 16) == -1             # the usual shift for the next token's loss
    assert _row_distance(x[:, 1:], None, 16) == -1
    assert _row_distance(x[:, -1:], None, 16) == 128            # the last position of each: 4 rows at that distance
    assert _row_distance(x[:, -1], None, 16) == 128
    assert _row_distance(x[:1, :-1], None, 16) == 16 and _row_distance(x[2:3, 1:], None, 16) == 16
    assert _row_distance(x[:, ::2], None, 16) == 32             # every second: 16 rows at 32
    assert _row_distance(x[::2], None, 16) == -1
    assert _row_distance(x.transpose(0, 1), None, 16) == -1
    assert _row_distance(x[:1, :1], None, 16) >= 16
    y = torch.zeros((2, 3, 4, 10))
    assert _row_distance(y, None, 10) == 10 and _row_distance(y[:, :, :1], None, 10) == 40
    assert _row_distance(y[:, :2], None, 10) == -1 and _row_distance(y[:, :2, :1], None, 10) == -1
    assert _row_distance(y[:1, :2], None, 10) == 10
    assert _row_distance(y[:1].expand(2, 3, 4, 10), None, 10) == -1


def test_entries_that_do_not_lie_side_by_side_are_refused():
    assert _row_distance(torch.zeros(32)[::2], None, 16) == -1 and _row_distance(torch.zeros(32), None, 16) == 16
    assert _row_distance(torch.zeros((4, 32))[:, ::2], None, 16) == -1
    assert _row_distance(torch.zeros(()), None, 16) == -1
    assert _row_distance(torch.zeros((4, 1, 2))[:, :, 1:], None, 1) == 2    # a vocabulary of one


def test_the_distance_that_a_matrix_has_is_that_of_flattening_it():
    """Every slice of three dimensions: where the result is a distance, the rows at it are those of reshape."""
    x = torch.arange(3 * 4 * 6.0).view(3, 4, 6)
    seen = 0
    for a in (slice(None), slice(1, None), slice(None, None, 2), slice(0, 1)):
        for b in (slice(None), slice(None, -1), slice(1, 3), slice(None, None, 2), slice(2, 3)):
            for c in (slice(None), slice(1, 5)):
                t = x[a, b, c]
                V, d = t.shape[2], _row_distance(t, None, t.shape[2])
                if d < 0:
                    assert t.flatten(0, 1).data_ptr() != t.data_ptr()     # torch has to copy it, too
                    continue
                T = t.shape[0] * t.shape[1]
                assert torch.equal(t.as_strided((T, V), (d, 1)), t.reshape(T, V))
                seen += 1
    assert seen > 20


@pytest.mark.parametrize("make", [lambda x: x[:, :-1], lambda x: x.transpose(0, 1)])
def test_the_calls_refuse_such_logits(make):
    P = 0x10000
    x, no = make(torch.zeros((4, 8, 16))), dict(stream=0, raise_on_error=False)
    assert m.modse_logprobs_fwd(28, 16, "f32", x, None, None, P, None, 0, None, None, None, 0, **no) == INVALID
    assert m.modse_logprobs_bwd(28, 16, "f32", P, None, P, P, None, P, x, **no) == INVALID
