"""The example's own checks, seen without a device: its buffers are a batch long, and the kernels write as many rows as they are told."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import tiny_lm  # noqa: E402


def model(batch):
    m = object.__new__(tiny_lm.TinyLM)
    m.T, m.V, m.d, m.dtype = batch, 50, 8, "f32"
    m.E = None           # nothing is looked up before the check
    return m


def test_more_tokens_than_the_buffers_hold_are_refused():
    with pytest.raises(ValueError):
        model(4).forward(torch.arange(5))
    with pytest.raises(ValueError):
        model(4).alternatives(torch.arange(5), 3)


def test_a_training_step_takes_a_whole_batch():
    m = model(4)
    for tokens, targets in ((3, 3), (5, 5), (5, 4), (3, 4), (4, 3), (4, 5)):
        with pytest.raises(ValueError):
            m.loss_and_gradients(torch.arange(tokens), torch.zeros(targets, dtype=torch.int32))
