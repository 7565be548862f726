"""Gradients of the model whose ends are the library's, with and without dropout, against differences along each gradient itself, where a gradient that is zero, lacks a
term or a factor of 1 / (1 - p) is off by far more than what is allowed: every slope is ten times its tolerance or more (see test_gpu_gradients_differences.py).

A row's log probability is right to 2^-20 of log V: logits of 64 products, 200 exponentials to 2^-22 each, under sums of one sign, and a logarithm; so is the mean."""
import pytest
from test_gpu_gradients_differences import slope_of_the_model, tiny_lm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("p", [0.0, 0.3])
@pytest.mark.parametrize("name", ["Wout", "W1", "W3", "W2", "gamma2", "E"])
def test_weights_of_a_routed_model(name, p):
    slope_of_the_model(name, tiny_lm.TinyLM(vocab=200, d_model=64, d_ff=(32, 96, 64, 64), dtype="f32", batch=96, ends=True, dropout=p))


@pytest.mark.parametrize("p", [0.0, 0.3])
@pytest.mark.parametrize("name", ["Wout", "W1", "W3", "W2", "gamma2", "gamma1", "E", "W_gate"])
def test_weights_of_a_model_whose_tokens_go_to_all_experts(name, p):
    model = tiny_lm.TinyLM(vocab=200, d_model=64, d_ff=(96, 64), dtype="f32", batch=96, ends=True, dropout=p)
    for w in (model.W1, model.W3, model.W2):
        w *= 4
    slope_of_the_model(name, model)
