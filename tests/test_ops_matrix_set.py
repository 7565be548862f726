"""What a set of matrices and the coefficients of its steps have to agree on, seen without a device."""
import pytest
import torch

import paper_2409_12210_amd as m


def test_the_type_of_the_results_is_that_of_the_tensors():
    """Told float32, the kernels would write twice as many bytes as a bfloat16 tensor has."""
    g, u = [torch.zeros((4, 6))], [torch.zeros((4, 6), dtype=torch.bfloat16)]
    for told in ("f32", torch.float32, 0):
        with pytest.raises(ValueError):
            m.MatrixSet(g, u, told)
    with pytest.raises(ValueError):
        m.MatrixSet(g, g, "bf16")
    assert m.MatrixSet(g, u, "bf16")._struct.dtype == 1 and m.MatrixSet(g, g, torch.float32)._struct.dtype == 0
    assert m.MatrixSet([], [], "bf16")._struct.dtype == 1


def test_every_step_has_three_coefficients():
    """Five of one step and one of the next make six in all."""
    P, s = 0x10000, m.MatrixSet([torch.zeros((4, 6))], [torch.zeros((4, 6))])
    for coeffs in ([(1.0, 2.0), (1.0, 2.0, 3.0, 4.0)], [(1.0, 0.0, 0.0, 0.0, 0.0), (1.0,)], [()]):
        with pytest.raises(ValueError):
            m.modse_orthogonalize(s, coeffs, 1e-7, P, 0, stream=0)
