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


def test_the_workspace_holds_two_squares_a_matrix_where_steps_go_alone():
    """8 (m n + m m) bytes and lists; sets whose steps go together have six squares, 8 (m n + 3 m m)."""
    def size(shapes):
        s = [torch.empty(r, c, device="meta") for r, c in shapes]
        return m.modse_orthogonalize_workspace_size(m.MatrixSet(s, s))
    lists = 1 << 20
    for shapes, squares in (([(256, 256)] * 3, 2), ([(2048, 2048)] * 3, 2), ([(384, 128)] * 24, 2), ([(1024, 4224)] * 12, 6)):
        n = sum(r * c * 8 + min(r, c) ** 2 * 4 * squares for r, c in shapes)
        assert n <= size(shapes) <= n + n // 50 + lists, (shapes, squares)
