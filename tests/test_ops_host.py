"""What the entry points of the operators around the layer refuse, before they touch a device, and their workspace sizes."""
import pytest
import torch

import paper_2409_12210_amd as m

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
P = 0x10000      # stands for a device pointer; every call below returns before anything is launched
NO = dict(stream=0, raise_on_error=False)


def norm_fwd(T=4, d=64, dtype="bf16", x=P, residual=P, gamma=P, eps=1e-6, y=P, h=P, rstd=P, q=None, scale=None, group=0):
    return m.modse_norm_fwd(T, d, dtype, x, residual, gamma, eps, y, h, rstd, q, scale, group, **NO)


@pytest.mark.parametrize("over,code", [
    (dict(T=-1), INVALID), (dict(d=0), INVALID), (dict(d=-5), INVALID), (dict(d=16385), UNSUPPORTED),
    (dict(T=1 << 31), UNSUPPORTED), (dict(dtype="fp8"), UNSUPPORTED), (dict(x=None), INVALID), (dict(gamma=None), INVALID),
    (dict(eps=-1e-6), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(q=P), INVALID), (dict(scale=P), INVALID), (dict(group=128), INVALID), (dict(q=P, scale=P, group=48), UNSUPPORTED),
    (dict(q=P, scale=P, group=256), UNSUPPORTED), (dict(y=None, h=None, rstd=None), INVALID), (dict(T=0, x=None, gamma=None), OK),
])
def test_norm_fwd_refuses(over, code):
    assert norm_fwd(**over) == code


def norm_bwd(T=4, d=64, dtype="bf16", h=P, gamma=P, rstd=P, dY=P, dH=P, dX=P, dgamma=P, ws=P, ws_bytes=1 << 30):
    return m.modse_norm_bwd(T, d, dtype, h, gamma, rstd, dY, dH, dX, dgamma, False, ws, ws_bytes, **NO)


@pytest.mark.parametrize("over,code", [
    (dict(T=-1), INVALID), (dict(d=0), INVALID), (dict(d=1 << 20), UNSUPPORTED), (dict(dtype=7), UNSUPPORTED),
    (dict(h=None), INVALID), (dict(gamma=None), INVALID), (dict(rstd=None), INVALID), (dict(dY=None), INVALID),
    (dict(dX=None), INVALID), (dict(dgamma=None), INVALID), (dict(ws=None), INVALID), (dict(ws=P + 4), INVALID),
    (dict(ws_bytes=63 * 4), WORKSPACE), (dict(T=0, h=None, ws=None, ws_bytes=0), OK),
])
def test_norm_bwd_refuses(over, code):
    assert norm_bwd(**over) == code


def logprobs_fwd(T=4, V=50000, dtype="f32", logits=P, ld=None, targets=P, logp=P, stats=P, entropy=P, top=3, top_idx=P,
                 top_logp=P, ws=P, ws_bytes=1 << 30):
    return m.modse_logprobs_fwd(T, V, dtype, logits, targets, logp, stats, entropy, top, top_idx, top_logp, ws, ws_bytes,
                                ld_logits=ld, **NO)


@pytest.mark.parametrize("over,code", [
    (dict(T=-1), INVALID), (dict(V=0), INVALID), (dict(top=-1), INVALID), (dict(top=65), UNSUPPORTED),
    (dict(V=(1 << 30) + 1), UNSUPPORTED), (dict(T=1 << 31), UNSUPPORTED), (dict(T=1 << 24, V=9), UNSUPPORTED), (dict(T=1 << 22, V=32000), UNSUPPORTED),
    (dict(dtype="fp16"), UNSUPPORTED), (dict(logits=None), INVALID), (dict(ld=49999), INVALID), (dict(targets=None), INVALID),
    (dict(logp=None), INVALID), (dict(top_idx=None), INVALID), (dict(top_logp=None), INVALID),
    (dict(targets=None, logp=None, stats=None, entropy=None, top=0), INVALID), (dict(ws=None), INVALID),
    (dict(ws=P + 8), INVALID), (dict(ws_bytes=64), WORKSPACE), (dict(T=0, logits=None, ws=None), OK),
])
def test_logprobs_fwd_refuses(over, code):
    assert logprobs_fwd(**over) == code


def logprobs_bwd(T=4, V=5000, dtype="bf16", logits=P, ld=None, targets=P, stats=P, entropy=P, d_logp=P, d_entropy=P,
                 d_logits=2 * P, ldd=None):
    return m.modse_logprobs_bwd(T, V, dtype, logits, targets, stats, entropy, d_logp, d_entropy, d_logits, ld, ldd, **NO)


@pytest.mark.parametrize("over,code", [
    (dict(T=-1), INVALID), (dict(V=0), INVALID), (dict(dtype=3), UNSUPPORTED), (dict(logits=None), INVALID),
    (dict(stats=None), INVALID), (dict(d_logits=None), INVALID), (dict(targets=None), INVALID), (dict(d_logp=None), INVALID),
    (dict(entropy=None), INVALID), (dict(ld=100), INVALID), (dict(ldd=100), INVALID),
    (dict(d_logits=P, ldd=5008), INVALID), (dict(T=0, logits=None), OK),
])
def test_logprobs_bwd_refuses(over, code):
    assert logprobs_bwd(**over) == code


def test_row_distance_comes_from_the_tensor_and_odd_strides_are_refused():
    from paper_2409_12210_amd.binding import _row_distance
    full = torch.zeros((6, 40))
    assert _row_distance(full[:, :33], None, 33) == 40
    assert _row_distance(full[:1, :33], None, 33) == 40
    assert _row_distance(full[::2], None, 40) == 80
    assert _row_distance(full[0], None, 40) == 40 and _row_distance(full[0].expand(1, 40), None, 40) == 40
    assert _row_distance(full.t(), None, 6) == -1 and _row_distance(full[:, ::2], None, 20) == -1
    assert _row_distance(P, None, 7) == 7 and _row_distance(P, 9, 7) == 9
    # the rows of an expanded tensor lie on each other
    assert logprobs_fwd(T=4, V=40, ld=_row_distance(full[0].expand(4, 40), None, 40)) == INVALID


def test_workspaces_serve_fewer_rows_and_refuse_what_the_call_refuses():
    size = lambda T, V=131072, top=20: m.modse_logprobs_workspace_size(T, V, "bf16", top)  # noqa: E731
    last = 0
    for T in (0, 1, 2, 3, 7, 64, 100, 341, 342, 512, 513, 5000):
        now = size(T)
        assert now >= last
        last = now
        for t in (1, T // 2, T):
            if t:
                assert logprobs_fwd(T=t, V=131072, dtype="bf16", top=20, ws_bytes=max(now, 1) - 1, logits=None) == INVALID
    assert size(5000) == size(512) and size(5000) < 2 << 20 and m.modse_logprobs_workspace_size(0, 100, "f32") == 0
    assert m.modse_logprobs_workspace_size(4, 0, "f32", raise_on_error=False) == INVALID
    norm = [m.modse_norm_bwd_workspace_size(T, 2048, "bf16") for T in (0, 1, 5, 1000, 1 << 20)]
    assert norm == sorted(norm) and norm[0] == 0 and norm[-1] < 16 << 20
    assert m.modse_norm_bwd_workspace_size(1, 0, "bf16", raise_on_error=False) == INVALID
    with pytest.raises(m.ModseError):
        m.modse_norm_bwd_workspace_size(-1, 64, "bf16")


# ---------------------------------------------------------------- orthogonalised update
COEFFS = [(3.4445, -4.7750, 2.0315)] * 5


def matrix_set(shapes=((4, 6), (200, 64)), dtype="f32", n=None, G=None):
    """A set of invented device pointers: what the library gets to see of tensors."""
    import ctypes as C

    from paper_2409_12210_amd.binding import _MatrixSet, _dtype_code
    s = object.__new__(m.MatrixSet)
    k = len(shapes)
    s._arrays = ((C.c_int32 * k)(*[r for r, _ in shapes]), (C.c_int32 * k)(*[c for _, c in shapes]),
                 (C.c_void_p * k)(*([P] * k if G is None else G)), (C.c_void_p * k)(*[P] * k))
    s._struct = _MatrixSet(k if n is None else n, *s._arrays, _dtype_code(dtype))
    return s


def ortho(s=None, coeffs=COEFFS, eps=1e-7, ws=P, ws_bytes=1 << 40):
    return m.modse_orthogonalize(s if s is not None else matrix_set(), coeffs, eps, ws, ws_bytes, **NO)


@pytest.mark.parametrize("over,code", [
    (dict(shapes=((0, 4),)), INVALID), (dict(shapes=((4, -1),)), INVALID), (dict(shapes=((65537, 2),)), UNSUPPORTED),
    (dict(dtype="fp8"), UNSUPPORTED), (dict(n=-1), INVALID), (dict(n=4097), UNSUPPORTED), (dict(shapes=()), OK),
    (dict(shapes=((65536, 65536),) * 64), UNSUPPORTED),
])
def test_orthogonalize_refuses_sets(over, code):
    s = matrix_set(**over)
    got = m.modse_orthogonalize_workspace_size(s, raise_on_error=False)
    assert got == (0 if code == OK else code)
    assert ortho(s) == code


@pytest.mark.parametrize("over,code", [
    (dict(coeffs=[]), INVALID), (dict(coeffs=COEFFS * 7), UNSUPPORTED), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(coeffs=[(float("inf"), 0, 0)]), UNSUPPORTED), (dict(coeffs=[(float("nan"), 0, 0)]), UNSUPPORTED),
    (dict(coeffs=[(1e9, 0.0, 0.0)] * 5), UNSUPPORTED), (dict(ws=None), INVALID), (dict(ws=P + 16), INVALID),
    (dict(ws_bytes=1000), WORKSPACE), (dict(s=matrix_set(G=[P, None])), INVALID),
])
def test_orthogonalize_refuses_arguments(over, code):
    assert ortho(**over) == code


def test_matrix_sets_refuse_what_the_library_could_not_see():
    g, u = torch.zeros((4, 6)), torch.zeros((4, 6))
    for G, U in (([g], []), ([g], [u.t()]), ([g[0]], [u[0]]), ([g[:, ::2]], [u[:, ::2]]), ([g.bfloat16()], [u]),
                 ([g, g], [u, u.bfloat16()])):
        with pytest.raises(ValueError):
            m.MatrixSet(G, U)
    with pytest.raises(ValueError):
        m.modse_orthogonalize(matrix_set(), [(1.0, 2.0)], 1e-7, P, 1 << 30, stream=0)
    assert m.MatrixSet([g], [u.bfloat16()])._struct.dtype == 1 and m.MatrixSet([], [])._struct.n_matrices == 0
    a, b = (m.modse_orthogonalize_workspace_size(matrix_set(((2048, k),))) for k in (512, 1024))
    assert 0 < a < b
