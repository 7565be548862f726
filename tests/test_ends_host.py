"""What the entry points of the operators at both ends of a model refuse, before they touch a device, and their workspace sizes."""
import pytest
import torch

import paper_2409_12210_amd as m

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
P = 0x10000      # stands for a device pointer; every call below returns before anything is launched
NO = dict(stream=0, raise_on_error=False)
NAN, INF = float("nan"), float("inf")


def embed_fwd(T=4, d=64, V=100, dtype="bf16", tokens=P, E=P, scale=1.0, x=P):
    return m.modse_embed_fwd(T, d, V, dtype, tokens, E, scale, x, **NO)


@pytest.mark.parametrize("over,code", [
    (dict(T=-1), INVALID), (dict(d=0), INVALID), (dict(d=16385), UNSUPPORTED), (dict(V=0), INVALID), (dict(V=-3), INVALID),
    (dict(V=(1 << 20) + 1), UNSUPPORTED), (dict(T=1 << 31), UNSUPPORTED), (dict(dtype="fp16"), UNSUPPORTED), (dict(tokens=None), INVALID),
    (dict(E=None), INVALID), (dict(x=None), INVALID), (dict(scale=NAN), INVALID), (dict(scale=INF), INVALID),
    (dict(T=0, tokens=None, E=None, x=None), OK),
])
def test_embed_fwd_refuses(over, code):
    assert embed_fwd(**over) == code


def embed_bwd(T=4, d=64, V=100, dtype="bf16", tokens=P, dX=P, scale=1.0, dE=P, ws=P, ws_bytes=1 << 40):
    return m.modse_embed_bwd(T, d, V, dtype, tokens, dX, scale, dE, False, ws, ws_bytes, **NO)


@pytest.mark.parametrize("over,code", [
    (dict(T=-1), INVALID), (dict(d=-1), INVALID), (dict(d=1 << 20), UNSUPPORTED), (dict(V=0), INVALID), (dict(V=1 << 21), UNSUPPORTED),
    (dict(T=1 << 30, d=16384), UNSUPPORTED), (dict(dtype=9), UNSUPPORTED), (dict(tokens=None), INVALID), (dict(dX=None), INVALID),
    (dict(dE=None), INVALID), (dict(ws=None), INVALID), (dict(ws=P + 8), INVALID), (dict(ws_bytes=100), WORKSPACE),
    (dict(scale=-INF), INVALID), (dict(T=0, tokens=None, ws=None, ws_bytes=0), OK),
])
def test_embed_bwd_refuses(over, code):
    assert embed_bwd(**over) == code


def test_embed_workspaces_serve_fewer_tokens():
    size = lambda T, d=300: m.modse_embed_bwd_workspace_size(T, d, 5000, "bf16")  # noqa: E731
    last = 0
    for T in (0, 1, 7, 8, 9, 1000, 8191, 8192, 8193, 20000, 32768, 32769, 40000, 65536, 65537, 200000):
        now = size(T)
        assert now >= last
        last = now
        for t in {1, T // 3, T - 1, T} - {0, -1}:
            assert embed_bwd(T=t, d=300, V=5000, ws_bytes=now, tokens=None) == INVALID
    # a call's own need is refused when a byte is missing of it, where no smaller batch needs more
    for T in (1, 1000, 8192, 200000):
        assert embed_bwd(T=T, d=300, V=5000, ws_bytes=size(T) - 1) == WORKSPACE
    assert m.modse_embed_bwd_workspace_size(4, 0, 5, "f32", raise_on_error=False) == INVALID
    with pytest.raises(m.ModseError):
        m.modse_embed_bwd_workspace_size(4, 8, 1 << 21, "f32")


def dropout(T=4, d=64, dtype="bf16", x=P, residual=P, p=0.1, rng=P, y=P, back=False):
    if back:
        return m.modse_dropout_bwd(T, d, dtype, x, p, rng, 0, y, **NO)
    return m.modse_dropout_fwd(T, d, dtype, x, residual, p, rng, 0, y, **NO)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("over,code", [
    (dict(T=-1), INVALID), (dict(d=0), INVALID), (dict(d=16385), UNSUPPORTED), (dict(T=1 << 21, d=16384), UNSUPPORTED),
    (dict(dtype="fp8"), UNSUPPORTED), (dict(x=None), INVALID), (dict(rng=None), INVALID), (dict(y=None), INVALID),
    (dict(p=-0.1), INVALID), (dict(p=1.0001), INVALID), (dict(p=NAN), INVALID), (dict(T=0, x=None, rng=None, y=None), OK),
])
def test_dropout_refuses(over, code, back):
    assert dropout(**over, back=back) == code


def test_tensors_that_the_library_could_not_see_are_refused():
    f, b, i = torch.zeros((4, 64)), torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    E = torch.zeros((100, 64), dtype=torch.bfloat16)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    for tokens, table, x in ((i.long(), E, b), (i, E.float(), b), (i, E, f), (i, E[:, ::2], b), (i, E, b.t())):
        assert embed_fwd(tokens=tokens, E=table, x=x) == INVALID
    for tokens, dX, dE in ((i.long(), b, f), (i, f, f), (i, b, b), (i, b[:, :32], f)):
        assert embed_bwd(tokens=tokens, dX=dX, dE=dE, ws=ws, ws_bytes=None) == INVALID
    pair = torch.zeros(2, dtype=torch.int64)
    for x, residual, rng, y in ((f, None, pair, b), (b, f, pair, b), (b, None, pair.int(), b), (b, None, pair[:1], b), (b, None, torch.zeros(4, dtype=torch.int64)[::2], b)):
        assert dropout(x=x, residual=residual, rng=rng, y=y) == INVALID
    assert dropout(x=b, rng=pair.float(), y=b, back=True) == INVALID
    assert dropout(x=b, rng=pair, residual=None, y=b) == INVALID      # seed and offset on the host
    with pytest.raises(m.ModseError, match="expected two int64"):
        m.modse_dropout_bwd(4, 64, "bf16", b, 0.1, pair.float(), 0, b, stream=0)


def head_fwd(T=4, d=64, V=100, dtype="bf16", x=P, W=P, targets=P, logp=P, log_z=P, ws=P, ws_bytes=1 << 40):
    return m.modse_head_fwd(T, d, V, dtype, x, W, targets, logp, log_z, ws, ws_bytes, **NO)


def head_bwd(T=4, d=64, V=100, dtype="bf16", x=P, W=P, targets=P, d_logp=P, logp=P, dX=P, dW=P, ws=P, ws_bytes=1 << 40):
    return m.modse_head_bwd(T, d, V, dtype, x, W, targets, d_logp, logp, dX, dW, False, ws, ws_bytes, **NO)


BOTH = [
    (dict(T=-1), INVALID), (dict(d=0), INVALID), (dict(d=48), INVALID), (dict(d=16416), UNSUPPORTED), (dict(V=0), INVALID),
    (dict(V=(1 << 20) + 1), UNSUPPORTED), (dict(T=(1 << 24) + 1), UNSUPPORTED), (dict(dtype="fp16"), UNSUPPORTED), (dict(x=None), INVALID),
    (dict(W=None), INVALID), (dict(targets=None), INVALID), (dict(ws=None), INVALID), (dict(ws=P + 8), INVALID), (dict(x=P + 2), INVALID),
    (dict(W=P + 8), INVALID), (dict(ws_bytes=100), WORKSPACE), (dict(T=0, x=None, W=None, ws=None, ws_bytes=0), OK),
]


@pytest.mark.parametrize("over,code", BOTH + [(dict(logp=None, log_z=None), INVALID)])
def test_head_fwd_refuses(over, code):
    assert head_fwd(**over) == code


@pytest.mark.parametrize("over,code", BOTH + [(dict(d_logp=None), INVALID), (dict(dX=None, dW=None), INVALID), (dict(dX=P + 4), INVALID),
                                              (dict(dW=P + 4), INVALID)])
def test_head_bwd_refuses(over, code):
    assert head_bwd(**over) == code


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,V", [(64, 100), (2048, 32000), (256, 50257), (4096, 131072), (16384, 1 << 20)])
def test_head_workspaces_serve_fewer_rows_and_stay_bounded(d, V, dtype):
    for which, call in ((m.WS_FWD, head_fwd), (m.WS_BWD, head_bwd)):
        size = lambda T: m.modse_head_workspace_size(T, d, V, dtype, which)  # noqa: E731
        last = 0
        for T in (0, 1, 2, 15, 16, 17, 32, 33, 64, 65, 100, 255, 256, 257, 1000, 2048, 2049, 4096, 8192, 8193, 9000, 16384, 20000, 100000):
            now = size(T)
            assert now >= last
            last = now
            if T:
                assert call(T=T, d=d, V=V, dtype=dtype, ws_bytes=now - 1) == WORKSPACE
                # (with all that it needs the call is refused for another reason)
                for t in {1, T // 2, T} - {0}:
                    assert call(T=t, d=d, V=V, dtype=dtype, ws_bytes=now, x=None) == INVALID
        assert last < 4 << 30
    assert m.modse_head_workspace_size(4, d, V, dtype, m.WS_FWD_SAVED, raise_on_error=False) == INVALID
    assert m.modse_head_workspace_size(4, d - 1, V, dtype, m.WS_FWD, raise_on_error=False) == INVALID


def test_head_refuses_tensors_that_the_library_could_not_see():
    x, W, i, f = torch.zeros((4, 64)), torch.zeros((100, 64)), torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    ws = torch.zeros(64, dtype=torch.uint8)
    for a, b, t, p in ((x.bfloat16(), W, i, f), (x, W.bfloat16(), i, f), (x, W, i.long(), f), (x, W, i, f.double()), (x[:, :32], W, i, f),
                       (x, torch.zeros((64, 100)).t(), i, f)):
        assert head_fwd(dtype="f32", x=a, W=b, targets=t, logp=p, log_z=None, ws=ws, ws_bytes=None) == INVALID
        assert head_bwd(dtype="f32", x=a, W=b, targets=t, d_logp=f, logp=p, dX=x, dW=W, ws=ws, ws_bytes=None) == INVALID
    assert head_bwd(dtype="bf16", x=x.bfloat16(), W=W.bfloat16(), targets=i, d_logp=f, logp=f, dX=x.bfloat16(), dW=W.bfloat16(), ws=ws) == INVALID
    # fitting ones come as far as the workspace
    assert head_bwd(dtype="f32", x=x, W=W, targets=i, d_logp=f, logp=f, dX=x, dW=W, ws=ws, ws_bytes=None) == WORKSPACE
