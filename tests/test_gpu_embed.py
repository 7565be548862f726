"""The embedding lookup and its gradient against their float64 oracle.

Tolerances, with u = 2^-24 and h half a step of the type: a looked-up value is the product with the scale rounded to float32 and
then to the type: (h + 2 u) of it.  A gradient is a sum of n terms in float32 in some order, off by at most n u times the sum of
their absolute values, times the scale (one rounding, one of the scale itself), added to an old value (one more)."""
import numpy as np
import pytest
import torch

import paper_2409_12210_amd as m
from oracle import ends_oracle as orc

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24


def host(t):
    return t.detach().double().cpu().numpy()


def normal(shape, dtype, seed, offset=0):
    """N(0, 1), `offset` elements behind an aligned address."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = int(np.prod(shape))
    return torch.empty(n + offset, dtype=TYPE[dtype], device="cuda").normal_(0.0, 1.0, generator=gen)[offset:].view(shape)


def tokens_for(kind, T, V, seed):
    rng = np.random.default_rng(seed)
    if kind == "one":
        t = np.full(T, V - 1)
    elif kind == "zipf":
        t = np.floor((V + 1.0) ** rng.random(T)).astype(np.int64) - 1
        t = rng.permutation(V)[np.clip(t, 0, V - 1)]
    elif kind == "runs":
        t = np.repeat(rng.permutation(V), 1 + rng.integers(0, 40, V))[:T]
        t = rng.permutation(np.concatenate([t, rng.integers(0, V, T - len(t))]))
    else:
        t = rng.integers(0, V, T)
    t = t.astype(np.int32)
    if kind == "absent":
        t[rng.random(T) < 0.5] = -1
        t[rng.random(T) < 0.1] = np.iinfo(np.int32).min
        t[rng.random(T) < 0.1] = V
        t[rng.random(T) < 0.05] = np.iinfo(np.int32).max
    return torch.from_numpy(t).cuda()


def backward(tokens, dX, scale, V, dtype, old=None, stream=None):
    T, d = dX.shape
    dE = torch.full((V, d), float("nan"), device="cuda") if old is None else old.clone()
    ws = torch.empty(m.modse_embed_bwd_workspace_size(T, d, V, dtype), dtype=torch.uint8, device="cuda").fill_(255)
    m.modse_embed_bwd(T, d, V, dtype, tokens, dX, scale, dE, old is not None, ws)
    return dE


def check(T, d, V, dtype, kind, scale=1.5, offset=0, seed=0):
    print("embed", T, d, V, dtype, kind, offset, flush=True)
    tokens = tokens_for(kind, T, V, seed)
    tk = tokens.cpu().numpy()
    E = normal((V, d), dtype, seed + 1, offset)
    out = torch.full((T * d + offset + 16,), 7.0, dtype=TYPE[dtype], device="cuda")
    x = out[offset:offset + T * d].view(T, d)
    m.modse_embed_fwd(T, d, V, dtype, tokens, E, scale, x)
    want = orc.embed_fwd(tk, host(E), scale)
    got = host(x)
    assert (out[offset + T * d:] == 7.0).all() and (out[:offset] == 7.0).all()
    ok = (np.abs(got - want) <= (HALF[dtype] + 2 * U) * np.abs(want)) | (np.isnan(got) & np.isnan(want))
    assert ok.all(), np.argwhere(~ok)[:4]

    dX = normal((T, d), dtype, seed + 2, offset)
    dX[(tokens < 0) | (tokens >= V)] = float("nan")      # rows that are not read
    want, size, count = orc.embed_bwd(tk, host(dX), scale, V)
    n = count[:, None]
    got = host(backward(tokens, dX, scale, V, dtype))
    assert (got[count == 0] == 0).all()
    err = np.abs(got - want)
    assert (err <= (n + 2) * U * size).all(), (np.nanmax(err / np.maximum(size, 1e-30)), np.argwhere(~(err <= (n + 2) * U * size))[:4])

    old = normal((V, d), "f32", seed + 3)
    summed = backward(tokens, dX, scale, V, dtype, old)
    got, o = host(summed), host(old)
    assert np.array_equal(got[count == 0], o[count == 0])
    err = np.abs(got - (o + want))
    assert (err <= (n + 2) * U * size + U * np.abs(o + want) + U * U).all(), np.nanmax(err)
    # the same bits again, with another workspace
    assert torch.equal(summed, backward(tokens, dX, scale, V, dtype, old))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["even", "zipf", "one", "absent"])
@pytest.mark.parametrize("T,d,V", [(1, 64, 100), (7, 1, 3), (8, 33, 1), (65, 257, 300), (513, 100, 257), (1021, 1535, 511), (200, 2049, 5000)])
def test_embedding_and_gradient(T, d, V, dtype, kind):
    check(T, d, V, dtype, kind, offset=T % 3, seed=T + d)


# chunks of 8, 32 and 64 places, and their neighbours; runs that cross many of them
@pytest.mark.parametrize("T", [8191, 8192, 8193, 32767, 32768, 32769, 70000])
@pytest.mark.parametrize("kind", ["runs", "zipf", "one", "absent"])
def test_gradient_of_long_batches(T, kind):
    check(T, 24, 1000, "bf16" if T % 2 else "f32", kind, seed=T)


@pytest.mark.parametrize("V", [255, 256, 257, 512, 131072, 131073, 1 << 20])
def test_vocabularies(V):
    check(3000, 20, V, "f32", "even", seed=V)
    check(3000, 5, V, "bf16", "zipf", seed=V + 1)


def test_wide_rows():
    check(40, 16384, 70, "bf16", "even")
    check(40, 16383, 70, "f32", "zipf")


def test_another_stream_and_many_tokens_of_a_few_rows():
    s = torch.cuda.Stream()
    tokens = tokens_for("even", 5000, 3, 1)
    dX = normal((5000, 300), "bf16", 2)
    want, size, count = orc.embed_bwd(tokens.cpu().numpy(), host(dX), 1.0, 3)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = backward(tokens, dX, 1.0, 3, "bf16")
    s.synchronize()
    assert (np.abs(host(got) - want) <= (count[:, None] + 2) * U * size).all()


def test_capture_and_replay_with_other_tokens():
    T, d, V = 3000, 96, 700
    tokens, E, dX = tokens_for("zipf", T, V, 1), normal((V, d), "bf16", 2), normal((T, d), "bf16", 3)
    x, dE = torch.zeros((T, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((V, d), device="cuda")
    ws = torch.empty(m.modse_embed_bwd_workspace_size(T, d, V, "bf16"), dtype=torch.uint8, device="cuda")

    def both():
        m.modse_embed_fwd(T, d, V, "bf16", tokens, E, 2.0, x)
        m.modse_embed_bwd(T, d, V, "bf16", tokens, dX, 0.5, dE, False, ws)
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in range(4):
        tokens.copy_(tokens_for(("zipf", "one", "absent", "even")[seed], T, V, seed))
        ws.fill_(seed * 80)
        dE.fill_(float("nan"))
        x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = x.clone(), dE.clone()
        both()
        torch.cuda.synchronize()
        assert torch.equal(got[0].nan_to_num(9.0), x.nan_to_num(9.0)) and torch.equal(got[1], dE)
        want, size, count = orc.embed_bwd(tokens.cpu().numpy(), host(dX), 0.5, V)
        assert (np.abs(host(dE) - want) <= (count[:, None] + 2) * U * size).all()
