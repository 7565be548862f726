"""The oracle of the operators at both ends of a model against torch and published values."""
import numpy as np
import torch

from oracle import ends_oracle as orc


def test_philox_gives_its_published_words():
    # known answers of the generator's authors, seven rounds and ten
    full = (0xFFFFFFFF,) * 4
    assert orc.philox4x32((0,) * 4, (0, 0), 7) == [0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48]
    assert orc.philox4x32((0,) * 4, (0, 0), 10) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert orc.philox4x32(full, (0xFFFFFFFF,) * 2, 10) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


def test_embedding_is_torchs():
    rng = np.random.default_rng(0)
    E, dX = rng.normal(size=(9, 5)), rng.normal(size=(30, 5))
    tokens = rng.integers(0, 9, 30)
    e = torch.tensor(E, requires_grad=True)
    x = 2.5 * torch.nn.functional.embedding(torch.tensor(tokens), e)
    (x * torch.tensor(dX)).sum().backward()
    assert np.allclose(orc.embed_fwd(tokens, E, 2.5), x.detach().numpy(), atol=1e-14)
    dE, size, count = orc.embed_bwd(tokens, dX, 2.5, 9)
    assert np.allclose(dE, e.grad.numpy(), atol=1e-13) and count.sum() == 30 and (size >= np.abs(dE) - 1e-12).all()
    odd = orc.embed_fwd([-1, 9, 3], E, 1.0)
    assert (odd[0] == 0).all() and np.isnan(odd[1]).all() and (odd[2] == E[3]).all()
    assert orc.embed_bwd([-1, 9, 3], dX[:3], 1.0, 9)[2].tolist() == [0, 0, 0, 1, 0, 0, 0, 0, 0]


def test_head_is_torchs_cross_entropy():
    rng = np.random.default_rng(1)
    x, W, w = rng.normal(size=(7, 6)), rng.normal(size=(11, 6)), rng.normal(size=7)
    targets = rng.integers(0, 11, 7)
    targets[2] = -1
    tx, tw = torch.tensor(x, requires_grad=True), torch.tensor(W, requires_grad=True)
    logp = -torch.nn.functional.cross_entropy(tx @ tw.T, torch.tensor(targets), ignore_index=-1, reduction="none")
    (logp * torch.tensor(w)).sum().backward()
    got = orc.head(x, W, targets, w)
    assert np.allclose(got[0], logp.detach().numpy()) and np.allclose(got[1], torch.logsumexp(tx @ tw.T, 1).detach().numpy())
    assert np.allclose(got[2], tx.grad.numpy()) and np.allclose(got[3], tw.grad.numpy())
    assert np.isnan(orc.head(x, W, [11] * 7)[0]).all()


def test_dropout_keeps_its_share_and_its_mean():
    bits = orc.dropout_bits(40000, 7, 1 << 40, 3)
    assert bits.min() >= 0 and bits.max() < 65536
    for p in (0.0, 0.1, 0.5, 1.0):
        y, kept = orc.dropout(np.ones(40000), None, p, bits)
        # (four standard deviations of a share of 40000)
        assert abs(kept.mean() - (1 - p)) <= 4 * np.sqrt(p * (1 - p) / 40000) + 2.0 ** -17
        assert abs(y.mean() - (p < 1)) <= 4 * np.sqrt(p / max(1 - p, 1e-9) / 40000) * (p < 1) + 1e-12
    assert np.array_equal(bits, orc.dropout_bits(40007, 7, 1 << 40, 3)[:40000])
    assert not np.array_equal(bits, orc.dropout_bits(40000, 7, 1 << 40, 4))
    y, _ = orc.dropout(np.array([np.inf, np.nan, 1.0]), np.array([1.0, 2.0, 3.0]), 1.0, bits[:3])
    assert y.tolist() == [1.0, 2.0, 3.0]
