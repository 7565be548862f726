"""Tensors that the operators around the layer would read as something else: other types, gaps between the elements.  All are refused
before anything is launched; the tensors are the CPU's."""
import pytest
import torch

import paper_2409_12210_amd as m

INVALID, UNSUPPORTED = 1, 2
NO = dict(stream=0, raise_on_error=False)
BF, F32, I32, I64 = torch.bfloat16, torch.float32, torch.int32, torch.int64


def z(*shape, dtype=F32):
    return torch.zeros(shape, dtype=dtype)


def refused(call, args, wrong):
    """Every argument of `wrong` in turn, with all others as they should be; those then pass (T = 0 launches nothing)."""
    assert call(**args) == 0
    for name, bad in wrong:
        assert call(**{**args, name: bad}) == INVALID, (name, bad.dtype, bad.stride())


def test_norm_forward():
    def call(**a):
        return m.modse_norm_fwd(0, 8, "bf16", a["x"], a["residual"], a["gamma"], 1e-6, a["y"], a["h"], a["rstd"], a["q"], a["scale"], **NO)
    args = {k: z(4, 8, dtype=BF) for k in ("x", "residual", "y", "h")}
    args.update(gamma=z(8, dtype=BF), rstd=z(4), scale=z(4), q=torch.zeros((4, 8), dtype=torch.uint8))
    wrong = [(k, z(4, 8)) for k in ("x", "residual", "y", "h")] + [(k, z(4, 16, dtype=BF)[:, :8]) for k in ("x", "residual", "y", "h")]
    wrong += [("gamma", z(8)), ("gamma", z(16, dtype=BF)[::2]), ("rstd", z(4, dtype=BF)), ("scale", z(4, dtype=torch.float64)),
              ("q", z(4, 8, dtype=BF)), ("q", torch.zeros((4, 16), dtype=torch.uint8)[:, :8])]
    refused(call, args, wrong)
    assert call(**{**args, "q": torch.zeros((4, 8), dtype=torch.float8_e4m3fn)}) == 0


def test_norm_backward():
    def call(**a):
        return m.modse_norm_bwd(0, 8, "f32", a["h"], a["gamma"], a["rstd"], a["dY"], a["dH"], a["dX"], a["dgamma"], False, None, **NO)
    args = {k: z(4, 8) for k in ("h", "dY", "dH", "dX")}
    args.update(gamma=z(8), rstd=z(4), dgamma=z(8))
    wrong = [(k, z(4, 8, dtype=BF)) for k in ("h", "dY", "dH", "dX")] + [(k, z(8, 4).t()) for k in ("h", "dY", "dH", "dX")]
    refused(call, args, wrong + [("gamma", z(8, dtype=BF)), ("rstd", z(1).expand(4)), ("dgamma", z(8, dtype=BF)), ("dgamma", z(16)[::2])])


def test_log_probabilities():
    def call(**a):
        return m.modse_logprobs_fwd(0, 10, "bf16", a["logits"], a["targets"], a["logp"], a["stats"], a["entropy"], 3, a["top_idx"],
                                    a["top_logp"], None, **NO)
    args = dict(logits=z(4, 16, dtype=BF)[:, :10], targets=z(4, dtype=I32), logp=z(4), stats=z(4, 2), entropy=z(4), top_idx=z(4, 3, dtype=I32),
                top_logp=z(4, 3))
    refused(call, args, [("targets", z(4, dtype=I64)), ("targets", z(4, 2, dtype=I32)[:, 1]), ("targets", z(4)), ("logits", z(4, 10)),
                         ("logp", z(4, dtype=BF)), ("stats", z(4, 4)[:, :2]), ("entropy", z(8)[::2]), ("top_idx", z(4, 3, dtype=I64)),
                         ("top_logp", z(4, 3, dtype=torch.float64)), ("top_logp", z(4, 5)[:, :3])])


def test_their_gradient():
    def call(**a):
        return m.modse_logprobs_bwd(0, 10, "f32", a["logits"], a["targets"], a["stats"], a["entropy"], a["d_logp"], a["d_entropy"],
                                    a["d_logits"], **NO)
    args = dict(logits=z(4, 10), targets=z(4, dtype=I32), stats=z(4, 2), entropy=z(4), d_logp=z(4), d_entropy=z(4), d_logits=z(4, 12)[:, :10])
    refused(call, args, [("targets", z(4, dtype=I64)), ("d_logp", z(1).expand(4)), ("d_logp", z(4, dtype=BF)), ("d_entropy", torch.zeros(()).expand(4)),
                         ("stats", z(4, 2, dtype=torch.float64)), ("entropy", z(4, dtype=BF)), ("logits", z(4, 10, dtype=BF)),
                         ("d_logits", z(4, 10, dtype=BF))])


def test_the_error_says_what_was_wrong():
    with pytest.raises(m.ModseError, match="int64") as e:
        m.modse_logprobs_fwd(4, 10, "f32", z(4, 10), z(4, dtype=I64), z(4), None, None, 0, None, None, None, stream=0)
    assert e.value.code == INVALID
    # a type that the library does not know stays the library's to refuse
    assert m.modse_norm_fwd(4, 8, "fp16", z(4, 8, dtype=torch.float16), None, z(8, dtype=torch.float16), 1e-6, z(4, 8), None, None, **NO) == UNSUPPORTED
