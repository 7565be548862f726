"""The work that the operators at both ends of a model of MoDSE layers are measured by: the embedding lookup and its gradient
(`modse_embed_fwd`, `modse_embed_bwd`), the log probabilities of the next tokens straight from the last hidden rows and the
output matrix, with their gradients (`modse_head_fwd`, `modse_head_bwd`), and the dropout on the stream between the two
(`modse_dropout_fwd`, `modse_dropout_bwd`).

    embed    x_t = scale E[token_t]; a negative token is none: zeros.  form "train": the lookup, then the gradient of E in float32,
             dE_v = scale times the sum of dX_t over the tokens t that are v, zeros for those that do not occur.
    head     log softmax(x W^T)[target] and log of the sum of exponentials, float32, form "score".  form "train": the log
             probabilities and the gradients of loss = sum_t d_logp[t] logp[t], dX in the layer's type and dW in float32.  A
             negative target is no target: log probability 0 and no gradient.
    dropout  y = residual + keep x / (1 - p), then dX = keep dY / (1 - p).  keep: 16 bits an element of Philox-4x32 with seven
             rounds (Salmon, Moraes, Dror and Shaw 2011), key = seed, counter = (index / 8, call, offset); an element is kept
             where its bits are at least round(65536 p), and 1 - p is what that leaves.

Values are those that the operators meet: tokens by Zipf's law, hidden rows and gradients N(0, 1), logits of standard deviation 2.5
with the target's raised.
"""
import math

import numpy as np
import torch

own = False

NO_TOKEN = -1


def _embed(name, form, n_tokens, d_model, vocab, dtype="bf16", scaled=True, absent=0.0):
    return {"name": name, "op": "embed", "form": form, "n_tokens": n_tokens, "d_model": d_model, "vocab": vocab, "dtype": dtype,
            "scaled": scaled, "absent": absent}


def _head(name, form, n_tokens, d_model, vocab, dtype="bf16", absent=0.05):
    return {"name": name, "op": "head", "form": form, "n_tokens": n_tokens, "d_model": d_model, "vocab": vocab, "dtype": dtype,
            "absent": absent}


def _dropout(name, n_tokens, d_model, p, dtype="bf16", residual=True):
    return {"name": name, "op": "dropout", "form": "train", "n_tokens": n_tokens, "d_model": d_model, "p": p, "dtype": dtype,
            "residual": residual}


def listed():
    return [
        # serving, one decoded token: latency alone counts
        _embed("embed_decode_1", "lookup", 1, 4096, 131072),
        # serving, a batched prompt pass
        _embed("embed_prefill_16384", "lookup", 16384, 2048, 32000, scaled=False),
        # a training step at the full batch, a few tokens of padding
        _embed("embed_train_32768", "train", 32768, 2048, 32000, absent=0.03),
        # float32: a small step over an odd vocabulary, rows that start at every alignment
        _embed("embed_train_f32_1021", "train", 1021, 1535, 50257, dtype="f32"),
        # serving: the log probability of one drafted token, bound by the output matrix
        _head("head_decode_1", "score", 1, 4096, 131072, absent=0.0),
        # serving: those of a decode batch
        _head("head_decode_64", "score", 64, 2048, 32000, absent=0.0),
        # scoring a corpus
        _head("head_score_16384", "score", 16384, 2048, 32000),
        # float32: a small training step over an odd vocabulary
        _head("head_train_f32_1021", "train", 1021, 256, 50257, dtype="f32"),
        # a micro-batch over a large vocabulary
        _head("head_train_2048", "train", 2048, 2048, 131072),
        # a training step's loss
        _head("head_train_16384", "train", 16384, 2048, 32000),
        # a small float32 layer's output onto the stream
        _dropout("dropout_512", 512, 256, 0.5, dtype="f32"),
        # a training step at the full batch
        _dropout("dropout_32768", 32768, 2048, 0.1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: the operator first, then its form, sizes over the logarithm of their range."""
    op = rng.choice(["embed", "embed", "head", "head", "head", "dropout"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "embed":
        d = rng.choice([2048, 4096, _log_int(rng, 64, 8200)])
        v = rng.choice([32000, 50257, 131072, _log_int(rng, 200, 160000)])
        case = _embed("", rng.choice(["lookup", "train", "train"]), _log_int(rng, 1, 32768), d, v, dtype, rng.random() < 0.5,
                      rng.choice([0.0, 0.0, 0.03, 0.5]))
        most = work(_embed("", "train", 32768, 2048, 32000))["bytes"]
        while work(case)["bytes"] > most:
            case["n_tokens"], case["d_model"] = max(1, case["n_tokens"] // 2), max(64, case["d_model"] * 2 // 3)
    elif op == "head":
        d = rng.choice([256, 2048, 4096, 32 * rng.randint(2, 160)])
        v = rng.choice([32000, 50257, 131072, _log_int(rng, 200, 160000)])
        case = _head("", rng.choice(["score", "score", "train"]), _log_int(rng, 1, 16384), d, v, dtype, rng.choice([0.0, 0.05, 0.5]))
        # (the same time in float32, at about a tenth of the rate)
        most = work(_head("", "train", 16384, 2048, 32000))["flops"] / (10 if dtype == "f32" else 1)
        while work(case)["flops"] > most:
            case["n_tokens"] = max(1, case["n_tokens"] // 2)
    else:
        d = rng.choice([256, 2048, 4096, _log_int(rng, 64, 8200)])
        t = min(_log_int(rng, 1, 32768), 32768 * 2048 // d)
        case = _dropout("", (t + 1) // 2 if dtype == "f32" else t, d, rng.choice([0.05, 0.1, 0.5, round(rng.uniform(0, 1), 3)]), dtype,
                        rng.random() < 0.7)
    del case["name"]
    return case


def work(case):
    b, t, d = 4 if case["dtype"] == "f32" else 2, float(case["n_tokens"]), float(case["d_model"])
    if case["op"] == "embed":
        look = 2 * t * d * b + 4 * t
        if case["form"] == "lookup":
            return {"bytes": look, "flops": t * d}
        return {"bytes": look + t * d * b + case["vocab"] * d * 4, "flops": 3 * t * d}
    if case["op"] == "head":
        v = float(case["vocab"])
        if case["form"] == "score":
            return {"bytes": (t + v) * d * b + 12 * t, "flops": 2 * t * v * d}
        return {"bytes": (2 * t + v) * d * b + v * d * 4 + 12 * t, "flops": 6 * t * v * d}
    n = t * d
    return {"bytes": n * b * (4 + case["residual"]), "flops": 3 * n}


class _State:
    pass


def prepare(case, seed):
    s = _State()
    s.case, s.op = case, case["op"]
    s.dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t, d = case["n_tokens"], case["d_model"]

    def normal(shape, sigma=1.0, dtype=None):
        return torch.empty(shape, dtype=dtype or s.dtype, device="cuda").normal_(0.0, sigma, generator=gen)

    def empty(shape, dtype=None):
        return torch.empty(shape, dtype=dtype or s.dtype, device="cuda")

    def tokens(v):
        """By Zipf's law: the token of rank r about as often as 1 / r; some are none."""
        rank = (v + 1.0) ** torch.rand(t, generator=gen, device="cuda", dtype=torch.float64)
        ids = torch.randperm(v, generator=gen, device="cuda")[(rank.long() - 1).clamp(0, v - 1)]
        none = torch.rand(t, generator=gen, device="cuda") < case["absent"]
        return ids, torch.where(none, torch.full_like(ids, NO_TOKEN), ids).to(torch.int32)

    f32 = torch.float32
    if s.op == "embed":
        v = case["vocab"]
        s.E, s.scale = normal((v, d), 0.02), float(np.float32(math.sqrt(d))) if case["scaled"] else 1.0
        s.tokens, s.x = tokens(v)[1], empty((t, d))
        if case["form"] == "train":
            s.dX, s.dE = normal((t, d)), empty((v, d), f32)
    elif s.op == "head":
        v = case["vocab"]
        s.W = normal((v, d), 2.5 / math.sqrt(d))
        ids, s.targets = tokens(v)
        s.x = (normal((t, d), dtype=f32) + 0.8 * s.W[ids].float()).to(s.dtype)   # the model knows something of its targets
        s.logp, s.log_z = empty((t,), f32), empty((t,), f32)
        if case["form"] == "train":
            # the mean over the tokens with a target, each with a weight of its own
            s.d_logp = -(1.0 + normal((t,), 0.2, f32)).abs() / t
            s.dX, s.dW = empty((t, d)), empty((v, d), f32)
    else:
        s.x, s.y, s.dY, s.dX = normal((t, d)), empty((t, d)), normal((t, d)), empty((t, d))
        s.residual = normal((t, d)) if case["residual"] else None
        s.rng = torch.tensor([seed * 0x9E3779B97F4A7C15 % 2 ** 63, 12345 + seed], dtype=torch.int64, device="cuda")
        s.call = 3
    return s


# ---------------------------------------------------------------- the plain forms

def _plain_embed(s):
    has = (s.tokens >= 0)[:, None]
    at = s.tokens.clamp_min(0).long()
    out = {"x": torch.where(has, s.E[at].float() * s.scale, 0.0).to(s.dtype)}
    if s.case["form"] == "train":
        dE = torch.zeros(s.E.shape, device="cuda")
        out["dE"] = dE.index_add_(0, at, torch.where(has, s.dX.float(), 0.0)) * s.scale
    return out


def _plain_head(s):
    x, W = s.x.float(), s.W.float()
    z = x @ W.t()
    m = z.amax(1, keepdim=True)
    z -= m
    log_total = z.exp().sum(1, keepdim=True).log()
    has = (s.targets >= 0)[:, None]
    at = s.targets.clamp_min(0).long()[:, None]
    logp = torch.where(has, z.gather(1, at) - log_total, 0.0)[:, 0]
    if s.case["form"] == "score":
        return {"logp": logp, "log_z": (m + log_total)[:, 0]}
    w = torch.where(has, s.d_logp[:, None], 0.0)
    g = -w * (z - log_total).exp()
    g.scatter_add_(1, at, w)
    return {"logp": logp, "dX": (g @ W).to(s.dtype), "dW": g.t() @ x}


def _philox(index, call, seed, offset):
    """Four words of 32 bits for every value of `index`, all in integers of 64 bits."""
    low = 0xFFFFFFFF

    def product(a, b):
        part, rest = a * (b >> 16), a * (b & 0xFFFF)
        return (part + (rest >> 16)) >> 16 & low, ((part << 16) + rest) & low

    k0, k1 = seed & low, seed >> 32 & low
    c = [index & low, torch.full_like(index, call), torch.zeros_like(index) + (offset & low), torch.zeros_like(index) + (offset >> 32 & low)]
    for _ in range(7):
        (h0, l0), (h1, l1) = product(0xD2511F53, c[0]), product(0xCD9E8D57, c[2])
        c = [h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c


def _plain_dropout(s):
    n, limit = s.x.numel(), round(s.case["p"] * 65536)
    words = torch.stack(_philox(torch.arange((n + 7) // 8, device="cuda"), s.call, s.rng[0], s.rng[1]), 1)
    bits = torch.stack([words & 0xFFFF, words >> 16], 2).view(-1)[:n].view(s.x.shape)
    keep, scale = bits >= limit, 65536.0 / (65536 - limit) if limit < 65536 else 0.0
    y = torch.where(keep, s.x.float() * scale, 0.0)
    if s.residual is not None:
        y = y + s.residual.float()
    return {"y": y.to(s.dtype), "dX": torch.where(keep, s.dY.float() * scale, 0.0).to(s.dtype)}


# ---------------------------------------------------------------- the framework's calls

def _own_embed(s):
    import paper_2409_12210_amd as modse

    case = s.case
    t, d, v, dt = case["n_tokens"], case["d_model"], case["vocab"], case["dtype"]
    modse.modse_embed_fwd(t, d, v, dt, s.tokens, s.E, s.scale, s.x)
    if case["form"] != "train":
        return {"x": s.x}
    if not hasattr(s, "ws"):
        s.ws = torch.empty(modse.modse_embed_bwd_workspace_size(t, d, v, dt), dtype=torch.uint8, device="cuda")
    modse.modse_embed_bwd(t, d, v, dt, s.tokens, s.dX, s.scale, s.dE, False, s.ws)
    return {"x": s.x, "dE": s.dE}


def _own_head(s):
    import paper_2409_12210_amd as modse

    case = s.case
    t, d, v, dt = case["n_tokens"], case["d_model"], case["vocab"], case["dtype"]
    train = case["form"] == "train"
    if not hasattr(s, "ws"):
        which = modse.WS_BWD if train else modse.WS_FWD
        s.ws = torch.empty(modse.modse_head_workspace_size(t, d, v, dt, which), dtype=torch.uint8, device="cuda")
    if not train:
        modse.modse_head_fwd(t, d, v, dt, s.x, s.W, s.targets, s.logp, s.log_z, s.ws)
        return {"logp": s.logp, "log_z": s.log_z}
    modse.modse_head_bwd(t, d, v, dt, s.x, s.W, s.targets, s.d_logp, s.logp, s.dX, s.dW, False, s.ws)
    return {"logp": s.logp, "dX": s.dX, "dW": s.dW}


def _own_dropout(s):
    import paper_2409_12210_amd as modse

    case = s.case
    t, d, dt = case["n_tokens"], case["d_model"], case["dtype"]
    modse.modse_dropout_fwd(t, d, dt, s.x, s.residual, case["p"], s.rng, s.call, s.y)
    modse.modse_dropout_bwd(t, d, dt, s.dY, case["p"], s.rng, s.call, s.dX)
    return {"y": s.y, "dX": s.dX}


def run(s):
    if s.op == "embed":
        return _own_embed(s) if own else _plain_embed(s)
    if s.op == "head":
        return _own_head(s) if own else _plain_head(s)
    return _own_dropout(s) if own else _plain_dropout(s)


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_embed(s):
    there = s.tokens >= 0
    ids = s.tokens[there].long()
    x = torch.zeros(s.x.shape, dtype=torch.float64, device="cuda")
    x[there] = s.E[ids].double() * s.scale
    if s.case["form"] != "train":
        return {"x": x}
    order = torch.argsort(ids, stable=True)
    dE = torch.zeros(s.E.shape, dtype=torch.float64, device="cuda")
    dE.index_put_((ids[order],), s.dX[there][order].double() * s.scale, accumulate=True)
    return {"x": x, "dE": dE}


def _exact_head(s):
    t, train = len(s.targets), s.case["form"] == "train"
    W = s.W.double()
    Wt = W.t().contiguous()
    got, dW = {}, torch.zeros_like(W) if train else None
    rows = max(1, (1 << 27) // len(W))
    for at in range(0, t, rows):
        x, tg = s.x[at:at + rows].double(), s.targets[at:at + rows].long()
        here = torch.arange(len(tg), device="cuda")
        logits = x.mm(Wt)
        lse = logits.logsumexp(1)
        there = tg >= 0
        logp = torch.where(there, logits[here, tg.clamp_min(0)] - lse, 0.0)
        if train:
            g = (logits - lse[:, None]).exp_().neg_()
            g[here, tg.clamp_min(0)] += 1.0
            g *= torch.where(there, s.d_logp[at:at + rows].double(), 0.0)[:, None]
            part = {"logp": logp, "dX": g.mm(W)}
            dW += g.t().contiguous().mm(x)
        else:
            part = {"logp": logp, "log_z": lse}
        for k, val in part.items():
            got.setdefault(k, []).append(val)
    got = {k: torch.cat(val) for k, val in got.items()}
    if train:
        got["dW"] = dW
    return got


def _exact_dropout(s):
    n, p = s.x.numel(), s.case["p"]
    seed, offset = s.rng.cpu().numpy().astype(np.uint64)
    low, half = np.uint64(2 ** 32 - 1), np.uint64(32)
    blocks = -(-n // 8)
    c0, c1 = np.arange(blocks, dtype=np.uint64), np.full(blocks, s.call, np.uint64)
    c2, c3 = np.full(blocks, offset & low), np.full(blocks, offset >> half)
    k0, k1 = int(seed & low), int(seed >> half)
    for r in range(7):
        p0, p1 = c0 * np.uint64(0xD2511F53), c2 * np.uint64(0xCD9E8D57)
        c0, c1, c2, c3 = ((p1 >> half) ^ c1 ^ np.uint64((k0 + r * 0x9E3779B9) % 2 ** 32), p1 & low,
                          (p0 >> half) ^ c3 ^ np.uint64((k1 + r * 0xBB67AE85) % 2 ** 32), p0 & low)
    words = np.empty((blocks, 4), np.uint32)
    words[:, 0], words[:, 1], words[:, 2], words[:, 3] = c0, c1, c2, c3
    limit = round(65536 * p)
    kept = words.reshape(-1).view(np.uint16)[:n] >= np.uint32(limit)       # (the low half first, as the machine has it)
    kept = torch.from_numpy(kept).cuda().view(s.x.shape)
    factor = 65536 / max(65536 - limit, 1)
    y = s.x.double().mul_(factor).masked_fill_(~kept, 0.0)
    if s.residual is not None:
        y += s.residual.double()
    return {"y": y, "dX": s.dY.double().mul_(factor).masked_fill_(~kept, 0.0)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"embed": _exact_embed, "head": _exact_head, "dropout": _exact_dropout}[s.op](s)
