"""The work that the operators around the MoDSE layer are measured by: the norm in front of it (`modse_norm_fwd`,
`modse_norm_bwd`), the log probabilities that a model of such layers is trained, scored and sampled by
(`modse_logprobs_fwd`, `modse_logprobs_bwd`), and the orthogonalised update of its expert matrices
(`modse_orthogonalize`).

    norm      h = x + residual, y = gamma h / sqrt(mean(h^2) + eps).  form "infer": y and h.  "q8": h, and y in e4m3 with one
              float32 scale per `group` columns (0: per row), y of the layer's type too where the router needs it.
              "train": y and h, then the backward pass: the gradient of the stream (that of y through the norm plus the
              one that arrives along the residual) and of gamma.
    logprobs  log softmax(logits)[target] in float32, the entropy of the distribution, the `top` most probable entries (ties
              to the lower index, no entry of logit -inf: index -1 in its place).  A negative target is no target: 0.
              form "train": the log probabilities, then the gradient of the logits.
    ortho     every matrix G of a set: X = G / (|G| + eps), then X <- a X + (b A + c A^2) X with A = X X^T, once per step.

Values are those that the operators meet: x, residual and gradients N(0, 1), gamma near 1, logits of standard deviation 2.5
with the target's raised, updates of a few strong directions in noise.
"""
import math

import torch

own = False

EPS = 1e-6
ORTHO_EPS = 1e-7
ORTHO_COEFFS = (3.4445, -4.7750, 2.0315)   # a, b, c of the quintic of every step
NO_TARGET = -1

# hidden widths of this repository's layers: d_model 2048, d_model 256, and 64 narrow experts of d_model 2048
WIDTHS_2048 = "2816,8448,4224,7040,4928,6336,5632,5632"
WIDTHS_256 = "128,384,192,320,224,288,256,256"
WIDTHS_FINE = ",".join("%d,%d" % (704 - w, 704 + w) for w in (32 * (p % 12) for p in range(32)))


def _norm(name, form, n_tokens, d_model, dtype="bf16", residual=True, group=0, keep_y=False):
    return {"name": name, "op": "norm", "form": form, "n_tokens": n_tokens, "d_model": d_model, "dtype": dtype,
            "residual": residual, "group": group, "keep_y": keep_y}


def _logprobs(name, form, n_tokens, vocab, dtype="bf16", top=0, entropy=False, pad=0, masked=0.0):
    return {"name": name, "op": "logprobs", "form": form, "n_tokens": n_tokens, "vocab": vocab, "dtype": dtype, "top": top,
            "entropy": entropy, "pad": pad, "masked": masked}


def _ortho(name, d_model, d_ff, dtype="f32", steps=5, idle=0):
    return {"name": name, "op": "ortho", "d_model": d_model, "d_ff": d_ff, "dtype": dtype, "steps": steps, "idle": idle}


def listed():
    return [
        # serving, one decoded token in front of the widest layer: latency alone counts
        _norm("norm_decode_1", "infer", 1, 4096),
        # serving, a decode batch whose experts run in 8 bits; the router reads y itself
        _norm("norm_q8_decode_64", "q8", 64, 4096, keep_y=True),
        # serving, a batched prompt pass into 8-bit experts with a scale per 128 columns
        _norm("norm_q8_prefill_16384", "q8", 16384, 2048, group=128),
        # a training step at the full batch
        _norm("norm_train_32768", "train", 32768, 2048),
        # float32: a small training step of a width that is not a multiple of the vector loads
        _norm("norm_train_f32_1021", "train", 1021, 1535, dtype="f32"),
        # serving: the next token of one sequence, with the alternatives that an interface shows
        _logprobs("logprobs_decode_1", "score", 1, 131072, top=5, entropy=True),
        # serving: a decode batch under a grammar that leaves one entry in ten
        _logprobs("logprobs_decode_64", "score", 64, 32000, top=20, entropy=True, masked=0.9),
        # scoring a corpus: float32 logits over an odd vocabulary, rows that start at every alignment
        _logprobs("logprobs_score_2047", "score", 2047, 50257, dtype="f32", top=5),
        # the loss of a training step, bf16 logits in rows that are padded for the product that makes them
        _logprobs("logprobs_train_16384", "train", 16384, 32000, pad=64),
        # the expert matrices of the small float32 layer: many tiny products
        _ortho("ortho_256", 256, WIDTHS_256),
        # 64 narrow experts, a few of which saw no token (their gradients are zero), updates kept in bf16
        _ortho("ortho_fine", 2048, WIDTHS_FINE, dtype="bf16", idle=3),
        # the expert matrices of one full layer
        _ortho("ortho_layer", 2048, WIDTHS_2048),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: the operator first, then its form, sizes over the logarithm of their range."""
    op = rng.choice(["norm", "norm", "logprobs", "logprobs", "ortho"])
    if op == "norm":
        d = rng.choice([2048, 4096, 32 * rng.randint(8, 256), _log_int(rng, 200, 8200)])
        t = min(_log_int(rng, 1, 32768), 32768 * 2048 // d)
        form = rng.choice(["infer", "q8", "train"])
        case = _norm("", form, t, d, rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.7)
        if form == "q8":
            case["group"], case["keep_y"] = rng.choice([0, 128]), rng.random() < 0.5
        if case["dtype"] == "f32":
            case["n_tokens"] = (t + 1) // 2
    elif op == "logprobs":
        v = rng.choice([32000, 50257, 131072, _log_int(rng, 1000, 160000)])
        t = min(_log_int(rng, 1, 16384), 16384 * 32000 // (2 * v))
        case = _logprobs("", rng.choice(["score", "train"]), max(t, 1), v, rng.choice(["bf16", "bf16", "f32"]),
                         entropy=rng.random() < 0.5, pad=rng.choice([0, 0, -v % 64]), masked=rng.choice([0.0, 0.0, 0.3, 0.95]))
        if case["form"] == "score":
            case["top"] = rng.choice([0, 1, 5, 20])
    else:
        d = rng.choice([256, 512, 1024, 2048, _log_int(rng, 64, 1500)])
        step = rng.choice([32, 32, 1])
        n = rng.choice([1, 2, 4, 8, 16])
        widths = [step * max(1, int(d * rng.uniform(0.3, 3.0)) // step) for _ in range(n)]
        case = _ortho("", d, ",".join(map(str, widths)), rng.choice(["f32", "f32", "bf16"]), rng.choice([3, 5, 5]),
                      rng.choice([0, 0, 1]) if n > 1 else 0)
        # no drawn case costs more than the largest listed one
        while work(case)["flops"] > work(_ortho("", 2048, WIDTHS_2048))["flops"]:
            widths = widths[1:]
            case["d_ff"] = ",".join(map(str, widths))
    del case["name"]
    return case


def _widths(case):
    return [int(f) for f in case["d_ff"].split(",")]


def _shapes(case):
    """The matrices of the set: W1 and W3 of every expert, then its W2."""
    d, f = case["d_model"], _widths(case)
    return [(w, d) for w in f] * 2 + [(d, w) for w in f]


def work(case):
    if case["op"] == "ortho":
        flops = nbytes = 0.0
        for r, c in _shapes(case):
            m, n = min(r, c), max(r, c)
            # A is symmetric, and so is its square: half of either product is enough
            flops += case["steps"] * (m * (m + 1.0) * n + m * (m + 1.0) * m + 2.0 * m * m * n)
            nbytes += r * c * (4 + (4 if case["dtype"] == "f32" else 2))
        return {"bytes": nbytes, "flops": flops}
    b, t = 4 if case["dtype"] == "f32" else 2, case["n_tokens"]
    if case["op"] == "logprobs":
        n = float(t) * case["vocab"]
        small = t * (8 + 4 * case["entropy"] + 8 * case["top"])
        if case["form"] == "score":
            return {"bytes": n * b + small, "flops": 4 * n}
        return {"bytes": 3 * n * b + small, "flops": 8 * n}       # the loss has to be known before its gradient: read twice
    n = float(t) * case["d_model"]
    inputs = n * b * (1 + case["residual"])
    hb = n * b if case["residual"] else 0.0                       # without a residual h is x and is not written
    if case["form"] == "infer":
        return {"bytes": inputs + n * b + hb, "flops": 5 * n}
    if case["form"] == "q8":
        scales = t * (-(-case["d_model"] // case["group"]) if case["group"] else 1) * 4
        return {"bytes": inputs + n + hb + scales + (n * b if case["keep_y"] else 0), "flops": 7 * n}
    back = n * b * (3 + case["residual"])                         # h, dy (and the stream's gradient), dx
    return {"bytes": inputs + n * b + hb + back, "flops": 15 * n}


class _State:
    pass


def prepare(case, seed):
    s = _State()
    s.case, s.op = case, case["op"]
    s.dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(shape, sigma=1.0, mean=0.0, dtype=None):
        return torch.empty(shape, dtype=dtype or s.dtype, device="cuda").normal_(mean, sigma, generator=gen)

    def empty(shape, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda")

    f32, i32 = torch.float32, torch.int32
    if s.op == "norm":
        t, d = case["n_tokens"], case["d_model"]
        s.x, s.gamma = normal((t, d)), normal((d,), 0.1, 1.0)
        s.residual = normal((t, d)) if case["residual"] else None
        s.y = empty((t, d), s.dtype) if case["form"] != "q8" or case["keep_y"] else None
        s.h = empty((t, d), s.dtype) if case["residual"] else None
        s.rstd = empty((t,), f32) if case["form"] == "train" else None
        if case["form"] == "q8":
            s.groups = -(-d // case["group"]) if case["group"] else 1
            s.q, s.scale = empty((t, d), torch.float8_e4m3fn), empty((t, s.groups), f32)
        if case["form"] == "train":
            s.dY, s.dX, s.dgamma = normal((t, d)), empty((t, d), s.dtype), empty((d,), f32)
            s.dH = normal((t, d)) if case["residual"] else None   # what arrives along the residual stream
    elif s.op == "logprobs":
        t, v = case["n_tokens"], case["vocab"]
        s.logits = normal((t, v + case["pad"]), 2.5)[:, :v]
        at = torch.randint(0, v, (t,), generator=gen, device="cuda")
        if case["masked"]:
            s.logits.masked_fill_(torch.rand((t, v), generator=gen, device="cuda") < case["masked"], -math.inf)
        lifted = normal((t,), 2.5, 8.0)                           # the model knows something of its targets
        s.logits[torch.arange(t, device="cuda"), at] = lifted
        none = torch.rand((t,), generator=gen, device="cuda") < 0.05
        s.targets = torch.where(none, torch.full_like(at, NO_TARGET), at).to(i32)
        s.logp, s.stats = empty((t,), f32), empty((t, 2), f32)
        s.entropy = empty((t,), f32) if case["entropy"] else None
        top = case["top"]
        s.top_idx, s.top_logp = (empty((t, top), i32), empty((t, top), f32)) if top else (None, None)
        if case["form"] == "train":
            # the mean over the tokens with a target, each with a weight of its own; now and then an entropy bonus
            s.d_logp = -normal((t,), 0.2, 1.0, f32).abs() / t
            s.d_entropy = torch.full((t,), -0.01 / t, device="cuda") if case["entropy"] else None
            s.d_logits = empty((t, v + case["pad"]), s.dtype)[:, :v]
    else:
        # the updates lie packed, as the layer's weights do
        shapes, n = _shapes(case), len(_widths(case))
        sizes = [r * c for r, c in shapes]
        s.packed = [empty((sum(sizes[i * n:(i + 1) * n]),), s.dtype) for i in range(3)]
        s.U = [v.view(shapes[i * n + j]) for i, p in enumerate(s.packed) for j, v in enumerate(p.split(sizes[i * n:(i + 1) * n]))]
        s.G = []
        idle = case["idle"]
        for i, (r, c) in enumerate(shapes):
            strong = min(32, r, c)
            g = normal((r, c), 8e-3, dtype=f32)
            decay = torch.exp(-0.15 * torch.arange(strong, device="cuda", dtype=f32)) * 0.02
            g.addmm_(normal((r, strong), dtype=f32) * decay, normal((strong, c), dtype=f32))
            if i % n < idle:
                g.zero_()
            s.G.append(g)
        s.coeffs = [ORTHO_COEFFS] * case["steps"]
    return s


# ---------------------------------------------------------------- the plain forms

def _plain_norm(s):
    case = s.case
    h = s.x.float() + s.residual.float() if s.residual is not None else s.x.float()
    gamma = s.gamma.float()
    rstd = torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)
    y = h * rstd * gamma
    out = {"h": h.to(s.dtype)} if s.residual is not None else {}
    if s.y is not None:
        out["y"] = y.to(s.dtype)
    if case["form"] == "q8":
        t, d = y.shape
        wide = -(-d // s.groups) if case["group"] == 0 else case["group"]
        yp = torch.nn.functional.pad(y, (0, s.groups * wide - d)).view(t, s.groups, wide)
        scale = (yp.abs().amax(2) / 448.0).clamp_min(2.0 ** -126)
        out["q"] = (yp / scale[:, :, None]).view(t, s.groups * wide)[:, :d].to(torch.float8_e4m3fn)
        out["scale"] = scale
    if case["form"] == "train":
        hat = h.to(s.dtype).float() * rstd
        dy = s.dY.float()
        g = dy * gamma
        dx = rstd * (g - hat * (g * hat).mean(1, keepdim=True))
        if s.dH is not None:
            dx = dx + s.dH.float()
        out.update(rstd=rstd[:, 0], dX=dx.to(s.dtype), dgamma=(dy * hat).sum(0))
    return out


def _top(x, n):
    """The n largest of every row, by falling value and rising index, and their indices."""
    bits = (x + 0.0).view(torch.int32).long()                     # (+0.0: the two zeros are one value)
    order = torch.where(bits >= 0, bits, -(bits & 0x7fffffff))
    key = (order << 20) + ((1 << 20) - 1 - torch.arange(x.shape[1], device=x.device))
    idx = key.topk(n, dim=1).indices
    return x.gather(1, idx), idx


def _plain_logprobs(s):
    case = s.case
    x = s.logits.float()
    m = x.amax(1, keepdim=True)
    z = x - m
    e = z.exp()
    total = e.sum(1, keepdim=True)
    log_total = total.log()
    has = s.targets >= 0
    at = s.targets.clamp_min(0).long()[:, None]
    logp = torch.where(has, (z.gather(1, at) - log_total)[:, 0], 0.0)
    out = {"logp": logp}
    if case["entropy"]:
        out["entropy"] = log_total[:, 0] - torch.where(e > 0, e * z, 0.0).sum(1) / total[:, 0]
    if case["top"]:
        value, idx = _top(x, case["top"])
        none = value == -math.inf
        out["top_idx"] = torch.where(none, -1, idx).to(torch.int32)
        out["top_logp"] = value - m - log_total
    if case["form"] == "train":
        p = e / total
        w = torch.where(has, s.d_logp, 0.0)[:, None]
        dx = -w * p
        dx.scatter_add_(1, at, w)
        if s.d_entropy is not None:
            dx = dx - s.d_entropy[:, None] * torch.where(p > 0, p * (z - log_total + out["entropy"][:, None]), 0.0)
        out["d_logits"] = dx.to(s.dtype)
    return out


def _plain_ortho(s):
    out = []
    for g in s.G:
        tall = g.shape[0] > g.shape[1]
        x = g.t() if tall else g
        x = x / (torch.linalg.vector_norm(g, dtype=torch.float64).float() + ORTHO_EPS)
        for a, b, c in s.coeffs:
            gram = x @ x.t()
            x = a * x + (b * gram + c * (gram @ gram)) @ x
        out.append((x.t() if tall else x).to(s.dtype).contiguous())
    return _flat(out)


def _flat(matrices):
    """W1 and W3 of all experts, then W2, as the layer keeps them: three outputs, packed."""
    n = len(matrices) // 3
    return [torch.cat([m.reshape(-1) for m in matrices[i * n:(i + 1) * n]]) for i in range(3)]


# ---------------------------------------------------------------- the framework's calls

def _own_norm(s):
    import paper_2409_12210_amd as modse

    case = s.case
    t, d, dt = case["n_tokens"], case["d_model"], case["dtype"]
    out = {"h": s.h} if s.residual is not None else {}
    if s.y is not None:
        out["y"] = s.y
    if case["form"] == "q8":
        modse.modse_norm_fwd(t, d, dt, s.x, s.residual, s.gamma, EPS, s.y, s.h, None, s.q, s.scale, case["group"])
        out.update(q=s.q, scale=s.scale)
        return out
    modse.modse_norm_fwd(t, d, dt, s.x, s.residual, s.gamma, EPS, s.y, s.h, s.rstd)
    if case["form"] == "train":
        if not hasattr(s, "ws"):
            s.ws = torch.empty(modse.modse_norm_bwd_workspace_size(t, d, dt), dtype=torch.uint8, device="cuda")
        h = s.h if s.residual is not None else s.x
        modse.modse_norm_bwd(t, d, dt, h, s.gamma, s.rstd, s.dY, s.dH, s.dX, s.dgamma, False, s.ws)
        out.update(rstd=s.rstd, dX=s.dX, dgamma=s.dgamma)
    return out


def _own_logprobs(s):
    import paper_2409_12210_amd as modse

    case = s.case
    t, v, dt, top = case["n_tokens"], case["vocab"], case["dtype"], case["top"]
    if not hasattr(s, "ws"):
        s.ws = torch.empty(modse.modse_logprobs_workspace_size(t, v, dt, top), dtype=torch.uint8, device="cuda")
    modse.modse_logprobs_fwd(t, v, dt, s.logits, s.targets, s.logp, s.stats, s.entropy, top, s.top_idx, s.top_logp, s.ws)
    out = {"logp": s.logp}
    if case["entropy"]:
        out["entropy"] = s.entropy
    if top:
        out.update(top_idx=s.top_idx, top_logp=s.top_logp)
    if case["form"] == "train":
        modse.modse_logprobs_bwd(t, v, dt, s.logits, s.targets, s.stats, s.entropy, s.d_logp, s.d_entropy, s.d_logits)
        out["d_logits"] = s.d_logits
    return out


def _own_ortho(s):
    import paper_2409_12210_amd as modse

    if not hasattr(s, "set"):
        s.set = modse.MatrixSet(s.G, s.U)
        s.ws = torch.empty(modse.modse_orthogonalize_workspace_size(s.set), dtype=torch.uint8, device="cuda")
    modse.modse_orthogonalize(s.set, s.coeffs, ORTHO_EPS, s.ws)
    return s.packed


def run(s):
    if s.op == "norm":
        return _own_norm(s) if own else _plain_norm(s)
    if s.op == "logprobs":
        return _own_logprobs(s) if own else _plain_logprobs(s)
    return _own_ortho(s) if own else _plain_ortho(s)


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_norm(s):
    case = s.case
    x = s.x.double()
    h = x + s.residual.double() if s.residual is not None else x
    d = h.shape[1]
    inv = 1.0 / ((h * h).sum(1) / d + EPS).sqrt()
    y = h * inv[:, None] * s.gamma.double()
    out = {"h": h} if s.residual is not None else {}
    if s.y is not None:
        out["y"] = y
    if case["form"] == "q8":
        width = case["group"] or d
        parts = y.split(width, 1)
        scales = [p.abs().max(1).values / 448.0 for p in parts]
        # (the nearest e4m3 value: a rounding from 64 bits to 32 in between moves only what lies next to a tie)
        out["q"] = torch.cat([(p / sc[:, None]).float() for p, sc in zip(parts, scales)], 1).to(torch.float8_e4m3fn).double()
        out["scale"] = torch.stack(scales, 1)
    if case["form"] == "train":
        kept = h.to(s.dtype).double()          # the backward pass reads the stream as it is stored
        dy, w = s.dY.double(), s.gamma.double()
        dot = (dy * w * kept).sum(1)
        dx = (dy * w) * inv[:, None] - kept * (dot * inv ** 3 / d)[:, None]
        if s.dH is not None:
            dx += s.dH.double()
        out.update(rstd=inv, dX=dx, dgamma=torch.einsum("td,td,t->d", dy, kept, inv))
    return out


def _exact_logprobs(s):
    case = s.case
    t, v = s.logits.shape
    got = {}
    rows = max(1, (1 << 27) // v)
    for at in range(0, t, rows):
        x, tg = s.logits[at:at + rows].double(), s.targets[at:at + rows].long()
        lse = x.logsumexp(1)
        lp = x - lse[:, None]
        p = lp.exp()
        has = tg >= 0
        logp = torch.where(has, lp[torch.arange(len(tg), device="cuda"), tg.clamp_min(0)], 0.0)
        part = {"logp": logp}
        plogp = torch.nan_to_num(p * lp, nan=0.0, posinf=0.0, neginf=0.0)
        ent = -plogp.sum(1)
        if case["entropy"]:
            part["entropy"] = ent
        if case["top"]:
            # (stable: equal values keep the order of their indices)
            value, idx = torch.sort(lp, dim=1, descending=True, stable=True)
            value, idx = value[:, :case["top"]], idx[:, :case["top"]]
            part["top_idx"], part["top_logp"] = torch.where(value == -math.inf, -1, idx).to(torch.int32), value
        if case["form"] == "train":
            g = torch.where(has, s.d_logp[at:at + rows].double(), 0.0)
            dx = p * -g[:, None]
            dx[torch.arange(len(tg), device="cuda"), tg.clamp_min(0)] += g
            if s.d_entropy is not None:
                dx -= s.d_entropy[at:at + rows].double()[:, None] * (plogp + p * ent[:, None])
            part["d_logits"] = dx
        for k, val in part.items():
            got.setdefault(k, []).append(val)
    return {k: torch.cat(val) for k, val in got.items()}


def _exact_ortho(s):
    out = []
    for g in s.G:
        x = g.double()
        x = x / (x.pow(2).sum().sqrt() + ORTHO_EPS)
        for a, b, c in s.coeffs:
            # the polynomial on the side that is the shorter one: X p(X^T X) = p(X X^T) X
            if x.shape[0] <= x.shape[1]:
                gram = x.mm(x.t().contiguous())
                x = a * x + b * gram.mm(x) + c * gram.mm(gram.mm(x))
            else:
                gram = x.t().contiguous().mm(x)
                x = a * x + b * x.mm(gram) + c * x.mm(gram).mm(gram)
        out.append(x)
    return _flat(out)


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "logprobs": _exact_logprobs, "ortho": _exact_ortho}[s.op](s)
