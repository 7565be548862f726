"""A language model of one MoDSE layer, trained and asked for its next tokens with this library's operators: the norm in front of
the layer and in front of the logits (modse_norm_*), the layer (modse_layer_*), the loss, its gradient and the alternatives of the next
token (modse_logprobs_*), and the orthogonalised update of the expert matrices (modse_orthogonalize).  PyTorch holds the memory, looks up
embeddings and multiplies by the output matrix; with --ends the library looks up embeddings, too (modse_embed_*), and in training multiplies by
the output matrix (modse_head_*), without the logits of a batch (the alternatives still come from logits); with --dropout P, which goes with it, a
share P of the layer's output is dropped in training (modse_dropout_*).

    python examples/tiny_lm.py [--dtype bf16] [--steps 60] [--ends [--dropout 0.1]]

    h1 = E[token]                    y1 = norm(h1; gamma1)
    h2 = h1 + layer(y1)              y2 = norm(h2; gamma2)         (the addition is the norm's, or the dropout's)
    logits = y2 Wout^T               loss = - mean log p(next token)

The text is made up: token t is followed by (5 t + 3) mod vocab three times out of four, and by any token else."""
import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

import paper_2409_12210_amd as modse  # noqa: E402

EPS = 1e-6
COEFFS = [(3.4445, -4.7750, 2.0315)] * 5


class TinyLM:
    ends, p = False, 0.0

    def __init__(self, vocab=512, d_model=256, d_ff=(128, 384, 192, 320, 224, 288, 256, 256), top_k=2, dtype="bf16", batch=512, seed=0,
                 ends=False, dropout=0.0):
        if dropout and not ends:
            raise ValueError("dropout goes with ends")
        self.ends, self.p = ends, dropout
        self.V, self.d, self.d_ff, self.k, self.dtype, self.T = vocab, d_model, list(d_ff), top_k, dtype, batch
        self.t = torch.bfloat16 if dtype == "bf16" else torch.float32
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def weights(*shape, sigma=0.05):
            return torch.empty(shape, dtype=self.t, device="cuda").normal_(0.0, sigma, generator=gen)
        d, V, F, N = d_model, vocab, sum(d_ff), len(d_ff)
        self.E, self.Wout = weights(V, d, sigma=1.0), weights(V, d)
        self.gamma1, self.gamma2 = (torch.ones(d, dtype=self.t, device="cuda") for _ in range(2))
        self.W_gate, self.W1, self.W3, self.W2 = weights(d, N), weights(F, d), weights(F, d), weights(d * F)
        # what a step writes: allocated once
        rows, f32 = lambda *s: torch.empty(s, dtype=self.t, device="cuda"), lambda *s: torch.empty(s, device="cuda")  # noqa: E731
        self.y1, self.moe, self.h2, self.y2, self.g, self.dy1, self.dh1, self.dh2 = (rows(batch, d) for _ in range(8))
        self.rstd1, self.rstd2, self.logp, self.stats = f32(batch), f32(batch), f32(batch), f32(batch, 2)
        self.dgamma1, self.dgamma2, self.dW_gate, self.dW1, self.dW3, self.dW2 = f32(d), f32(d), f32(d, N), f32(F, d), f32(F, d), f32(d * F)
        self.routing = modse.Routing.empty(batch, N, top_k)
        layer = (d, self.d_ff, top_k, dtype)
        size = max(modse.modse_workspace_size(*layer, batch, w) for w in (modse.WS_FWD, modse.WS_FWD_SAVED, modse.WS_BWD))
        size = max(size, modse.modse_norm_bwd_workspace_size(batch, d, dtype), modse.modse_logprobs_workspace_size(batch, V, dtype, 8))
        # the expert matrices' gradients, and what becomes of them
        self.updates = [torch.empty_like(w) for w in (self.dW1, self.dW3, self.dW2)]
        G, U = self._matrices(self.dW1, self.dW3, self.dW2), self._matrices(*self.updates)
        self.experts = modse.MatrixSet(G, U)
        size = max(size, modse.modse_orthogonalize_workspace_size(self.experts))
        if ends:
            size = max(size, modse.modse_embed_bwd_workspace_size(batch, d, V, dtype), modse.modse_head_workspace_size(batch, d, V, dtype, modse.WS_BWD))
            self.h1, self.dmoe = rows(batch, d), rows(batch, d)
            self.dE, self.dWout = f32(V, d), f32(V, d)
            self.rng = torch.tensor([seed, 0], dtype=torch.int64, device="cuda")       # the second one counts steps
        self.ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        self.saved = torch.empty(modse.modse_saved_size(*layer, batch), dtype=torch.uint8, device="cuda")

    def _matrices(self, W1, W3, W2):
        flat = [w.view(f, self.d) for W in (W1, W3) for w, f in zip(W.view(-1).split([f * self.d for f in self.d_ff]), self.d_ff)]
        return flat + [w.view(self.d, f) for w, f in zip(W2.split([f * self.d for f in self.d_ff]), self.d_ff)]

    def forward(self, tokens, train=False):
        """Logits of the token after each of `tokens`, a batch of them at the most."""
        self.hidden(tokens, train)
        return self.y2[:len(tokens)] @ self.Wout.t()

    def hidden(self, tokens, train=False):
        """The rows y2 that the logits are made from."""
        T, d, dt = len(tokens), self.d, self.dtype
        if T > self.T or (train and T != self.T):
            raise ValueError(f"{T} tokens where the buffers hold {self.T}")
        if self.ends:
            h1 = self.h1[:T]
            modse.modse_embed_fwd(T, d, self.V, dt, tokens.int(), self.E, 1.0, h1)
        else:
            h1 = self.E[tokens]
        modse.modse_norm_fwd(T, d, dt, h1, None, self.gamma1, EPS, self.y1, None, self.rstd1 if train else None)
        modse.modse_layer_fwd(d, self.d_ff, self.k, dt, T, self.y1, self.W_gate, None, self.W1, self.W3, self.W2, self.moe,
                              self.routing, self.saved if train else None, self.ws)
        if self.p and train:
            modse.modse_dropout_fwd(T, d, dt, self.moe, h1, self.p, self.rng, 0, self.h2)
            modse.modse_norm_fwd(T, d, dt, self.h2, None, self.gamma2, EPS, self.y2, None, self.rstd2)
        else:
            modse.modse_norm_fwd(T, d, dt, self.moe, h1, self.gamma2, EPS, self.y2, self.h2, self.rstd2 if train else None)
        if not self.ends:
            self.h1 = h1

    def loss_and_gradients(self, tokens, targets):
        """Mean negative log probability of `targets` (int32; negative: none), and the gradients of all weights."""
        T, d, dt = self.T, self.d, self.dtype
        if len(targets) != T:
            raise ValueError(f"{len(targets)} targets of {T} tokens")
        count = (targets >= 0).sum().clamp_min(1)
        d_logp = (-1.0 / count).expand(T).float().contiguous()
        if self.ends:
            self.hidden(tokens, train=True)
            modse.modse_head_bwd(T, d, self.V, dt, self.y2, self.Wout, targets, d_logp, self.logp, self.g, self.dWout, False, self.ws)
        else:
            logits = self.forward(tokens, train=True)
            modse.modse_logprobs_fwd(T, self.V, dt, logits, targets, self.logp, self.stats, None, 0, None, None, self.ws)
            # the gradient of the logits takes their place
            modse.modse_logprobs_bwd(T, self.V, dt, logits, targets, self.stats, None, d_logp, None, logits)
            self.dWout = logits.t() @ self.y2
            torch.mm(logits, self.Wout, out=self.g)
        modse.modse_norm_bwd(T, d, dt, self.h2, self.gamma2, self.rstd2, self.g, None, self.dh2, self.dgamma2, False, self.ws)
        dmoe = self.dh2
        if self.p:
            dmoe = self.dmoe
            modse.modse_dropout_bwd(T, d, dt, self.dh2, self.p, self.rng, 0, dmoe)
        modse.modse_layer_bwd(d, self.d_ff, self.k, dt, T, self.y1, self.W_gate, self.W1, self.W3, self.W2, self.routing, self.saved,
                              dmoe, self.dy1, self.dW_gate, self.dW1, self.dW3, self.dW2, False, self.ws)
        # the stream's gradient: through the norm, and past it
        modse.modse_norm_bwd(T, d, dt, self.h1, self.gamma1, self.rstd1, self.dy1, self.dh2, self.dh1, self.dgamma1, False, self.ws)
        if self.ends:
            modse.modse_embed_bwd(T, d, self.V, dt, tokens.int(), self.dh1, 1.0, self.dE, False, self.ws)
        else:
            self.dE = torch.zeros((self.V, d), device="cuda").index_add_(0, tokens, self.dh1.float())
        return -self.logp.sum() / count

    def step(self, tokens, targets, lr=0.02):
        loss = self.loss_and_gradients(tokens, targets)
        modse.modse_orthogonalize(self.experts, COEFFS, 1e-7, self.ws)
        for w, u in zip((self.W1, self.W3, self.W2), self.updates):
            w -= (lr * u).to(self.t)                               # rows of unit length: the step's size is lr's alone
        for w, g, rate in ((self.E, self.dE, 20.0), (self.Wout, self.dWout, 2.0), (self.W_gate, self.dW_gate, 0.5),
                           (self.gamma1, self.dgamma1, 0.05), (self.gamma2, self.dgamma2, 0.05)):
            w -= (rate * g.float()).to(self.t)
        if self.ends:
            self.rng[1] += 1                                       # another mask for the next step
        return loss

    def alternatives(self, tokens, n=5):
        """The n most probable next tokens of each, with their log probabilities and the entropy."""
        T = len(tokens)
        logits = self.forward(tokens)
        idx, logp = torch.empty((T, n), dtype=torch.int32, device="cuda"), torch.empty((T, n), device="cuda")
        entropy = torch.empty(T, device="cuda")
        modse.modse_logprobs_fwd(T, self.V, self.dtype, logits, None, None, None, entropy, n, idx, logp, self.ws)
        return idx, logp, entropy


def text(n, vocab, gen):
    tokens = torch.randint(0, vocab, (n,), generator=gen, device="cuda")
    after = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.75, (5 * tokens + 3) % vocab,
                        torch.randint(0, vocab, (n,), generator=gen, device="cuda")).int()
    return tokens, after


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--ends", action="store_true", help="lookup of embeddings, and in training output matrix and loss, by the library, too")
    p.add_argument("--dropout", type=float, default=0.0, help="share of the layer's output that is dropped in training (with --ends)")
    a = p.parse_args()
    model, gen = TinyLM(dtype=a.dtype, ends=a.ends, dropout=a.dropout), torch.Generator(device="cuda").manual_seed(1)
    for i in range(a.steps):
        loss = model.step(*text(model.T, model.V, gen))
        if i % 10 == 0 or i == a.steps - 1:
            print("step %3d  loss %.3f" % (i, float(loss)), flush=True)
    idx, logp, entropy = model.alternatives(torch.arange(4, device="cuda"), 3)
    for t in range(4):
        print("after %d (%d in the text): %s, entropy %.2f" % (
            t, (5 * t + 3) % model.V, ", ".join("%d %.2f" % (j, p) for j, p in zip(idx[t].tolist(), logp[t].exp().tolist())), float(entropy[t])))


if __name__ == "__main__":
    main()
