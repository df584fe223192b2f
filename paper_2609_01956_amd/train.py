"""A classifier of KAN layers and a model of the next token, trained and asked with the framework's
own operators.

    python -m paper_2609_01956_amd.train [--model classes|tokens] [--steps N] [--batch B]
                                         [--dtype bf16|f32]

Each layer's input is normalised (layer_norm), so that it stays on the layer's grid, and where
two layers have the same width the second reads the sum of the first's input and output (the
norm's residual).  The loss is the mean of the given classes' log probabilities
(token_logprobs) with a small entropy bonus; the gradients of all parameters are clipped by
their global norm (clip_grad_norm) before the update.  The data is synthetic: inputs from a
normal distribution, classes by a random linear map.

The token model reads a window of tokens through an embedding (embedding) and asks for the next one
under the same table as a linear head (linear_logprobs), without logits in memory; the table's
gradient as the head's weights is what the embedding's is added to (embedding_backward).  Its data:
each token follows from the two before it.
"""
from __future__ import annotations

import argparse
from typing import Sequence

import torch

from . import binding as kb

# Normalised inputs have unit variance: the grid reaches three standard deviations.
GRID_LO, GRID_HI = -3.0, 3.0


class KanClassifier:
    """Parameters per layer: the norm's weight and bias (fp32), coef and base_w (dtype)."""

    def __init__(self, sizes: Sequence[int], grid_size: int = 10, dtype=torch.bfloat16,
                 device="cuda", seed: int = 42):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.grid = (int(grid_size), GRID_LO, GRID_HI)
        self.params = []
        for n_in, n_out in zip(sizes, sizes[1:]):
            draw = lambda *s: torch.randn(*s, device=device, generator=g)
            self.params.append([torch.ones(n_in, device=device), torch.zeros(n_in, device=device),
                                (draw(n_out, n_in, grid_size + 3) * n_in ** -0.5).to(dtype),
                                (draw(n_out, n_in) * n_in ** -0.5).to(dtype)])

    def forward(self, x, need_stats: bool = True):
        """Logits, and per layer what its backward needs: (z, h, mean, rstd, residual used)."""
        kept, stream, out = [], None, x
        for w, b, coef, base_w in self.params:
            res = stream if stream is not None and stream.shape == out.shape else None
            z, stream, mean, rstd = kb.layer_norm(out, w, b, residual=res, need_stats=need_stats)
            out = kb.layer_forward(z, coef, base_w, *self.grid)
            kept.append((z, stream, mean, rstd, res is not None))
        return out, kept

    def gradients(self, x, targets, entropy_bonus: float = 0.0):
        """Mean log probability of the targets, and the gradients of its negative (less the
        bonus times the mean entropy) with respect to the parameters, in their order."""
        logits, kept = self.forward(x)
        rows = x.shape[0]
        logp, stats, ent, _, _ = kb.token_logprobs(logits, targets, entropy=entropy_bonus != 0)
        dlogp = torch.full_like(logp, -1.0 / rows)
        dent = None if ent is None else torch.full_like(ent, -entropy_bonus / rows)
        d = kb.token_logprobs_backward(logits, targets, stats, dlogp, entropy=ent, dentropy=dent)
        return logp.mean(), self.backward(kept, d)[0]

    def backward(self, kept, d):
        """For the gradient d of the logits: those of the parameters, in their order, and of x."""
        grads, dh = [], None
        for (w, _, coef, base_w), (z, h, mean, rstd, res) in zip(reversed(self.params),
                                                                  reversed(kept)):
            dz, dcoef, dbase = kb.layer_backward(z, coef, base_w, d, *self.grid)
            d, dw, db = kb.layer_norm_backward(h, mean, rstd, w, dz, dh=dh)
            grads.append([dw, db, dcoef, dbase])
            dh = d if res else None
        return [g for layer in reversed(grads) for g in layer], d

    def step(self, x, targets, lr: float = 0.5, max_norm: float = 1.0,
             entropy_bonus: float = 0.0):
        """One update; the mean log probability and the gradients' norm, on the device."""
        logp, grads = self.gradients(x, targets, entropy_bonus)
        norm = kb.clip_grad_norm(grads, max_norm)
        for p, g in zip([p for layer in self.params for p in layer], grads):
            p.add_(g, alpha=-lr)
        return logp, norm

    def alternatives(self, x, targets, top_k: int = 3):
        """Serving form: the targets' log probabilities and the top_k classes with theirs."""
        logits, _ = self.forward(x, need_stats=False)
        logp, _, _, top_logp, top_index = kb.token_logprobs(logits, targets, top_k=top_k)
        return logp, top_logp, top_index


class KanTokenModel:
    """The next token after a window of `context`: their rows of a table [classes, width], side by
    side, through KAN layers to `width` values, whose products with the table's rows are the
    logits.  Tokens and targets of `ignore_index` are padding."""

    def __init__(self, classes: int, width: int, context: int = 2, hidden: Sequence[int] = (),
                 grid_size: int = 10, dtype=torch.bfloat16, device="cuda", seed: int = 42,
                 ignore_index: int = -100):
        g = torch.Generator(device=device)
        g.manual_seed(seed + 1)
        self.table = (torch.randn(classes, width, device=device, generator=g) *
                      width ** -0.5).to(dtype)
        self.scale = width ** 0.5  # (embedded tokens have unit variance)
        self.ignore_index = int(ignore_index)
        self.body = KanClassifier((context * width, *hidden, width), grid_size, dtype, device, seed)

    def parameters(self):
        return [self.table] + [p for layer in self.body.params for p in layer]

    def forward(self, tokens, need_stats: bool = True):
        """tokens [rows, context] -> what the head reads [rows, width], and what the backward needs."""
        x = kb.embedding(tokens, self.table, scale=self.scale, ignore_index=self.ignore_index)
        return self.body.forward(x.view(tokens.shape[0], -1), need_stats)

    def gradients(self, tokens, targets):
        """Mean log probability of the targets that are no padding, and the gradients of its negative
        with respect to parameters(), in their order."""
        h, kept = self.forward(tokens)
        logp, stats, _ = kb.linear_logprobs(h, self.table, targets, ignore_index=self.ignore_index)
        share = (targets != self.ignore_index).float()
        share /= share.sum().clamp(min=1.0)
        dh, dtable = kb.linear_logprobs_backward(h, self.table, targets, stats, -share,
                                                 ignore_index=self.ignore_index)
        grads, dx = self.body.backward(kept, dh)
        kb.embedding_backward(tokens, dx.view(*tokens.shape, -1), self.table.shape[0],
                              scale=self.scale, ignore_index=self.ignore_index, base=dtable,
                              out=dtable)
        return (logp * share).sum(), [dtable] + grads

    def step(self, tokens, targets, lr: float = 0.5, max_norm: float = 1.0):
        """One update; the mean log probability and the gradients' norm, on the device."""
        logp, grads = self.gradients(tokens, targets)
        norm = kb.clip_grad_norm(grads, max_norm)
        for p, g in zip(self.parameters(), grads):
            p.add_(g, alpha=-lr)
        return logp, norm

    def next_tokens(self, tokens):
        """Serving form: the most probable next token of each window, and its log probability."""
        h, _ = self.forward(tokens, need_stats=False)
        none = torch.full((tokens.shape[0],), self.ignore_index, device=tokens.device)
        _, stats, best = kb.linear_logprobs(h, self.table, none, best=True,
                                            ignore_index=self.ignore_index)
        return best, -stats[:, 1]


def train_tokens(steps: int, batch: int, dtype, classes: int = 1000) -> None:
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    model = KanTokenModel(classes, 64, hidden=(64,), dtype=dtype)
    for i in range(steps):
        tokens = torch.randint(0, classes, (batch, 2), device="cuda", generator=g)
        targets = (tokens[:, 0] // 8 * 8 + tokens[:, 1] % 8).clamp(max=classes - 1)
        logp, norm = model.step(tokens, targets)
        if i % 10 == 0 or i == steps - 1:
            print(f"step {i}: mean log probability {float(logp):.4f}, gradient norm "
                  f"{float(norm):.4f}", flush=True)
    best, lp = model.next_tokens(tokens[:1])
    print(f"after {tokens[0].tolist()}: {int(best[0])} at {float(lp[0]):.4f} (target "
          f"{int(targets[0])})")


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--model", choices=["classes", "tokens"], default="classes")
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--batch", type=int, default=4096)
    ap.add_argument("--dtype", choices=["bf16", "f32"], default="bf16")
    args = ap.parse_args()
    dtype = torch.bfloat16 if args.dtype == "bf16" else torch.float32
    if args.model == "tokens":
        train_tokens(args.steps, args.batch, dtype)
        return
    sizes = (784, 256, 256, 10)
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    teacher = torch.randn(sizes[0], sizes[-1], device="cuda", generator=g)
    model = KanClassifier(sizes, dtype=dtype)
    for i in range(args.steps):
        x = torch.randn(args.batch, sizes[0], device="cuda", generator=g)
        targets = (x @ teacher).argmax(1)
        logp, norm = model.step(x.to(dtype), targets)
        if i % 10 == 0 or i == args.steps - 1:
            print(f"step {i}: mean log probability {float(logp):.4f}, gradient norm "
                  f"{float(norm):.4f}", flush=True)
    logp, top_logp, top_index = model.alternatives(x[:1].to(dtype), targets[:1])
    print(f"class {int(targets[0])}: log probability {float(logp[0]):.4f}; best classes "
          f"{top_index[0].tolist()} at {[round(v, 4) for v in top_logp[0].tolist()]}")


if __name__ == "__main__":
    main()
