"""A classifier of KAN layers, trained and asked with the framework's own operators.

    python -m paper_2609_01956_amd.train [--steps N] [--batch B] [--dtype bf16|f32]

Each layer's input is normalised (layer_norm), so that it stays on the layer's grid, and where
two layers have the same width the second reads the sum of the first's input and output (the
norm's residual).  The loss is the mean of the given classes' log probabilities
(token_logprobs) with a small entropy bonus; the gradients of all parameters are clipped by
their global norm (clip_grad_norm) before the update.  The data is synthetic: inputs from a
normal distribution, classes by a random linear map.
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
        grads, dh = [], None
        for (w, _, coef, base_w), (z, h, mean, rstd, res) in zip(reversed(self.params),
                                                                  reversed(kept)):
            dz, dcoef, dbase = kb.layer_backward(z, coef, base_w, d, *self.grid)
            d, dw, db = kb.layer_norm_backward(h, mean, rstd, w, dz, dh=dh)
            grads.append([dw, db, dcoef, dbase])
            dh = d if res else None
        return logp.mean(), [g for layer in reversed(grads) for g in layer]

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


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--batch", type=int, default=4096)
    ap.add_argument("--dtype", choices=["bf16", "f32"], default="bf16")
    args = ap.parse_args()
    dtype = torch.bfloat16 if args.dtype == "bf16" else torch.float32
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
