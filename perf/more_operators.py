"""Performance cases of the operators at the two ends of a token model: the embedding of tokens
with scaling and its gradient, and the log probabilities of given tokens under a linear head over
a long vocabulary, without its logits in memory, and their gradient.

    listed()            the fixed cases
    draw(rng)           one more case of the same ranges
    prepare(case, seed) what a program has in hand before the call, from the seed alone
    run(state)          one pass through an operator: the framework's where `own`, else the
                        plain form in 32 bits
    work(case)          bytes and operations the pass cannot do without
    exact(case, seed)   the same outputs from the definitions in 64 bits

A case names its kind: "embed" and "embed_grad" (rows tokens of a table of classes x n), "head"
and "head_grad" (rows x n against classes x n).
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
IGNORE = -100


def listed():
    return [
        # One decoded token on its way into the model: latency.
        embed("embed_serve_1x256_f32", "embed", "f32", "f32", 1, 256, 50001),
        # A training batch of contexts, the table in the model's own type.
        embed("embed_65536x1024_bf16", "embed", "bf16", "bf16", 65536, 1024, 50001),
        # The gradient of a hidden layer's width in full precision: the common tokens fill a large
        # part of the batch.
        embed("embed_grad_65536x256_f32", "embed_grad", "f32", "f32", 65536, 256, 50001),
        # Sizes that are multiples of nothing; added to the gradient that the same table has as the
        # head's weights, in 32 bits; padding in the batch.
        embed("embed_grad_30001x1001_tied_bf16", "embed_grad", "bf16", "f32", 30001, 1001, 50001,
              base=True, ignored=True),
        # The largest table.
        embed("embed_grad_65536x4096_bf16", "embed_grad", "bf16", "bf16", 65536, 4096, 131072),
        # One decoded token: the next one's probability and the most probable one; one pass over
        # the head's weights.
        head("head_serve_1x1024_131072_bf16", "head", "bf16", 1, 1024, 131072, best=True),
        # A few sequences decoded together, in full precision.
        head("head_serve_13x256_50001_f32", "head", "f32", 13, 256, 50001, best=True),
        # Scoring a ragged batch: odd sizes throughout, rows of a wider tensor.
        head("head_2001x1001_50001_bf16", "head", "bf16", 2001, 1001, 50001, pad=15),
        # The loss of a training batch.
        head("head_8192x2048_131072_bf16", "head", "bf16", 8192, 2048, 131072, ignored=True),
        # Gradients of a small vocabulary on a hidden width of 256 in full precision.
        head("head_grad_8192x256_10007_f32", "head_grad", "f32", 8192, 256, 10007),
        # Odd sizes, some targets ignored.
        head("head_grad_2001x1001_50001_bf16", "head_grad", "bf16", 2001, 1001, 50001, pad=15,
             ignored=True),
        # The gradients of a training batch over a long vocabulary.
        head("head_grad_8192x2048_131072_bf16", "head_grad", "bf16", 8192, 2048, 131072,
             ignored=True),
    ]


def embed(name, kind, dtype, params, rows, n, classes, base=False, ignored=False):
    return dict(name=name, kind=kind, dtype=dtype, params=params, rows=rows, n=n, classes=classes,
                scale=n ** 0.5, base=base, ignored=ignored)


def head(name, kind, dtype, rows, n, classes, pad=0, best=False, ignored=False):
    return dict(name=name, kind=kind, dtype=dtype, params=dtype, rows=rows, n=n, classes=classes,
                scale=n ** -0.5, pad=pad, best=best, ignored=ignored)


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """1 to 65536 embedded tokens, 1 to 8192 rows of a head; widths 8 to 4096; 2 to 131072
    classes; at most the work of the largest listed case of the kind."""
    most = {}
    for c in listed():
        w = work(c)
        for k in w:
            most[c["kind"], k] = max(most.get((c["kind"], k), 0), w[k])
    while True:
        kind = rng.choice(["embed", "embed_grad", "head", "head_grad"])
        dtype = rng.choice(["f32", "bf16"])
        n, classes = _log(rng, 8, 4096), _log(rng, 2, 131072)
        ignored = rng.random() < 0.3
        if kind in ("embed", "embed_grad"):
            c = embed("", kind, dtype, rng.choice(["f32", dtype]), _log(rng, 1, 65536), n, classes,
                      base=kind == "embed_grad" and rng.random() < 0.4, ignored=ignored)
        else:
            rows = _log(rng, 1, 8192)
            c = head("", kind, dtype, rows, n, classes, pad=rng.choice([0, 0, 1, 8, 15]),
                     best=kind == "head" and rows <= 64 and rng.random() < 0.5, ignored=ignored)
        del c["name"]
        w = work(c)
        # (32-bit products: within the operations of an eighth of the largest 16-bit ones)
        share = 8 if dtype == "f32" else 1
        if w["bytes"] <= most[kind, "bytes"] and w["flops"] * share <= most[kind, "flops"]:
            return c


def work(case):
    """Each input read once, each output written once; the operations of the formulas.  The
    head's gradient cannot do without its logits, which nobody kept: three products."""
    kind, rows, n, V = case["kind"], case["rows"], case["n"], case["classes"]
    e, p = (4 if case[k] == "f32" else 2 for k in ("dtype", "params"))
    if kind == "embed":
        return {"bytes": rows * (n * e + 8) + min(rows, V) * n * p, "flops": rows * n}
    if kind == "embed_grad":
        return {"bytes": rows * (n * e + 8) + V * n * p * (2 if case["base"] else 1),
                "flops": 2 * rows * n}
    if kind == "head":
        return {"bytes": (rows + V) * n * e + rows * (8 + 12 + (8 if case["best"] else 0)),
                "flops": 2 * rows * V * n + 4 * rows * V}
    return {"bytes": (2 * rows + V) * n * e + V * n * p + rows * 20,
            "flops": 6 * rows * V * n + 4 * rows * V}


# ---------------------------------------------------------------- inputs

def prepare(case, seed):
    dev, dt, pt = torch.device("cuda"), DTYPES[case["dtype"]], DTYPES[case["params"]]
    kind, rows, n, V = case["kind"], case["rows"], case["n"], case["classes"]
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)

    def randn(*shape, std=1.0, dtype=dt):
        return torch.randn(*shape, device=dev, generator=gen).mul_(std).to(dtype)

    # tokens as a text has them: the r-th most common one about 1 / r as often as the first, and
    # the common ones anywhere in the table
    u = torch.rand(rows, device=dev, generator=gen, dtype=torch.float64)
    rank = (u * math.log(V + 1)).exp().long().clamp(1, V) - 1
    tokens = torch.randperm(V, device=dev, generator=gen)[rank]
    if case["ignored"]:
        drop = torch.rand(rows, device=dev, generator=gen) < 0.1
        tokens = torch.where(drop, IGNORE, tokens)
    state = dict(case=case, tokens=tokens)
    if kind == "embed":
        state["table"] = randn(V, n, std=n ** -0.5, dtype=pt)
    elif kind == "embed_grad":
        state["dy"] = randn(rows, n, std=0.02)
        if case["base"]:
            state["base"] = randn(V, n, std=0.02, dtype=pt)
            state["out"] = torch.empty_like(state["base"])
    else:
        # normalised hidden states, which lie towards their targets' weights as after training
        state["weight"] = w = randn(V, n, std=2.0)
        x = torch.randn(rows, n + case["pad"], device=dev, generator=gen)
        x[:, :n] += w[tokens.clamp(min=0)].float() * (1.5 * n ** -0.5)
        state["x"] = x.to(dt)[:, :n]
        if kind == "head_grad":
            z = (state["x"].float() @ w.float().t()).mul_(case["scale"])
            m = z.amax(1)
            state["stats"] = torch.stack([m, z.sub_(m[:, None]).exp_().sum(1).log()], 1)
            state["dlogp"] = -torch.rand(rows, device=dev, generator=gen)
    return state


# ---------------------------------------------------------------- one pass

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(state):
    from paper_2609_01956_amd import binding as kb
    case, kind, tokens = state["case"], state["case"]["kind"], state["tokens"]
    if kind == "embed":
        return kb.embedding(tokens, state["table"], scale=case["scale"], ignore_index=IGNORE,
                            dtype=DTYPES[case["dtype"]])
    if kind == "embed_grad":
        return kb.embedding_backward(tokens, state["dy"], case["classes"], scale=case["scale"],
                                     ignore_index=IGNORE, dtype=DTYPES[case["params"]],
                                     base=state.get("base"), out=state.get("out"))
    if kind == "head":
        logp, stats, best = kb.linear_logprobs(state["x"], state["weight"], tokens,
                                               scale=case["scale"], best=case["best"],
                                               ignore_index=IGNORE)
        return [logp, stats] + ([best] if case["best"] else [])
    return kb.linear_logprobs_backward(state["x"], state["weight"], tokens, state["stats"],
                                       state["dlogp"], scale=case["scale"], ignore_index=IGNORE)


def _run_plain(state):
    case, kind, tokens = state["case"], state["case"]["kind"], state["tokens"]
    dt, pt, scale = DTYPES[case["dtype"]], DTYPES[case["params"]], case["scale"]
    valid = tokens != IGNORE
    index = torch.where(valid, tokens, 0)
    if kind == "embed":
        rows = state["table"][index].float() * scale
        return torch.where(valid[:, None], rows, 0.0).to(dt)
    if kind == "embed_grad":
        dy = torch.where(valid[:, None], state["dy"].float() * scale, 0.0)
        base = state.get("base")
        if base is None:
            total = torch.zeros(case["classes"], case["n"], device=dy.device)
        else:
            total = base.float().clone()
        return total.index_add_(0, index, dy).to(pt)
    x, w = state["x"].float(), state["weight"].float()
    z = (x @ w.t()) * scale
    if kind == "head":
        m = z.amax(1)
        z = z - m[:, None]
        logs = z.exp().sum(1).log()
        logp = torch.where(valid, z.gather(1, index[:, None])[:, 0] - logs, 0.0)
        if not case["best"]:
            return [logp, torch.stack([m, logs], 1)]
        # (argmax gives the first of equal values)
        return [logp, torch.stack([m, logs], 1), z.argmax(1)]
    d = torch.where(valid, state["dlogp"], 0.0)
    stats = state["stats"]
    dz = (z - stats[:, :1] - stats[:, 1:]).exp() * -d[:, None]
    dz[torch.arange(dz.shape[0], device=dz.device), index] += d
    return ((dz @ w) * scale).to(dt), ((dz.t() @ x) * scale).to(pt)


# ---------------------------------------------------------------- 64 bits

def exact(case, seed):
    state, kind = prepare(case, seed), case["kind"]
    tokens, scale, V, n = state["tokens"], case["scale"], case["classes"], case["n"]
    keep = (tokens != IGNORE).nonzero()[:, 0]
    if kind == "embed":
        y = torch.zeros(case["rows"], n, dtype=torch.float64, device=tokens.device)
        y[keep] = state["table"].index_select(0, tokens[keep]).double() * scale
        return y
    if kind == "embed_grad":
        g = torch.zeros(V, n, dtype=torch.float64, device=tokens.device)
        g.index_add_(0, tokens[keep], state["dy"][keep].double(), alpha=scale)
        if case["base"]:
            g += state["base"]
        return g
    w = state["weight"].double()
    step = max(1, (1 << 28) // V)
    if kind == "head":
        parts = []
        for i in range(0, case["rows"], step):
            z = torch.mm(state["x"][i:i + step].double() * scale, w.t())
            t = tokens[i:i + step]
            lse, (m, best) = torch.logsumexp(z, 1), z.max(1)
            lp = (z.gather(1, t.clamp(min=0).unsqueeze(1)).squeeze(1) - lse).masked_fill(
                t == IGNORE, 0.0)
            # (the lowest of equal ones)
            first = torch.where(z == m.unsqueeze(1), torch.arange(V, device=z.device), V).amin(1) \
                if case["best"] else best
            parts.append([lp, torch.stack([m, lse - m], 1)] + ([first] if case["best"] else []))
        return [torch.cat(p) for p in zip(*parts)]
    dxs, dw = [], torch.zeros_like(w)
    for i in range(0, case["rows"], step):
        x, t = state["x"][i:i + step].double(), tokens[i:i + step]
        lse = state["stats"][i:i + step].double().sum(1, keepdim=True)
        d = state["dlogp"][i:i + step].double().masked_fill(t == IGNORE, 0.0).unsqueeze(1)
        g = torch.mm(x * scale, w.t()).sub_(lse).exp_().mul_(-d)
        g.scatter_add_(1, t.clamp(min=0).unsqueeze(1), d)
        g.mul_(scale)
        dxs.append(torch.mm(g, w))
        dw.addmm_(g.t(), x)
    return torch.cat(dxs), dw
