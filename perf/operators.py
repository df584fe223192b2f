"""Performance cases of the operators around a KAN layer in a training or serving step: layer
norm (with the residual sum before it) and its gradient, log probabilities of given classes
(tokens) with entropy and top alternatives and their gradient, and the clipping of gradients by
their global norm.

    listed()            the fixed cases
    draw(rng)           one more case of the same ranges
    prepare(case, seed) what a program has in hand before the call, from the seed alone
    run(state)          one pass through an operator: the framework's where `own`, else the
                        plain form in 32 bits
    work(case)          bytes and operations the pass cannot do without
    exact(case, seed)   the same outputs from the definitions in 64 bits

A case names its kind: "norm" and "norm_grad" (rows x n), "logprob" and "logprob_grad" (rows x
classes), "clip" (the gradients of a stack of KAN layers with their norms).
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
IGNORE = -100


def listed():
    return [
        # One served row of a hidden width, residual added, no statistics kept: latency.
        norm("norm_serve_1x256_f32", "norm", "f32", "f32", 1, 256, residual=True, stats=False),
        # The input normalisation of the 784-256-256-10 network at its training batch.
        norm("norm_train_65536x784_bf16", "norm", "bf16", "bf16", 65536, 784),
        # A hidden layer's gradient in full precision.
        norm("norm_grad_16384x256_f32", "norm_grad", "f32", "f32", 16384, 256),
        # Sizes that are multiples of nothing, master weights in 32 bits, and the gradient that
        # comes round the block on the residual stream.
        norm("norm_grad_30001x1001_bf16", "norm_grad", "bf16", "f32", 30001, 1001, residual=True),
        # Wide rows, many of them: the largest gradient.
        norm("norm_grad_16384x8192_bf16", "norm_grad", "bf16", "f32", 16384, 8192, residual=True),
        # The classifier's loss: ten classes, entropy for the regulariser.
        logprob("logprob_65536x10_f32", "logprob", "f32", 65536, 10, entropy=True),
        # One decoded token over a long vocabulary, half of it masked by a constraint, with the
        # alternatives that a serving API reports.
        logprob("logprob_serve_1x131072_bf16", "logprob", "bf16", 1, 131072, top_k=20,
                entropy=True, masked=True),
        # Scoring a ragged batch: an odd vocabulary in padded rows.
        logprob("logprob_2001x50001_bf16", "logprob", "bf16", 2001, 50001, pad=15, top_k=5,
                entropy=True),
        # The gradient of the loss over a long vocabulary, some targets ignored, with the
        # entropy's gradient.
        logprob("logprob_grad_4096x131072_bf16", "logprob_grad", "bf16", 4096, 131072,
                entropy=True, ignored=True),
        # The gradients of the 784-256-256-10 network: few tensors, clipped.
        clip("clip_mlp_784_256_256_10_g10_f32", "f32", "784,256,256,10", 10, clipped=True),
        # A deep stack of narrow layers: hundreds of small tensors, the norm within bounds (the
        # usual step), in place.
        clip("clip_64x_37_g5_f32", "f32", ",".join(["37"] * 65), 5, clipped=False),
        # A large stack, clipped.
        clip("clip_16x_1024_g10_bf16", "bf16", ",".join(["1024"] * 17), 10, clipped=True),
    ]


def norm(name, kind, dtype, params, rows, n, residual=False, stats=True):
    return dict(name=name, kind=kind, dtype=dtype, params=params, rows=rows, n=n,
                residual=residual, stats=stats)


def logprob(name, kind, dtype, rows, classes, pad=0, top_k=0, entropy=False, masked=False,
            ignored=False):
    return dict(name=name, kind=kind, dtype=dtype, rows=rows, classes=classes, pad=pad,
                top_k=top_k, entropy=entropy, masked=masked, ignored=ignored)


def clip(name, dtype, sizes, G, clipped):
    return dict(name=name, kind="clip", dtype=dtype, sizes=sizes, G=G, clipped=clipped)


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Rows 1 to 65536; normalised widths 8 to 16384; 2 to 131072 classes, 0 to 20 alternatives;
    stacks of 1 to 64 layers of width 8 to 1024 on grids 3 to 20; at most the work of the largest
    listed case of the kind."""
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0), work(c)["bytes"])
    most["norm"], most["logprob"] = most["norm_grad"], most["logprob_grad"]
    while True:
        kind = rng.choice(["norm", "norm_grad", "logprob", "logprob_grad", "clip"])
        dtype = rng.choice(["f32", "bf16"])
        if kind in ("norm", "norm_grad"):
            c = norm("", kind, dtype, rng.choice(["f32", dtype]), _log(rng, 1, 65536),
                     _log(rng, 8, 16384), residual=rng.random() < 0.5,
                     stats=kind == "norm_grad" or rng.random() < 0.75)
        elif kind in ("logprob", "logprob_grad"):
            V = _log(rng, 2, 131072)
            k = min(V, rng.choice([0, 0, 1, 5, 20])) if kind == "logprob" else 0
            c = logprob("", kind, dtype, _log(rng, 1, 65536), V, pad=rng.choice([0, 0, 1, 8, 15]),
                        top_k=k, entropy=rng.random() < 0.5,
                        masked=V >= 1000 and rng.random() < 0.3, ignored=rng.random() < 0.3)
        else:
            width, G = _log(rng, 8, 1024), _log(rng, 3, 20)
            widths = [str(max(2, width - rng.choice([0, 0, 1, 5]))) for _ in
                      range(_log(rng, 1, 64) + 1)]
            c = clip("", dtype, ",".join(widths), G, clipped=rng.random() < 0.6)
        del c["name"]
        if work(c)["bytes"] <= most[kind]:
            return c


def _tensor_shapes(case):
    """Per layer of the stack: the norm's weight and bias, coef and base_w."""
    s, nb = [int(v) for v in case["sizes"].split(",")], case["G"] + 3
    for n_in, n_out in zip(s, s[1:]):
        yield from ((n_in,), (n_in,), (n_out, n_in, nb), (n_out, n_in))


def work(case):
    """Each input read once, each output written once; the operations of the formulas, an
    exponential counted as one."""
    e = 4 if case["dtype"] == "f32" else 2
    kind = case["kind"]
    if kind == "clip":
        n = sum(math.prod(s) for s in _tensor_shapes(case))
        return {"bytes": n * e * (2 if case["clipped"] else 1) + 4,
                "flops": n * (3 if case["clipped"] else 2)}
    rows = case["rows"]
    if kind in ("norm", "norm_grad"):
        n, p = case["n"], 4 if case["params"] == "f32" else 2
        if kind == "norm":
            b = rows * n * e * (4 if case["residual"] else 2) + 2 * n * p
            return {"bytes": b + (8 * rows if case["stats"] else 0), "flops": 8 * rows * n}
        b = rows * n * e * (4 if case["residual"] else 3) + 3 * n * p + 8 * rows
        return {"bytes": b, "flops": 14 * rows * n}
    V, ent = case["classes"], case["entropy"]
    if kind == "logprob":
        b = rows * (V * e + 8 + 4 + 8 + (4 if ent else 0) + 12 * case["top_k"])
        return {"bytes": b, "flops": rows * V * (6 if ent else 4)}
    b = rows * (2 * V * e + 8 + 8 + 4 + (8 if ent else 0))
    return {"bytes": b, "flops": rows * V * (6 if ent else 4)}


# ---------------------------------------------------------------- inputs

def prepare(case, seed):
    dev, dt, kind = torch.device("cuda"), DTYPES[case["dtype"]], case["kind"]
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)

    def randn(*shape, std=1.0, mean=0.0, dtype=dt):
        return (torch.randn(*shape, device=dev, generator=gen) * std + mean).to(dtype)

    state = dict(case=case)
    if kind in ("norm", "norm_grad"):
        rows, n, pt = case["rows"], case["n"], DTYPES[case["params"]]
        # rows of different centres and spreads, as a residual stream has
        centre = torch.randn(rows, 1, device=dev, generator=gen)
        spread = torch.rand(rows, 1, device=dev, generator=gen) * 2 + 0.25
        x = torch.randn(rows, n, device=dev, generator=gen).mul_(spread).add_(centre).to(dt)
        state.update(x=x, weight=randn(n, std=0.2, mean=1.0, dtype=pt),
                     bias=randn(n, std=0.2, dtype=pt))
        if kind == "norm":
            state["residual"] = randn(rows, n) if case["residual"] else None
        else:
            h = x.float()
            mean = h.mean(1)
            var = (h - mean[:, None]).square_().mean(1)
            state.update(mean=mean, rstd=(var + EPS).rsqrt_(), dy=randn(rows, n),
                         dh=randn(rows, n) if case["residual"] else None)
    elif kind in ("logprob", "logprob_grad"):
        rows, V = case["rows"], case["classes"]
        z = torch.randn(rows, V + case["pad"], device=dev, generator=gen).mul_(3.0)
        target = torch.randint(0, V, (rows,), device=dev, generator=gen)
        if case["masked"]:
            mask = torch.rand(rows, V + case["pad"], device=dev, generator=gen) < 0.5
            z.masked_fill_(mask.scatter_(1, target[:, None], False), -math.inf)
        if case["ignored"]:
            drop = torch.rand(rows, device=dev, generator=gen) < 0.1
            target = torch.where(drop, IGNORE, target)
        z = z.to(dt)[:, :V]
        state.update(z=z, target=target)
        if kind == "logprob_grad":
            zf = z.float()
            m = zf.amax(1)
            e = (zf - m[:, None]).exp_()
            s = e.sum(1)
            state["stats"] = torch.stack([m, s.log()], 1)
            # (the loss: a weighted mean over the rows, less an entropy bonus)
            state["dlogp"] = -torch.rand(rows, device=dev, generator=gen)
            if case["entropy"]:
                zm = (zf - m[:, None]).clamp_(min=-1e4)
                state["ent"] = s.log() - (e * zm).sum(1) / s
                state["dent"] = torch.rand(rows, device=dev, generator=gen) * -0.1
    else:
        # views of one buffer, one after the other, as gradients that are also summed over GPUs are
        # held; the clipped ones go to a second buffer, so that a pass can be run again
        total = sum(math.prod(s) for s in _tensor_shapes(case))
        norm2 = 0.02 * math.sqrt(total)
        flat = randn(total, std=0.02)
        state["flat"] = torch.empty_like(flat) if case["clipped"] else flat
        state["grads"] = _views(case, flat)
        state["max_norm"] = norm2 / 8 if case["clipped"] else norm2 * 4
        state["out"] = _views(case, state["flat"]) if case["clipped"] else None
    return state


def _views(case, flat):
    shapes = list(_tensor_shapes(case))
    parts = flat.split([math.prod(s) for s in shapes])
    return [p.view(s) for p, s in zip(parts, shapes)]


# ---------------------------------------------------------------- one pass

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(state):
    from paper_2609_01956_amd import binding as kb
    case, kind = state["case"], state["case"]["kind"]
    if kind == "norm":
        y, h, mean, rstd = kb.layer_norm(state["x"], state["weight"], state["bias"], EPS,
                                         residual=state["residual"], need_stats=case["stats"])
        return ([y] + ([h] if case["residual"] else []) + ([mean, rstd] if case["stats"] else []))
    if kind == "norm_grad":
        return kb.layer_norm_backward(state["x"], state["mean"], state["rstd"], state["weight"],
                                      state["dy"], dh=state["dh"])
    if kind == "logprob":
        logp, stats, ent, top, idx = kb.token_logprobs(
            state["z"], state["target"], top_k=case["top_k"], entropy=case["entropy"],
            ignore_index=IGNORE)
        return [logp, stats] + ([ent] if case["entropy"] else []) + \
            ([top, idx] if case["top_k"] else [])
    if kind == "logprob_grad":
        return kb.token_logprobs_backward(
            state["z"], state["target"], state["stats"], state["dlogp"], entropy=state.get("ent"),
            dentropy=state.get("dent"), ignore_index=IGNORE)
    return kb.clip_grad_norm(state["grads"], state["max_norm"], out=state["out"]), state["flat"]


def _run_plain(state):
    case, kind = state["case"], state["case"]["kind"]
    dt = DTYPES[case["dtype"]]
    if kind == "norm":
        h = state["x"].float()
        if case["residual"]:
            h = h + state["residual"].float()
        mean = h.mean(1)
        c = h - mean[:, None]
        rstd = ((c * c).mean(1) + EPS).rsqrt()
        y = (c * rstd[:, None] * state["weight"].float() + state["bias"].float()).to(dt)
        return ([y] + ([h.to(dt)] if case["residual"] else []) +
                ([mean, rstd] if case["stats"] else []))
    if kind == "norm_grad":
        dy, rstd = state["dy"].float(), state["rstd"][:, None]
        xh = (state["x"].float() - state["mean"][:, None]) * rstd
        g = dy * state["weight"].float()
        dx = (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) * rstd
        if case["residual"]:
            dx = dx + state["dh"].float()
        pt = DTYPES[case["params"]]
        return dx.to(dt), (dy * xh).sum(0).to(pt), dy.sum(0).to(pt)
    if kind == "logprob":
        z, target = state["z"].float(), state["target"]
        m = z.amax(1)
        zm = z - m[:, None]
        e = zm.exp()
        s = e.sum(1)
        logs = s.log()
        valid = target != IGNORE
        zt = zm.gather(1, torch.where(valid, target, 0)[:, None])[:, 0]
        out = [torch.where(valid, zt - logs, 0.0), torch.stack([m, logs], 1)]
        if case["entropy"]:
            out.append(logs - torch.where(e > 0, e * zm, 0.0).sum(1) / s)
        if case["top_k"]:
            # (argmax gives the first of equal values)
            values, indices = [], []
            for _ in range(case["top_k"]):
                i = zm.argmax(1, keepdim=True)
                values.append(zm.gather(1, i))
                indices.append(i)
                zm = zm.scatter(1, i, -math.inf)
            out += [torch.cat(values, 1) - logs[:, None], torch.cat(indices, 1)]
        return out
    if kind == "logprob_grad":
        target, stats = state["target"], state["stats"]
        valid = target != IGNORE
        d = torch.where(valid, state["dlogp"], 0.0)
        lp = state["z"].float() - stats[:, :1] - stats[:, 1:]
        p = lp.exp()
        dz = p * -d[:, None]
        if case["entropy"]:
            lp = torch.where(p > 0, lp, 0.0) + state["ent"][:, None]
            dz = dz - p * lp * state["dent"][:, None]
        rows = torch.arange(dz.shape[0], device=dz.device)
        dz[rows, torch.where(valid, target, 0)] += d
        return dz.to(dt)
    grads = state["grads"]
    total = torch.stack([g.float().square().sum() for g in grads]).sum().sqrt()
    coef = (state["max_norm"] / (total + 1e-6)).clamp(max=1.0)
    for g, o in zip(grads, grads if state["out"] is None else state["out"]):
        o.copy_(g.float() * coef)
    return total, state["flat"]


# ---------------------------------------------------------------- 64 bits

def exact(case, seed):
    state, kind = prepare(case, seed), case["kind"]
    if kind == "norm":
        parts = []
        w, b = state["weight"].double(), state["bias"].double()
        step = max(1, (1 << 26) // case["n"])
        for i in range(0, case["rows"], step):
            h = state["x"][i:i + step].double()
            if case["residual"]:
                h = h + state["residual"][i:i + step].double()
            var, mean = torch.var_mean(h, 1, correction=0)
            rstd = 1.0 / (var + EPS).sqrt()
            y = torch.addcmul(b, (h - mean.unsqueeze(1)) * rstd.unsqueeze(1), w)
            parts.append([y] + ([h] if case["residual"] else []) +
                         ([mean, rstd] if case["stats"] else []))
        return [torch.cat(p) for p in zip(*parts)]
    if kind == "norm_grad":
        n, dxs = case["n"], []
        w = state["weight"].double()
        dw, db = torch.zeros_like(w), torch.zeros_like(w)
        step = max(1, (1 << 26) // n)
        for i in range(0, case["rows"], step):
            rstd = state["rstd"][i:i + step].double().unsqueeze(1)
            dy = state["dy"][i:i + step].double()
            xh = (state["x"][i:i + step].double() -
                  state["mean"][i:i + step].double().unsqueeze(1)) * rstd
            dw += torch.linalg.vecdot(dy, xh, dim=0)
            db += dy.sum(0)
            # the projection of w dy that leaves out the row's constant and its xh direction
            g = w * dy
            along = torch.linalg.vecdot(g, xh, dim=1).unsqueeze(1) / n
            dx = rstd * (g - g.sum(1, keepdim=True) / n - along * xh)
            dxs.append(dx + state["dh"][i:i + step].double() if case["residual"] else dx)
        return torch.cat(dxs), dw, db
    if kind == "logprob":
        parts = []
        step = max(1, (1 << 25) // case["classes"])
        for i in range(0, case["rows"], step):
            z, t = state["z"][i:i + step].double(), state["target"][i:i + step]
            m = z.amax(1)
            lse = torch.logsumexp(z, 1)
            lp = z - lse.unsqueeze(1)
            lpt = lp.gather(1, t.clamp(min=0).unsqueeze(1)).squeeze(1).masked_fill(t == IGNORE, 0.0)
            out = [lpt, torch.stack([m, lse - m], 1)]
            if case["entropy"]:
                out.append(torch.special.entr(lp.exp()).sum(1))
            if case["top_k"]:
                idx = torch.sort(z, dim=1, descending=True, stable=True)[1][:, :case["top_k"]]
                out += [lp.gather(1, idx), idx.clone()]
            parts.append(out)
        return [torch.cat(p) for p in zip(*parts)]
    if kind == "logprob_grad":
        parts = []
        step = max(1, (1 << 25) // case["classes"])
        for i in range(0, case["rows"], step):
            t = state["target"][i:i + step]
            lse = state["stats"][i:i + step].double().sum(1, keepdim=True)
            d = state["dlogp"][i:i + step].double().masked_fill(t == IGNORE, 0.0).unsqueeze(1)
            lp = state["z"][i:i + step].double() - lse
            p = lp.exp()
            slope = d
            if case["entropy"]:
                h = state["ent"][i:i + step].double().unsqueeze(1)
                slope = d + state["dent"][i:i + step].double().unsqueeze(1) * \
                    (lp.clamp(min=-1e5) + h)
            dz = -p * slope
            dz.scatter_add_(1, t.clamp(min=0).unsqueeze(1), d)
            parts.append(dz)
        return torch.cat(parts)
    grads = state["grads"]
    total = math.sqrt(sum(float(torch.linalg.vector_norm(g, dtype=torch.float64)) ** 2
                          for g in grads))
    c = min(1.0, state["max_norm"] / (total + 1e-6))
    return (torch.tensor(total, dtype=torch.float64, device=grads[0].device),
            torch.cat([g.double().reshape(-1) for g in grads]) * c)
