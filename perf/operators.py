"""The training operators that stand next to the barrier search, as measurable cases.

What a worker computes between two barriers and what the server does at one: the gated feed-forward block with its
backward pass, the distillation loss from a teacher's top logits with its gradient, and the merge of the workers' pushes
weighted by the iterations that a search gave them.  ``run`` computes them in plain torch operations in 32 bits, or, where
``own`` is set, by the package's entry points.  Inputs are drawn on the GPU from the seed.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}


def _ff(name, mode, M, K, F, dtype, act="silu"):
    """M tokens of width K through F gated units; ``mode``: "forward" (answers) or "train" (with the gradients)."""
    case = {"op": "ff", "mode": mode, "M": M, "K": K, "F": F, "dtype": dtype, "act": act}
    return {"name": name, **case} if name else case


def _distill(name, mode, N, V, top, dtype, temperature=2.0, kl=1.0, ce=0.0, masked=False):
    """N rows over a vocabulary of V, ``top`` teacher entries a row; ``mode``: "loss" (evaluation), "step" (loss and gradient
    in one call) or "separate" (the loss first, its gradient from what the loss saved).  ``masked``: the last 16 entries of
    the vocabulary are padding, masked with -inf."""
    case = {"op": "distill", "mode": mode, "N": N, "V": V, "top": top, "dtype": dtype, "temperature": temperature, "kl": kl,
            "ce": ce, "masked": masked}
    return {"name": name, **case} if name else case


def _merge(name, P, n, dtype, momentum=0.0, nesterov=False):
    """Pushes of P workers over n weights."""
    case = {"op": "merge", "P": P, "n": n, "dtype": dtype, "momentum": momentum, "nesterov": nesterov}
    return {"name": name, **case} if name else case


def listed():
    return [
        # answering with the trained model, one token at a time: the weights are read once, latency counts
        _ff("ff_token", "forward", 1, 4096, 12288, "bf16"),
        # the same for sixteen requests at once, in the other 16-bit type
        _ff("ff_requests_16", "forward", 16, 2048, 6144, "f16", "gelu_tanh"),
        # a prompt, or an evaluation without gradients
        _ff("ff_prompt_2048", "forward", 2048, 2048, 8192, "bf16"),
        # a worker's iteration at full size: the block and all its gradients
        _ff("ff_train_8192", "train", 8192, 4096, 12288, "bf16"),
        # a batch whose tokens, width and units are no multiples of anything (packed ragged sequences, pruned units)
        _ff("ff_train_odd", "train", 1021, 1000, 2730, "bf16", "gelu"),
        # a small model in full precision, as a convergence study trains it
        _ff("ff_train_f32", "train", 1024, 1024, 2816, "f32"),
        # evaluating a single row: latency counts
        _distill("distill_row", "loss", 1, 32000, 16, "bf16"),
        # a worker's iteration at full size: loss and gradient, labels mixed in, vocabulary padding masked
        _distill("distill_step_4096", "step", 4096, 128000, 64, "bf16", 2.0, 0.9, 0.1, True),
        # an odd vocabulary in full precision, the gradient in a call of its own
        _distill("distill_separate_odd", "separate", 509, 50021, 100, "f32", 1.0, 0.5, 0.5),
        # four workers of a small model: launches count
        _merge("merge_4x1M", 4, 1_000_003, "f32"),
        # configuration 2's sixteen workers over a larger model, with the server's momentum
        _merge("merge_16x64M", 16, 64_000_000, "bf16", 0.9, True),
        # configuration 5's 1024 workers over a small one
        _merge("merge_1024x512K", 1024, 524_309, "bf16"),
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _size(rng, lo, hi):
    """A width: a multiple of 64 half of the time, of 8 for a quarter, anything else."""
    n = _log(rng, lo, hi)
    step = rng.choice([64, 64, 8, 1])
    return max(lo, n // step * step)


def draw(rng):
    op = rng.choice(["ff", "ff", "distill", "merge"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "ff":
        mode = rng.choice(["forward", "train"])
        M = _log(rng, 1, 1024 if dtype == "f32" else 8192)
        K, F = _size(rng, 64, 4096), _size(rng, 64, 12288)
        if dtype == "f32":
            F = min(F, 4096)
        return _ff("", mode, M, K, F, dtype, rng.choice(["silu", "gelu", "gelu_tanh", "relu", "sigmoid"]))
    if op == "distill":
        V = _size(rng, 1000, 128000)
        N = _log(rng, 1, min(4096, (4096 * 128000) // (V * (2 if dtype == "f32" else 1))))
        kl, ce = rng.choice([(1.0, 0.0), (0.5, 0.5), (0.9, 0.1)])
        return _distill("", rng.choice(["loss", "step", "separate"]), N, V, _log(rng, 1, 256), dtype, rng.choice([1.0, 2.0, 4.0]),
                        kl, ce, rng.random() < 0.5)
    P = _log(rng, 2, 1024)
    n = _log(rng, 1000, min(64_000_000, (16 * 64_000_000) // P // (2 if dtype == "f32" else 1)))
    momentum = rng.choice([0.0, 0.9])
    return _merge("", P, n, dtype, momentum, momentum > 0 and rng.random() < 0.5)


def _gen(seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    return gen


def _normal(gen, shape, scale, dtype):
    return (torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32) * scale).to(dtype)


def prepare(case, seed):
    gen = _gen(seed)
    state = {"case": case}
    if case["op"] == "ff":
        t, M, K, F = TYPES[case["dtype"]], case["M"], case["K"], case["F"]
        state["x"] = _normal(gen, (M, K), 1.0, t)                       # tokens behind a normalisation
        state["wg"] = _normal(gen, (F, K), K ** -0.5, t)
        state["wu"] = _normal(gen, (F, K), K ** -0.5, t)
        if case["mode"] == "train":
            state["dh"] = _normal(gen, (M, F), 0.05, t)
    elif case["op"] == "distill":
        t, N, V, top = TYPES[case["dtype"]], case["N"], case["V"], case["top"]
        logits = _normal(gen, (N, V), 2.5, t)
        if case["masked"]:
            logits[:, V - 16:] = float("-inf")
        noise = torch.randn((N, V), generator=gen, device=DEVICE, dtype=torch.float32)
        values, index = torch.topk(noise.add_(logits.float()), top, dim=1)     # the teacher: near the student, not the same
        del noise
        draws = torch.rand((2, N), generator=gen, device=DEVICE)
        # a tenth of the rows come with fewer entries than there is room for; if there are many rows, one comes with none
        length = torch.where(draws[0] < 0.1, (draws[0] * 10 * top).long(), top)
        if N >= 8:
            length[N // 2] = 0
        else:
            length.clamp_(min=1)
        state["index"] = torch.where(torch.arange(top, device=DEVICE)[None, :] < length[:, None], index, -1)
        state["values"] = values.to(t)
        state["labels"] = None
        if case["ce"] > 0:
            state["labels"] = torch.where(draws[1] < 0.05, -100, index[:, 0])  # some positions of a sequence have no label
        state["logits"] = logits
        state["weight"] = torch.full((N,), 1.0 / N, device=DEVICE)
    else:
        t, P, n = TYPES[case["dtype"]], case["P"], case["n"]
        state["weights"] = _normal(gen, (n,), 0.02, torch.float32)
        state["velocity"] = _normal(gen, (n,), 1e-3, torch.float32) if case["momentum"] > 0 else None
        state["iters"] = torch.randint(1, 65, (P,), generator=gen, device=DEVICE, dtype=torch.int32)
        pushes = torch.empty((P, n), dtype=t, device=DEVICE)
        for p in range(P):
            pushes[p] = _normal(gen, (n,), 1e-3, t)
        state["pushes"] = pushes
        state["lr"] = 0.7
    return state


def _act(name, g):
    """act(g) and act'(g), in g's own precision."""
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    if name == "sigmoid":
        s = torch.sigmoid(g)
        return s, s * (1 - s)
    if name == "relu":
        return g.clamp(min=0), (g > 0).to(g.dtype)
    if name == "gelu":
        cdf = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    c, a = math.sqrt(2 / math.pi), 0.044715                             # gelu_tanh
    th = torch.tanh(c * (g + a * g * g * g))
    return 0.5 * g * (1 + th), 0.5 * (1 + th) + 0.5 * g * (1 - th * th) * c * (1 + 3 * a * g * g)


def _run_ff(state):
    case, x, wg, wu = state["case"], state["x"], state["wg"], state["wu"]
    if own:
        from paper_2001_01347_amd import training
        if case["mode"] == "forward":
            return training.ebsp_gated_ff_forward(x, wg, wu, case["act"])[0]
        h, g, u = training.ebsp_gated_ff_forward(x, wg, wu, case["act"], save=True)
        return (h, *training.ebsp_gated_ff_backward(state["dh"], x, wg, wu, g, u, case["act"]))
    t = x.dtype
    xf, gf, uf = x.float(), wg.float(), wu.float()
    g, u = xf @ gf.t(), xf @ uf.t()
    a, da = _act(case["act"], g)
    h = (a * u).to(t)
    if case["mode"] == "forward":
        return h
    dh = state["dh"].float()
    dg, du = dh * u * da, dh * a
    return h, (dg @ gf + du @ uf).to(t), (dg.t() @ xf).to(t), (du.t() @ xf).to(t)


def _run_distill(state):
    case, s, labels = state["case"], state["logits"], state["labels"]
    T, kl, ce = case["temperature"], case["kl"], case["ce"]
    if own:
        from paper_2001_01347_amd import training
        args = dict(temperature=T, kl_weight=kl, labels=labels, ce_weight=ce)
        if case["mode"] == "step":
            loss, grad, _ = training.ebsp_distill_loss_grad(s, state["index"], state["values"], state["weight"], **args)
            return loss, grad
        loss, stats, _ = training.ebsp_distill_forward(s, state["index"], state["values"], **args)
        if case["mode"] == "loss":
            return loss
        return loss, training.ebsp_distill_backward(s, state["index"], state["values"], stats, state["weight"], **args)
    t, sf = s.dtype, s.float()
    index, given = state["index"].clamp(min=0), state["index"] >= 0
    some = given.any(dim=1, keepdim=True)
    top = torch.where(given, state["values"].float(), float("-inf"))
    top = torch.where(some, top - top.amax(dim=1, keepdim=True), 0.0) / T
    weight = torch.where(given, torch.exp(top), 0.0)
    total = weight.sum(dim=1, keepdim=True).clamp(min=1e-30)
    q = weight / total
    high = sf.amax(dim=1, keepdim=True)
    e = torch.exp((sf - high) / T)
    sums = e.sum(dim=1, keepdim=True)
    logp = (sf.gather(1, index) - high) / T - torch.log(sums)
    term = torch.where(q > 0, q * (top - torch.log(total) - logp), 0.0)
    loss = kl * T * T * term.sum(dim=1)
    if labels is not None:
        has = labels >= 0
        e1 = torch.exp(sf - high)
        sums1 = e1.sum(dim=1, keepdim=True)
        at = labels.clamp(min=0)[:, None]
        nll = -((sf.gather(1, at) - high) - torch.log(sums1))
        loss = loss + ce * torch.where(has, nll[:, 0], 0.0)
    if case["mode"] == "loss":
        return loss
    grad = e.div_(sums).mul_(some)
    grad = grad.scatter_add_(1, index, -q).mul_(kl * T)
    if labels is not None:
        p1 = e1.div_(sums1).scatter_add_(1, at, torch.full_like(sums1, -1.0))
        grad.add_(p1.mul_(ce * has[:, None]))
    return loss, grad.mul_(state["weight"][:, None]).to(t)


def _run_merge(state):
    case = state["case"]
    w, v, pushes, lr, mu = state["weights"], state["velocity"], state["pushes"], state["lr"], case["momentum"]
    if own:
        from paper_2001_01347_amd import training
        out, v2, pulled = training.ebsp_merge_pushes(w, pushes, state["iters"], lr=lr, momentum=mu, nesterov=case["nesterov"],
                                                     velocity=v, pull=pushes.dtype)
        return (out, pulled) if v is None else (out, pulled, v2)
    c = state["iters"].float()
    c = c / c.sum()
    avg = torch.zeros_like(w)
    for p in range(case["P"]):
        avg += pushes[p].float() * c[p]
    step = avg
    if v is not None:
        v2 = mu * v + avg
        step = avg + mu * v2 if case["nesterov"] else v2
    out = w + lr * step
    pulled = out.to(pushes.dtype)
    return (out, pulled) if v is None else (out, pulled, v2)


def run(state):
    return {"ff": _run_ff, "distill": _run_distill, "merge": _run_merge}[state["case"]["op"]](state)


def work(case):
    s = SIZE[case["dtype"]]
    if case["op"] == "ff":
        M, K, F = case["M"], case["K"], case["F"]
        read, product = M * K + 2 * F * K, 2.0 * M * K * F
        if case["mode"] == "forward":
            return {"bytes": s * (read + M * F), "flops": 2 * product}
        return {"bytes": s * (read + M * F + M * F + M * K + 2 * F * K), "flops": 6 * product}
    if case["op"] == "distill":
        N, V, top = case["N"], case["V"], case["top"]
        small = N * top * (8 + s) + (8 * N if case["ce"] > 0 else 0) + 4 * N
        per = 4 + (4 if case["ce"] > 0 else 0)                          # the largest, a difference, an exponential, a sum
        if case["mode"] == "loss":
            return {"bytes": s * N * V + small, "flops": float(per * N * V)}
        return {"bytes": 2 * s * N * V + small + 4 * N, "flops": float((per + 3) * N * V)}
    P, n = case["P"], case["n"]
    momentum = 8 * n if case["momentum"] > 0 else 0
    return {"bytes": P * n * s + 8 * n + n * s + momentum + 4 * P, "flops": 2.0 * P * n}


def _exact_ff(case, state):
    x, wg, wu = (state[k].double() for k in ("x", "wg", "wu"))
    g = (x @ wg.t()).requires_grad_(case["mode"] == "train")
    F = torch.nn.functional
    a = {"silu": F.silu, "relu": F.relu, "sigmoid": torch.sigmoid, "gelu": F.gelu,
         "gelu_tanh": lambda v: F.gelu(v, approximate="tanh")}[case["act"]](g)
    u = x @ wu.t()
    h = a.detach() * u
    if case["mode"] == "forward":
        return h
    du = state["dh"].double()
    (dg,) = torch.autograd.grad(a, g, du * u)
    du = du * a.detach()
    dx = dg @ wg
    dx += du @ wu
    return h, dx, dg.t() @ x, du.t() @ x


def _exact_distill(case, state):
    N, V, T = case["N"], case["V"], case["temperature"]
    losses, grads = [], []
    rows = max(1, (1 << 27) // V)
    for r in range(0, N, rows):
        at = slice(r, min(r + rows, N))
        s = state["logits"][at].double().requires_grad_()
        index, values = state["index"][at], state["values"][at].double()
        n = s.shape[0]
        logq = torch.log_softmax(torch.where(index >= 0, values, float("-inf")) / T, dim=1)
        logq = torch.where(index >= 0, logq, float("-inf"))
        logp = torch.log_softmax(s / T, dim=1).gather(1, index.clamp(min=0))
        q = torch.exp(logq)
        kl = torch.where(q > 0, q * (torch.where(q > 0, logq, 0.0) - torch.where(q > 0, logp, 0.0)), 0.0).sum(dim=1)
        loss = case["kl"] * T * T * kl
        if state["labels"] is not None:
            label = state["labels"][at]
            nll = -torch.log_softmax(s, dim=1)[torch.arange(n, device=s.device), label.clamp(min=0)]
            loss = loss + case["ce"] * torch.where(label >= 0, nll, 0.0)
        losses.append(loss.detach())
        if case["mode"] != "loss":
            (grad,) = torch.autograd.grad(loss, s, state["weight"][at].double())
            grads.append(grad)
        del s, logp, loss
    return torch.cat(losses) if case["mode"] == "loss" else (torch.cat(losses), torch.cat(grads))


def _exact_merge(case, state):
    c = state["iters"].double()
    c = c / c.sum()
    n = case["n"]
    avg = torch.empty(n, dtype=torch.float64, device=DEVICE)
    cols = max(1, (1 << 28) // case["P"])
    for r in range(0, n, cols):
        avg[r:r + cols] = c @ state["pushes"][:, r:r + cols].double()
    w, mu, lr = state["weights"].double(), case["momentum"], state["lr"]
    if state["velocity"] is None:
        out = w + lr * avg
        return out, out
    v = mu * state["velocity"].double() + avg
    out = w + lr * (avg + mu * v if case["nesterov"] else v)
    return out, out, v


def exact(case, seed):
    state = prepare(case, seed)
    return {"ff": _exact_ff, "distill": _exact_distill, "merge": _exact_merge}[case["op"]](case, state)
