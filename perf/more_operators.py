"""The operators of fine-tuning that stand next to the feed-forward block and the distillation loss, as measurable cases.

What a worker that tunes a model on answers computes between two barriers: the residual stream around a block (the norm behind
the block, its gate and residual scale, dropout, and the norm before the next block, as one operator), dropout by itself, the
log-probabilities of tokens, the clipped policy loss with a KL term, and the preference loss of pairs of answers.  ``run``
computes them in plain torch operations in 32 bits (sums over a whole answer in 64), or, where ``own`` is set, by the package's
entry points.  Inputs are drawn on the GPU from the seed.
"""
import math
import random

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
NONE = -100                                                                  # the token of a row that has none


def _norm(name, mode, M, K, dtype, stream="", branch=True, post=False, gate="none", p=0.0):
    """M tokens of width K; ``mode``: "forward" (answers) or "train" (with all gradients).  ``stream``: the residual stream's type where it
    is another than the block's; ``branch``: a block's output is added (else the first norm of a model); ``post``: it is normed
    before; ``gate``: "none", "channel" or "token" (a gate for every element)."""
    case = {"op": "norm", "mode": mode, "M": M, "K": K, "dtype": dtype, "stream": stream or dtype, "branch": branch, "post": post and branch,
            "gate": gate if branch else "none", "p": p if branch else 0.0}
    return {"name": name, **case} if name else case


def _dropout(name, mode, M, K, dtype, p):
    case = {"op": "dropout", "mode": mode, "M": M, "K": K, "dtype": dtype, "p": p}
    return {"name": name, **case} if name else case


def _logp(name, mode, N, V, dtype, temperature=1.0, masked=False):
    """N rows over a vocabulary of V; ``mode``: "forward" (a rollout's record) or "train" (with the logits' gradient).  ``masked``: the last
    16 entries of the vocabulary are padding, masked with -inf."""
    case = {"op": "logp", "mode": mode, "N": N, "V": V, "dtype": dtype, "temperature": temperature, "masked": masked}
    return {"name": name, **case} if name else case


def _policy(name, mode, N, V, dtype, temperature=1.0, kl=0.0, low=0.2, high=0.2, masked=False):
    """``mode``: "loss" (evaluation), "step" (loss and gradient in one call) or "separate" (the gradient in a call of its own)."""
    case = {"op": "policy", "mode": mode, "N": N, "V": V, "dtype": dtype, "temperature": temperature, "kl": kl, "low": low, "high": high,
            "masked": masked}
    return {"name": name, **case} if name else case


def _preference(name, mode, pairs, length, V, dtype, kind="sigmoid", beta=0.1, smoothing=0.0, mean=False, behind=0):
    """Pairs of answers of length // 2 to ``length`` tokens, the first quarter of each a prompt without tokens to score, packed one behind
    the other; ``behind``: rows of the batch behind the last answer."""
    case = {"op": "preference", "mode": mode, "pairs": pairs, "length": length, "V": V, "dtype": dtype, "kind": kind, "beta": beta,
            "smoothing": smoothing, "mean": mean, "behind": behind}
    return {"name": name, **case} if name else case


def listed():
    return [
        # answering, one token at a time: a block's output joins the stream, which is normed for the next block; latency counts
        _norm("norm_token", "forward", 1, 4096, "bf16"),
        # a prompt, or an evaluation without gradients, with the norm behind the block
        _norm("norm_prompt_2048", "forward", 2048, 4096, "bf16", post=True),
        # a worker's iteration at full size: both norms, a gate for every channel, dropout, and all the gradients
        _norm("norm_train_8192", "train", 8192, 4096, "bf16", post=True, gate="channel", p=0.1),
        # a batch of odd size and width on a stream kept in full precision, gated element by element
        _norm("norm_train_odd", "train", 1021, 1003, "f16", stream="f32", gate="token", p=0.05),
        # the hidden units of a block at full size
        _dropout("dropout_8192", "train", 8192, 12288, "bf16", 0.1),
        # a small, odd batch in full precision: launches count
        _dropout("dropout_odd", "forward", 61, 1001, "f32", 0.25),
        # a rollout records the log-probability of the token that it drew: one row, latency counts
        _logp("logp_token", "forward", 1, 32000, "bf16"),
        # the same for a batch of rollouts under the reference model, and the gradient for a loss of the user's own
        _logp("logp_train_1024", "train", 1024, 64000, "f16", 0.7, True),
        # a worker's iteration at full size: loss and gradient, vocabulary padding masked
        _policy("policy_step_4096", "step", 4096, 128000, "bf16", 1.0, 0.05, 0.2, 0.28, True),
        # an odd vocabulary in full precision, the gradient in a call of its own
        _policy("policy_separate_odd", "separate", 509, 50021, "f32", 0.8, 0.1),
        # sixteen pairs of answers in one step
        _preference("preference_step_16", "step", 16, 160, 64000, "bf16"),
        # one short, odd batch in full precision: rows behind the last answer, lengths divided out
        _preference("preference_separate_odd", "separate", 3, 41, 10007, "f32", "sigmoid", 2.0, 0.1, True, 5),
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
    op = rng.choice(["norm", "norm", "dropout", "logp", "policy", "policy", "preference"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    wide = 2 if dtype == "f32" else 1
    if op == "norm":
        K = _size(rng, 64, 16384)
        return _norm("", rng.choice(["forward", "train"]), _log(rng, 1, min(8192, 8192 * 4096 // K)), K, dtype,
                     rng.choice([dtype, dtype, "f32"]), rng.random() < 0.85, rng.random() < 0.5, rng.choice(["none", "channel", "token"]),
                     rng.choice([0.0, 0.0, 0.1, 0.5]))
    if op == "dropout":
        K = _size(rng, 64, 12288)
        return _dropout("", rng.choice(["forward", "train"]), _log(rng, 1, min(8192, 8192 * 12288 // K // wide)), K, dtype,
                        rng.choice([0.05, 0.1, 0.3, 0.5]))
    if op == "preference":
        V = _size(rng, 1000, 128000)
        pairs = _log(rng, 1, 32)
        length = _log(rng, 4, max(4, min(512, 2048 * 64000 // (V * wide) // (2 * pairs))))
        return _preference("", rng.choice(["loss", "step", "separate"]), pairs, length, V, dtype, rng.choice(["sigmoid", "sigmoid", "hinge", "square"]),
                           rng.choice([0.1, 0.3, 2.0]), rng.choice([0.0, 0.1]), rng.random() < 0.5, rng.choice([0, 0, 7]))
    V = _size(rng, 1000, 128000)
    N = _log(rng, 1, min(4096, 4096 * 128000 // (V * wide)))
    if op == "logp":
        return _logp("", rng.choice(["forward", "train"]), N, V, dtype, rng.choice([1.0, 1.0, 0.7, 2.0]), rng.random() < 0.5)
    return _policy("", rng.choice(["loss", "step", "separate"]), N, V, dtype, rng.choice([1.0, 1.0, 0.7]), rng.choice([0.0, 0.05, 0.2]), 0.2,
                   rng.choice([0.2, 0.28]), rng.random() < 0.5)


def _gen(seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    return gen


def _normal(gen, shape, scale, dtype):
    return (torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32) * scale).to(dtype)


def _lengths(case):
    """Tokens of every answer: the same for any seed, so that what a pass has to move is known."""
    rng = random.Random(case["pairs"] * 1009 + case["length"])
    return [rng.randint(max(1, case["length"] // 2), case["length"]) for _ in range(2 * case["pairs"])]


def _tokens(gen, logits, temperature):
    """A token of every row, drawn from its distribution, and its log-probability."""
    N, V = logits.shape
    tokens = torch.empty(N, dtype=torch.int64, device=DEVICE)
    logp = torch.empty(N, device=DEVICE)
    rows = max(1, (1 << 28) // V)
    for r in range(0, N, rows):
        s = logits[r:r + rows].float() / temperature
        draws = torch.rand(s.shape, generator=gen, device=DEVICE).clamp_(min=1e-20)
        tokens[r:r + rows] = torch.argmax(s - torch.log(-torch.log(draws)), dim=1)
        logp[r:r + rows] = torch.log_softmax(s, dim=1).gather(1, tokens[r:r + rows, None])[:, 0]
    return tokens, logp


def prepare(case, seed):
    gen = _gen(seed)
    state = {"case": case}
    if case.get("p", 0.0) > 0:
        state["rng"] = (0x5DEECE66D * (seed + 1) % (1 << 63), 7 * seed + 1)  # a run's seed, and the place of this call in it
    if case["op"] == "norm":
        t, ts, M, K = TYPES[case["dtype"]], TYPES[case["stream"]], case["M"], case["K"]
        state["x"] = _normal(gen, (M, K), 1.5, ts)
        state["branch"] = _normal(gen, (M, K), 0.7, t) if case["branch"] else None
        state["weight"] = 1 + _normal(gen, (K,), 0.1, t)
        state["post_weight"] = 1 + _normal(gen, (K,), 0.1, t) if case["post"] else None
        state["gate"] = {"none": None, "channel": _normal(gen, (K,), 0.5, t) if case["gate"] == "channel" else None,
                         "token": torch.sigmoid(_normal(gen, (M, K), 1.0, torch.float32)).to(t) if case["gate"] == "token" else None}[case["gate"]]
        state["scale"] = 0.5 if case["branch"] else 1.0
        if case["mode"] == "train":
            state["dy"] = _normal(gen, (M, K), 0.05, ts)
            state["dn"] = _normal(gen, (M, K), 0.05, t)
    elif case["op"] == "dropout":
        t, M, K = TYPES[case["dtype"]], case["M"], case["K"]
        state["x"] = _normal(gen, (M, K), 1.0, t)
        if case["mode"] == "train":
            state["dy"] = _normal(gen, (M, K), 0.05, t)
    else:
        t, V = TYPES[case["dtype"]], case["V"]
        lengths = _lengths(case) if case["op"] == "preference" else None
        N = case["N"] if lengths is None else sum(lengths) + case["behind"]
        logits = _normal(gen, (N, V), 2.5, t)
        if case.get("masked"):
            logits[:, V - 16:] = float("-inf")
        tokens, logp = _tokens(gen, logits, case.get("temperature", 1.0))
        state["logits"], state["tokens"] = logits, tokens
        if lengths is None:
            tokens[15::16] = NONE                                            # padding of the answers
        else:
            starts, sums = [0], []
            for n in lengths:
                tokens[starts[-1]:starts[-1] + n // 4] = NONE
                sums.append(logp[starts[-1] + n // 4:starts[-1] + n].double().sum())
                starts.append(starts[-1] + n)
            state["starts"] = torch.tensor(starts, dtype=torch.int64, device=DEVICE)
            spread = torch.tensor([n ** 0.5 for n in lengths], device=DEVICE)
            count = torch.tensor([n - n // 4 for n in lengths], device=DEVICE)
            ref = torch.stack(sums) + 0.3 * spread * torch.randn(2 * case["pairs"], generator=gen, device=DEVICE)
            state["ref"] = (ref / count if case["mean"] else ref).float()
            state["dloss"] = torch.full((case["pairs"],), 1.0 / case["pairs"], device=DEVICE)
        if case["op"] == "policy":
            moved = 0.15 * torch.randn(N, generator=gen, device=DEVICE)      # how far the policy has moved since the rollout
            for border in (math.log(1 - case["low"]), math.log(1 + case["high"])):
                moved = torch.where((moved - border).abs() < 1e-3, moved + 0.004, moved)    # no gradient depends on a last bit
            state["old"] = logp - moved
            state["ref"] = logp + 0.2 * torch.randn(N, generator=gen, device=DEVICE) if case["kl"] > 0 else None
            state["advantage"] = torch.randn(N, generator=gen, device=DEVICE)
        if case["op"] != "preference":
            state["dloss"] = torch.full((N,), 1.0 / N, device=DEVICE)
    return state


def _threshold(p):
    """Elements whose 16 bits are below this are dropped."""
    return int(round(p * 65536))


def _keep(M, K, p, rng):
    """Which elements of M rows of K stay: 16 bits each from the counter-based generator Philox4x32 of seven rounds (Salmon et al., 2011),
    eight of a row from the counter (place / 8, row, offset) and the key (seed)."""
    mask = 0xFFFFFFFF
    seed, offset = rng
    places = torch.arange((K + 7) // 8, dtype=torch.int64, device=DEVICE)[None, :]
    rows = torch.arange(M, dtype=torch.int64, device=DEVICE)[:, None]
    c = [places + 0 * rows, rows + 0 * places, torch.full_like(places + rows, offset & mask), torch.full_like(places + rows, offset >> 32)]
    k0, k1 = seed & mask, seed >> 32
    for _ in range(7):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57                          # modulo 2^64
        c = [(b >> 32 & mask) ^ c[1] ^ k0, b & mask, (a >> 32 & mask) ^ c[3] ^ k1, a & mask]
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    bits = torch.stack([v >> s & 0xFFFF for v in c for s in (0, 16)], dim=2).reshape(M, -1)[:, :K]
    return bits >= _threshold(p)


def _kept_factor(p):
    t = _threshold(p)
    return 65536.0 / (65536 - t) if t < 65536 else 0.0


def _run_norm(state):
    case, x, branch, weight, post_weight, gate = (state[k] for k in ("case", "x", "branch", "weight", "post_weight", "gate"))
    p, scale, eps = case["p"], state["scale"], 1e-6
    if own:
        from paper_2001_01347_amd import training
        args = dict(weight=weight, post_weight=post_weight, gate=gate, scale=scale, p=p, rng=state.get("rng"))
        y, n, stats = training.ebsp_residual_norm_forward(x, branch, eps=eps, **args)
        if case["mode"] == "forward":
            return (y, n) if branch is not None else (n,)
        grads = training.ebsp_residual_norm_backward(state["dy"], state["dn"], y, stats, branch, x=x, **args)
        return tuple(t for t in ((y if branch is not None else None), n, *grads) if t is not None)
    M, K = x.shape
    t, w = weight.dtype, weight.float()
    y = x.float()
    if branch is not None:
        b = branch.float()
        factor = torch.full((), scale, device=x.device)
        if p > 0:
            factor = torch.where(_keep(M, K, p, state["rng"]), scale * _kept_factor(p), 0.0)
        g = factor if gate is None else factor * gate.float()
        d = b
        if post_weight is not None:
            rb = torch.rsqrt((b * b).mean(dim=1, keepdim=True) + eps)
            b = b * rb
            d = b * post_weight.float()
        y = y + g * d
    ry = torch.rsqrt((y * y).mean(dim=1, keepdim=True) + eps)
    yh = y * ry
    out = ([y.to(x.dtype)] if branch is not None else []) + [(yh * w).to(t)]
    if case["mode"] == "forward":
        return tuple(out)
    dn = state["dn"].float()
    dw = (dn * yh).sum(dim=0)
    dn = dn * w
    dt = state["dy"].float() + ry * (dn - yh * (dn * yh).mean(dim=1, keepdim=True))
    out.append(dt.to(x.dtype))
    if branch is None:
        return (*out, dw.to(t))
    dd = g * dt
    dwp = None
    db = dd
    if post_weight is not None:
        dwp = (dd * b).sum(dim=0).to(t)
        db = dd * post_weight.float()
        db = rb * (db - b * (db * b).mean(dim=1, keepdim=True))
    out += [db.to(t), dw.to(t)]
    if dwp is not None:
        out.append(dwp)
    if gate is not None:
        dgate = factor * d * dt
        out.append((dgate.sum(dim=0) if gate.dim() == 1 else dgate).to(t))
    return tuple(out)


def _run_dropout(state):
    case, p = state["case"], state["case"]["p"]
    parts = [state["x"]] + ([state["dy"]] if case["mode"] == "train" else [])
    if own:
        from paper_2001_01347_amd import training
        return tuple(training.ebsp_dropout(t, p, state["rng"]) for t in parts)
    keep = _keep(case["M"], case["K"], p, state["rng"])
    return tuple(torch.where(keep, t.float() * _kept_factor(p), 0.0).to(t.dtype) for t in parts)


def _softmax(s, temperature):
    """p and the logarithms of a row's softmax, in 32 bits."""
    z = s.float() / temperature
    z = z - z.amax(dim=1, keepdim=True)
    e = torch.exp(z)
    total = e.sum(dim=1, keepdim=True)
    return e, total, z


def _spread(e, total, tokens, has, slope, temperature, dtype):
    """dL/dlogits from every row's dL/dlogp."""
    c = torch.where(has, slope / temperature, 0.0)[:, None]
    return e.div_(total).mul_(-c).scatter_add_(1, tokens[:, None], c).to(dtype)


def _run_logp(state):
    case, s, tokens, T = state["case"], state["logits"], state["tokens"], state["case"]["temperature"]
    if own:
        from paper_2001_01347_amd import training
        logp, stats, _ = training.ebsp_token_logp(s, tokens, T)
        if case["mode"] == "forward":
            return logp
        return logp, training.ebsp_token_logp_backward(s, tokens, stats, state["dloss"], T)
    has, at = tokens >= 0, tokens.clamp(min=0)
    e, total, z = _softmax(s, T)
    logp = torch.where(has, z.gather(1, at[:, None])[:, 0] - torch.log(total[:, 0]), 0.0)
    return logp if case["mode"] == "forward" else (logp, _spread(e, total, at, has, state["dloss"], T, s.dtype))


def _run_policy(state):
    case, s, tokens, T = state["case"], state["logits"], state["tokens"], state["case"]["temperature"]
    old, ref, advantage, kl = state["old"], state["ref"], state["advantage"], case["kl"]
    if own:
        from paper_2001_01347_amd import training
        args = dict(temperature=T, clip_low=case["low"], clip_high=case["high"], ref_logp=ref, kl_weight=kl)
        if case["mode"] == "step":
            loss, grad, logp, _ = training.ebsp_policy_loss_grad(s, tokens, old, advantage, state["dloss"], **args)
            return loss, logp, grad
        loss, logp, stats, _ = training.ebsp_policy_forward(s, tokens, old, advantage, **args)
        if case["mode"] == "loss":
            return loss, logp
        return loss, logp, training.ebsp_policy_backward(s, tokens, old, advantage, stats, state["dloss"], **args)
    has, at = tokens >= 0, tokens.clamp(min=0)
    e, total, z = _softmax(s, T)
    logp = torch.where(has, z.gather(1, at[:, None])[:, 0] - torch.log(total[:, 0]), 0.0)
    ratio = torch.exp(logp - old)
    whole, held = ratio * advantage, ratio.clamp(1 - case["low"], 1 + case["high"]) * advantage
    loss = -torch.minimum(whole, held)
    slope = torch.where(whole <= held, -whole, 0.0)
    if ref is not None:
        gap = ref - logp
        loss = loss + kl * (torch.expm1(gap) - gap)
        slope = slope - kl * torch.expm1(gap)
    loss = torch.where(has, loss, 0.0)
    if case["mode"] == "loss":
        return loss, logp
    return loss, logp, _spread(e, total, at, has, slope * state["dloss"], T, s.dtype)


def _pair_loss(case, h):
    """The loss of a pair and its slope, from the margin between its answers."""
    beta, smoothing = case["beta"], case["smoothing"]
    if case["kind"] == "hinge":
        return (1 - beta * h).clamp(min=0), torch.where(beta * h < 1, -beta, 0.0)
    if case["kind"] == "square":
        gap = h - 0.5 / beta
        return gap * gap, 2 * gap
    z = beta * h
    loss = torch.clamp(-z, min=0) + torch.log1p(torch.exp(-z.abs())) + smoothing * z
    return loss, beta * (torch.sigmoid(z) - 1 + smoothing)


def _run_preference(state):
    case, s, tokens, starts, ref = (state[k] for k in ("case", "logits", "tokens", "starts", "ref"))
    if own:
        from paper_2001_01347_amd import training
        smoothing = case["smoothing"] if case["kind"] == "sigmoid" else 0.0      # the other losses have none
        args = dict(ref=ref, beta=case["beta"], kind=case["kind"], smoothing=smoothing, mean=case["mean"])
        if case["mode"] == "step":
            loss, grad, sums, _ = training.ebsp_preference_loss_grad(s, tokens, starts, state["dloss"], **args)
            return loss, sums, grad
        loss, sums, saved, _ = training.ebsp_preference_forward(s, tokens, starts, **args)
        if case["mode"] == "loss":
            return loss, sums
        return loss, sums, training.ebsp_preference_backward(s, tokens, starts, saved, state["dloss"])
    has, at = tokens >= 0, tokens.clamp(min=0)
    e, total, z = _softmax(s, 1.0)
    logp = torch.where(has, z.gather(1, at[:, None])[:, 0] - torch.log(total[:, 0]), 0.0)
    answers = 2 * case["pairs"]
    of = torch.bucketize(torch.arange(tokens.shape[0], device=s.device), starts, right=True) - 1      # the answer that a row is part of
    inside = of < answers
    of = of.clamp(max=answers - 1)
    member = ((of[None, :] == torch.arange(answers, device=s.device)[:, None]) & (inside & has)[None, :]).double()
    sums = member @ logp.double()
    share = torch.ones(answers, dtype=torch.float64, device=s.device)
    if case["mean"]:
        share = 1 / member.sum(dim=1).clamp(min=1)
        sums = sums * share
    margin = (sums - ref.double()).reshape(-1, 2)
    loss, slope = _pair_loss(case, margin[:, 0] - margin[:, 1])
    if case["mode"] == "loss":
        return loss.float(), sums.float()
    slope = slope * state["dloss"].double()
    slope = (torch.stack([slope, -slope], dim=1).reshape(-1) * share)[of].float()
    return loss.float(), sums.float(), _spread(e, total, at, has & inside, slope, 1.0, s.dtype)


def run(state):
    return {"norm": _run_norm, "dropout": _run_dropout, "logp": _run_logp, "policy": _run_policy,
            "preference": _run_preference}[state["case"]["op"]](state)


def work(case):
    s = SIZE[case["dtype"]]
    train = case["mode"] == "train"
    if case["op"] == "norm":
        M, K, ss = case["M"], case["K"], SIZE[case["stream"]]
        matrix, token = M * K, case["gate"] == "token"
        size = ss + s                                                        # x is read, n written
        if case["branch"]:
            size += ss + s + (s if token else 0)                             # y written, the block's output and a full gate read
        if train:
            size += 2 * ss + s                                               # dy and dn read, dx written
            if case["branch"]:
                size += s + (s if token else 0)                              # the gradients of the block's output and of the gate
        vectors = 1 + case["post"] + (case["gate"] == "channel")
        flops = 6 + (4 if case["branch"] else 0) + (3 if case["post"] else 0)
        if train:
            flops += 10 + (3 if case["branch"] else 0) + (9 if case["post"] else 0)
        return {"bytes": matrix * size + vectors * K * s * (2 if train else 1), "flops": float(flops * matrix)}
    if case["op"] == "dropout":
        passes = 2 if train else 1
        return {"bytes": 2 * passes * case["M"] * case["K"] * s, "flops": float(passes * case["M"] * case["K"])}
    V = case["V"]
    if case["op"] == "preference":
        lengths = _lengths(case)
        N, scored = sum(lengths) + case["behind"], sum(n - n // 4 for n in lengths)
        small = 8 * N + 32 * case["pairs"]
    else:
        N = case["N"]
        scored, small = N - N // 16, {"logp": 12, "policy": 28}[case["op"]] * N
    grad = case["mode"] not in ("forward", "loss")                           # rows without a token have no need of their logits
    return {"bytes": s * V * (scored + (N if grad else 0)) + small, "flops": float((4 + (3 if grad else 0)) * V * scored)}


def _bits(M, K, rng):
    """The generator's 16 bits for every element, with products put together from halves."""
    seed, offset = rng

    def product(a, m):
        """High and low word of a 32-bit number times m."""
        lo, hi = a & 0xFFFF, a >> 16
        low = lo * m                                                         # below 2^48
        high = hi * m + (low >> 16)                                          # the product over 2^16
        return high >> 16, (high & 0xFFFF) << 16 | (low & 0xFFFF)
    words = (K + 7) // 8
    at = torch.arange(M * words, dtype=torch.int64, device=DEVICE)
    x0, x1 = at % words, at // words
    x2, x3 = torch.zeros_like(at) + (offset & 0xFFFFFFFF), torch.zeros_like(at) + (offset >> 32)
    for r in range(7):
        h0, l0 = product(x0, 0xD2511F53)
        h1, l1 = product(x2, 0xCD9E8D57)
        key0, key1 = ((seed & 0xFFFFFFFF) + r * 0x9E3779B9) % (1 << 32), ((seed >> 32) + r * 0xBB67AE85) % (1 << 32)
        x0, x1, x2, x3 = h1 ^ x1 ^ key0, l1, h0 ^ x3 ^ key1, l0
    out = torch.empty((M * words, 8), dtype=torch.int64, device=DEVICE)
    for i, x in enumerate((x0, x1, x2, x3)):
        out[:, 2 * i], out[:, 2 * i + 1] = x % 65536, x // 65536
    return out.reshape(M, words * 8)[:, :K]


def _exact_norm(case, state):
    leaf = {k: state[k].double().requires_grad_(case["mode"] == "train") for k in ("x", "branch", "weight", "post_weight", "gate") if state[k] is not None}

    def normed(v):
        return v * (v.square().sum(dim=1, keepdim=True) / v.shape[1] + 1e-6) ** -0.5
    y = leaf["x"]
    if case["branch"]:
        b = leaf["branch"]
        if case["post"]:
            b = normed(b) * leaf["post_weight"]
        if case["gate"] != "none":
            b = b * leaf["gate"]
        if case["p"] > 0:
            dropped = _bits(case["M"], case["K"], state["rng"]) < _threshold(case["p"])
            b = torch.where(dropped, torch.zeros_like(b), b / (1 - _threshold(case["p"]) / 65536))
        y = y + state["scale"] * b
    n = normed(y) * leaf["weight"]
    out = ([y.detach()] if case["branch"] else []) + [n.detach()]
    if case["mode"] == "forward":
        return tuple(out)
    names = [k for k in ("x", "branch", "weight", "post_weight", "gate") if k in leaf]
    return (*out, *torch.autograd.grad([y, n], [leaf[k] for k in names], [state["dy"].double(), state["dn"].double()]))


def _exact_dropout(case, state):
    kept = _bits(case["M"], case["K"], state["rng"]) >= _threshold(case["p"])
    share = 1 - _threshold(case["p"]) / 65536
    return tuple(state[k].double() / share * kept for k in (("x", "dy") if case["mode"] == "train" else ("x",)))


def _exact_rows(state, temperature, some):
    """The tokens' log-probabilities, and a function for the logits' gradient from every row's dL/dlogp."""
    logits, tokens = state["logits"], state["tokens"]
    N, V = logits.shape
    step = max(1, (1 << 26) // V)
    parts = [slice(r, min(r + step, N)) for r in range(0, N, step)]
    logp = torch.zeros(N, dtype=torch.float64, device=DEVICE)
    for at in parts:
        rows = torch.log_softmax(logits[at].double() / temperature, dim=1)
        logp[at] = torch.where(some[at], rows[torch.arange(rows.shape[0], device=DEVICE), tokens[at].clamp(min=0)], 0.0)

    def gradient(slope):
        out = torch.empty((N, V), dtype=torch.float64, device=DEVICE)
        for at in parts:
            weight = torch.where(some[at], slope[at], 0.0) / temperature
            out[at] = torch.softmax(logits[at].double() / temperature, dim=1) * -weight[:, None]
            out[at, :][torch.arange(weight.shape[0], device=DEVICE), tokens[at].clamp(min=0)] += weight
        return out
    return logp, gradient


def _exact_logp(case, state):
    logp, gradient = _exact_rows(state, case["temperature"], state["tokens"] >= 0)
    return logp if case["mode"] == "forward" else (logp, gradient(state["dloss"].double()))


def _exact_policy(case, state):
    some = state["tokens"] >= 0
    logp, gradient = _exact_rows(state, case["temperature"], some)
    leaf = logp.clone().requires_grad_()
    ratio = torch.exp(leaf - state["old"].double())
    advantage = state["advantage"].double()
    clipped = torch.where(advantage >= 0, torch.clamp(ratio, max=1 + case["high"]), torch.clamp(ratio, min=1 - case["low"]))
    loss = -clipped * advantage
    if state["ref"] is not None:
        gap = state["ref"].double() - leaf
        loss = loss + case["kl"] * (torch.exp(gap) - gap - 1)
    loss = torch.where(some, loss, torch.zeros_like(loss))
    if case["mode"] == "loss":
        return loss.detach(), logp
    (slope,) = torch.autograd.grad(loss, leaf, state["dloss"].double())
    return loss.detach(), logp, gradient(slope)


def _exact_preference(case, state):
    starts = state["starts"].tolist()
    some = state["tokens"] >= 0
    some[starts[-1]:] = False
    logp, gradient = _exact_rows(state, 1.0, some)
    leaf = logp.clone().requires_grad_()
    sums = torch.stack([leaf[a:b].sum() / (max(1, int(some[a:b].sum())) if case["mean"] else 1) for a, b in zip(starts, starts[1:])])
    margin = sums - state["ref"].double()
    h = margin[0::2] - margin[1::2]
    logsigmoid = torch.nn.functional.logsigmoid
    beta, smoothing = case["beta"], case["smoothing"]
    if case["kind"] == "sigmoid":
        loss = -(1 - smoothing) * logsigmoid(beta * h) - smoothing * logsigmoid(-beta * h)
    elif case["kind"] == "hinge":
        loss = torch.relu(1 - beta * h)
    else:
        loss = (h - 1 / (2 * beta)) ** 2
    if case["mode"] == "loss":
        return loss.detach(), sums.detach()
    (slope,) = torch.autograd.grad(loss, leaf, state["dloss"].double())
    return loss.detach(), sums.detach(), gradient(slope)


def exact(case, seed):
    state = prepare(case, seed)
    return {"norm": _exact_norm, "dropout": _exact_dropout, "logp": _exact_logp, "policy": _exact_policy,
            "preference": _exact_preference}[case["op"]](case, state)
