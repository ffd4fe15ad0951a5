"""The operators of tuning together, as a worker uses them: blocks on a residual stream, a policy or preference loss on their logits (needs an MI355X).

Everything is in float32 here, so results agree with 64 bits up to the sums' rounding: a few hundred additions a result at most, 2^-24 each, over four steps."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import philox  # noqa: E402

K, F, V, N = 64, 96, 160, 24
EPS = 1e-6


@pytest.fixture(scope="module")
def tr():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2001_01347_amd import training
    training.load()
    return training


def weights(seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def draw(*shape):
        return torch.randn(shape, generator=gen, device="cuda") * shape[-1] ** -0.5
    return {"embed": draw(V, K) * 8, "w0": 1 + 0.1 * draw(K), "wg": draw(F, K), "wu": draw(F, K), "wd": draw(K, F), "post": 1 + 0.1 * draw(K),
            "gate": draw(K) * 4, "w1": 1 + 0.1 * draw(K), "out": draw(V, K)}


def model(tr, w, tokens, rng):
    x, n = tr.residual_norm(w["embed"][tokens], None, w["w0"])
    h = tr.dropout(tr.gated_ff(n, w["wg"], w["wu"]), 0.1, (rng[0], rng[1] + 1))
    x, n = tr.residual_norm(x, h @ w["wd"].t(), w["w1"], w["post"], w["gate"], 0.5, 0.2, rng)
    return n @ w["out"].t()


def model64(w, tokens, rng):
    def normed(v):
        return v * (v.square().mean(dim=1, keepdim=True) + EPS) ** -0.5

    def drop(v, p, offset):
        keep = torch.from_numpy(philox.keep(*v.shape, p, rng[0], offset)).cuda()
        return torch.where(keep, v * philox.kept_factor(p), torch.zeros_like(v))
    x = w["embed"][tokens]
    n = normed(x) * w["w0"]
    h = drop(torch.nn.functional.silu(n @ w["wg"].t()) * (n @ w["wu"].t()), 0.1, rng[1] + 1)
    x = x + 0.5 * drop(normed(h @ w["wd"].t()) * w["post"] * w["gate"], 0.2, rng[1])
    return normed(x) * w["w1"] @ w["out"].t()


def grads(loss, w):
    return dict(zip(w, torch.autograd.grad(loss, list(w.values()))))


def compare(got, want):
    for k in got:
        off = (got[k].double() - want[k]).abs().max()
        assert off <= 2e-5 * want[k].abs().max(), (k, off.item(), want[k].abs().max().item())


def inputs():
    gen = torch.Generator(device="cuda").manual_seed(5)
    prompt, tokens = (torch.randint(0, V, (N,), generator=gen, device="cuda") for _ in range(2))
    tokens[3] = -100
    return prompt, tokens, torch.randn(N, generator=gen, device="cuda")


def test_policy_step_of_a_block(tr):
    prompt, tokens, advantage = inputs()
    rng = (99, 12)
    w = {k: v.requires_grad_() for k, v in weights().items()}
    with torch.no_grad():
        old = tr.token_logp(model(tr, w, prompt, rng), tokens) + 0.03
        other = old - 0.1
    loss = tr.policy_loss(model(tr, w, prompt, rng), tokens, old, advantage, ref_logp=other, kl_weight=0.1)
    got = grads(loss.mean(), w)
    w64 = {k: v.detach().double().requires_grad_() for k, v in w.items()}
    logp = torch.log_softmax(model64(w64, prompt, rng), dim=1).gather(1, tokens.clamp(min=0)[:, None])[:, 0]
    x, g = torch.exp(logp - old.double()), other.double() - logp
    want = -torch.minimum(x * advantage, x.clamp(0.8, 1.2) * advantage) + 0.1 * (torch.exp(g) - g - 1)
    want = torch.where(tokens >= 0, want, 0.0)
    assert torch.allclose(loss.detach().double(), want.detach(), rtol=1e-4, atol=1e-5)
    compare(got, grads(want.mean(), w64))


def test_preference_step_of_a_block(tr):
    prompt, tokens, _ = inputs()
    starts, rng = torch.tensor([0, 5, 12, 18, 24], device="cuda"), (3, 4)
    w = {k: v.requires_grad_() for k, v in weights(1).items()}
    loss = tr.preference_loss(model(tr, w, prompt, rng), tokens, starts, beta=0.5, smoothing=0.1)
    got = grads(loss.mean(), w)
    w64 = {k: v.detach().double().requires_grad_() for k, v in w.items()}
    logp = torch.log_softmax(model64(w64, prompt, rng), dim=1).gather(1, tokens.clamp(min=0)[:, None])[:, 0]
    logp = torch.where(tokens >= 0, logp, 0.0)
    sums = [logp[a:b].sum() for a, b in ((0, 5), (5, 12), (12, 18), (18, 24))]
    h = 0.5 * torch.stack([sums[0] - sums[1], sums[2] - sums[3]])
    want = -0.9 * torch.nn.functional.logsigmoid(h) - 0.1 * torch.nn.functional.logsigmoid(-h)
    assert torch.allclose(loss.detach().double(), want.detach(), rtol=1e-4, atol=1e-5)
    compare(got, grads(want.mean(), w64))


def test_replayed_step_is_the_eager_one(tr):
    """Forward and backward pass of a step in one graph, its place in the random numbers on the device; every replay against the same step run eagerly."""
    prompt, tokens, advantage = inputs()
    w = {k: v.requires_grad_() for k, v in weights(2).items()}
    place = torch.tensor([8, 50], dtype=torch.int64, device="cuda")
    old = torch.full((N,), -5.0, device="cuda")

    def step():
        x, n = tr.residual_norm(w["embed"][prompt], None, w["w0"])
        h = tr.gated_ff(n, w["wg"], w["wu"])
        x, n = tr.residual_norm(x, h @ w["wd"].t(), w["w1"], w["post"], w["gate"], 0.5, 0.2, place)
        loss = tr.policy_loss(n @ w["out"].t(), tokens, old, advantage)
        return [loss.detach(), *torch.autograd.grad(loss, [w[k] for k in ("w0", "wg", "post", "gate", "w1", "out")], torch.ones_like(loss))]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        out = step()
    for i in range(4):
        place[1] = 50 + 3 * i
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in out]
        eager = step()
        torch.cuda.synchronize()
        for a, b in zip(replayed, eager):
            assert torch.equal(a, b), i


def test_two_graphs_and_two_streams(tr):
    """Calls on two streams at once, and two captured graphs replayed one after the other, each with workspaces of its own, give what they give alone."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    cases = []
    for n, v in ((3, 60000), (2, 90000)):
        logits = torch.randn((n, v), generator=gen, device="cuda").to(torch.bfloat16)
        cases.append((logits, torch.randint(0, v, (n,), generator=gen, device="cuda"), torch.full((n,), -9.0, device="cuda"),
                      torch.randn(n, generator=gen, device="cuda"), torch.ones(n, device="cuda")))
    want = [tr.ebsp_policy_loss_grad(*c)[:3] for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [None, None]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = tr.ebsp_policy_loss_grad(*cases[i])[:3]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i in range(2) for a, b in zip(got[i], want[i]))
    graphs, outs = [], []
    for c in cases:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(tr.ebsp_policy_loss_grad(*c)[:3])
        graphs.append(graph)
    for _ in range(3):
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for i in range(2) for a, b in zip(outs[i], want[i]))
        tr.ebsp_policy_loss_grad(*cases[0])
        torch.cuda.synchronize()


def test_preference_loss_in_a_graph_with_new_inputs(tr):
    """A captured call, replayed on other logits, tokens, starts and weights in the same places."""
    gen = torch.Generator(device="cuda").manual_seed(10)
    n, v = 40, 5000
    logits, tokens = torch.zeros((n, v), device="cuda", dtype=torch.bfloat16), torch.zeros(n, dtype=torch.int64, device="cuda")
    starts, weight = torch.zeros(5, dtype=torch.int64, device="cuda"), torch.zeros(2, device="cuda")

    def call():
        loss, sums, saved, status = tr.ebsp_preference_forward(logits, tokens, starts, beta=0.2)
        both = tr.ebsp_preference_loss_grad(logits, tokens, starts, weight, beta=0.2)
        return [loss, sums, status, tr.ebsp_preference_backward(logits, tokens, starts, saved, weight), *both]
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for at in ([0, 10, 20, 30, 40], [5, 5, 17, 30, 31], [0, 40, 40, 40, 40], [0, 10, 5, 30, 41]):
        logits.copy_(torch.randn((n, v), generator=gen, device="cuda"))
        tokens.copy_(torch.randint(-5, v, (n,), generator=gen, device="cuda"))
        starts.copy_(torch.tensor(at, device="cuda"))
        weight.copy_(torch.randn(2, generator=gen, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, call()):
            assert torch.equal(a, b), at
        torch.cuda.synchronize()
        assert torch.equal(out[0], out[4]) and torch.equal(out[3], out[5])   # one call and two


def test_without_gradients_and_forward_mode(tr):
    """No graph where gradients are off, by either way; tangents are refused by the losses too; one tensor in two places; a stream that is changed under a graph."""
    import torch.autograd.forward_ad as forward_ad
    x, w = torch.randn((4, 64), device="cuda", requires_grad=True), torch.ones(64, device="cuda", requires_grad=True)
    tokens, f, starts = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(4, device="cuda"), torch.tensor([0, 2, 4], device="cuda")
    calls = [lambda v: tr.token_logp(v, tokens), lambda v: tr.policy_loss(v, tokens, f, f), lambda v: tr.preference_loss(v, tokens, starts)]
    for mode in (torch.no_grad, torch.inference_mode):
        with mode():
            outs = [*tr.residual_norm(x, x, w), tr.residual_norm(x, None, w)[1], tr.dropout(x, 0.5, (1, 2)), *(c(x) for c in calls)]
            assert not any(t.requires_grad for t in outs)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x.detach(), torch.ones_like(x))
        for c in calls:
            with pytest.raises(NotImplementedError):
                c(dual)
    one, two = x.detach().clone().requires_grad_(), x.detach().clone().requires_grad_()
    for a, b in ((x, x), (one, two)):
        y, n = tr.residual_norm(a, b, w)
        (y.sum() + n.square().sum()).backward()
    assert torch.allclose(x.grad, one.grad + two.grad, rtol=1e-6, atol=1e-6)
    y, n = tr.residual_norm(x, x, w)
    y.mul_(2)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        n.sum().backward()
