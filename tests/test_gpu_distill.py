"""The distillation loss and its gradient against the definition in 64 bits (needs an MI355X).

Tolerances.  A gradient is rounded once to its type: half a step, ``finfo.eps / 2`` of its size.  Everything before is in 32
bits.  An exponent (s - m) c - log2(sum) is off by at most 2^-22 of the sizes that go into it (two roundings of each, and the
exponential's own), which is the relative error ``rp`` of one p (ln 2 < 1).  Their sum is off by the mean of that, and by 2^-24 for
every addition in a chain of no more than V / 64 + 64.  The same for the teacher's entries.  The terms of a difference keep their own errors."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = [torch.bfloat16, torch.float16, torch.float32]
LOG2E = 1.4426950408889634
STEP = 2.0 ** -22


@pytest.fixture(scope="module")
def tr():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2001_01347_amd import training
    training.load()
    return training


def reference(logits, index, values, T, kl, labels, ce, dloss):
    """Loss and gradient in 64 bits, and how far off each may be."""
    s, t, w = logits.double(), values.double(), dloss.double()
    N, V = s.shape
    K = index.shape[1]
    rows = torch.arange(N, device=s.device)

    def soft(T):
        z = s / T
        m = z.amax(dim=1, keepdim=True)
        m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
        e = torch.exp(z - m)
        total = e.sum(dim=1, keepdim=True)
        logsum = torch.where(total > 0, torch.log(total), torch.zeros_like(total))
        p = e * torch.exp(-logsum)
        size = torch.where(p > 0, (z - m).abs(), torch.zeros_like(z)) * LOG2E + logsum.abs() * LOG2E + 8
        err = STEP * size + STEP * (p * size).sum(dim=1, keepdim=True) + (V / 64 + 64) * 2.0 ** -24
        return p, (z - m) - logsum, err                                      # p, log p, the relative error of p

    p, logp, err = soft(T)
    given = index >= 0
    at = index.clamp(min=0).long()
    x = torch.where(given, t, float("-inf")) / T
    any_entry = (x > float("-inf")).any(dim=1, keepdim=True) if K else torch.zeros((N, 1), dtype=torch.bool, device=s.device)
    if K:
        top = torch.where(any_entry, x.amax(dim=1, keepdim=True), 0.0)
        e = torch.where(any_entry, torch.exp(x - top), 0.0)
        total = e.sum(dim=1, keepdim=True).clamp(min=1e-300)
        q = e / total
        logq = (x - top) - torch.log(total)
        eq = STEP * (torch.where(q > 0, (x - top).abs(), 0.0) * LOG2E + 8) + (K + 64) * 2.0 ** -24
        eq = eq + (q * eq).sum(dim=1, keepdim=True)
        gap = torch.where(q > 1e-37, logq - logp.gather(1, at), 0.0)
        ratio = torch.where(torch.isinf(gap), 0.0, gap)
        loss = kl * T * T * torch.where(q > 1e-37, q * gap, 0.0).sum(dim=1)
        loss_tol = kl * T * T * (q * (err.gather(1, at) + 2 * eq + ratio.abs() * (eq + (K + 16) * 2.0 ** -24))).sum(dim=1)
        spread, spread_tol = torch.zeros_like(s).scatter_add_(1, at, q), torch.zeros_like(s).scatter_add_(1, at, q * eq)
    else:
        loss, loss_tol = torch.zeros(N, dtype=torch.float64, device=s.device), torch.zeros(N, dtype=torch.float64, device=s.device)
        spread, spread_tol = torch.zeros_like(s), torch.zeros_like(s)
    a = torch.where(any_entry, kl * T * w[:, None], torch.zeros_like(w[:, None]))
    grad = a * (p - spread)
    grad_tol = a.abs() * (p * (err + STEP) + spread_tol + spread * STEP)
    if labels is not None:
        has = (labels >= 0) & (ce != 0)
        p1, logp1, err1 = soft(1.0)
        lab = labels.clamp(min=0)
        hot = torch.zeros_like(s)
        hot[rows[has], lab[has]] = 1.0
        nll = -logp1[rows, lab]
        loss = loss + torch.where(has, ce * nll, torch.zeros_like(nll))
        fin = torch.where(torch.isinf(nll), torch.zeros_like(nll), nll)
        loss_tol = loss_tol + torch.where(has, ce * (err1[rows, lab] + 4 * STEP * fin.abs()), torch.zeros_like(nll))
        b = torch.where(has, ce * w, torch.zeros_like(w))[:, None]
        grad = grad + b * (p1 - hot)
        grad_tol = grad_tol + b.abs() * (p1 * (err1 + STEP) + hot * STEP)
    u = torch.finfo(logits.dtype).eps / 2
    tiny = 2.0 ** -25 * (1 + 2 ** -8) if logits.dtype == torch.float16 else 1e-37
    loss_tol = loss_tol + 4 * STEP * torch.where(torch.isinf(loss), torch.zeros_like(loss), loss).abs() + 1e-37
    return loss, loss_tol, grad, grad_tol * (1 + 2 * u) + u * grad.abs() + tiny


def make(N, V, K, dtype, seed=0, index_type=torch.int64, top_type=None, pad=0, padding=True, spread=2.5):
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + N + 31 * V + 1009 * K)

    def rows(values, dt):
        fill = float("nan") if dt.is_floating_point else 0
        full = torch.full((values.shape[0], values.shape[1] + 2 * pad), fill, dtype=dt, device="cuda")
        full[:, pad:pad + values.shape[1]] = values.to(dt)
        return full[:, pad:pad + values.shape[1]]
    logits = rows(torch.randn((N, V), generator=gen, device="cuda") * spread, dtype)
    values, index = torch.topk(logits.float() + torch.randn((N, V), generator=gen, device="cuda"), min(K, V), dim=1)
    if K > V:                                                                # more room than the vocabulary has: padding
        values = torch.cat([values, torch.zeros((N, K - V), device="cuda")], dim=1)
        index = torch.cat([index, torch.full((N, K - V), -1, device="cuda")], dim=1)
    if padding and K:
        index[torch.rand((N, K), generator=gen, device="cuda") < 0.1] = -1
        if N > 2:
            index[N // 2] = -1                                               # a row without any entry
            values[N - 1, :K // 2] = float("-inf")
    labels = torch.randint(0, V, (N,), generator=gen, device="cuda")
    labels[torch.rand((N,), generator=gen, device="cuda") < 0.2] = -100
    dloss = torch.randn((N,), generator=gen, device="cuda")
    return logits, rows(index, index_type), rows(values, top_type or dtype), labels, dloss


def check(tr, logits, index, values, labels, dloss, T, kl, ce):
    args = dict(temperature=T, kl_weight=kl, labels=labels, ce_weight=ce)
    loss, loss_tol, grad, grad_tol = reference(logits, index, values, T, kl, labels, ce, dloss)
    got, stats, status = tr.ebsp_distill_forward(logits, index, values, **args)
    got_grad = tr.ebsp_distill_backward(logits, index, values, stats, dloss, **args)
    both, both_grad, both_status = tr.ebsp_distill_loss_grad(logits, index, values, dloss, **args)
    assert bool((status == 0).all()) and bool((both_status == 0).all())
    for l in (got, both):
        off = (l.double() - loss).abs()
        off = torch.where(torch.isinf(loss) & (l.double() == loss), torch.zeros_like(off), off)
        assert bool((off <= loss_tol).all()), f"loss: {(off / loss_tol).max().item():.3g} times its bound"
    for g in (got_grad, both_grad):
        off = (g.double() - grad).abs()
        assert bool((off <= grad_tol).all()), f"gradient: {(off / grad_tol).max().item():.3g} times its bound"
    return got, got_grad


SHAPES = [(1, 1, 1), (1, 2, 1), (3, 7, 5), (2, 8, 0), (5, 63, 63), (4, 100, 200), (1, 1000, 16), (300, 1000, 64), (7, 4097, 300), (260, 2051, 1000),
          (1, 32003, 16), (33, 50021, 100), (2, 150001, 64), (270, 16390, 8), (257, 33000, 70)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V,K", SHAPES)
def test_shapes(tr, N, V, K, dtype):
    logits, index, values, labels, dloss = make(N, V, K, dtype)
    check(tr, logits, index, values, labels, dloss, 2.0, 0.7, 0.3)
    check(tr, logits, index, values, None, dloss, 1.0, 1.0, 0.0)


@pytest.mark.parametrize("dtype", TYPES)
def test_many_long_rows(tr, dtype):
    """Rows as long as the largest vocabularies, one workgroup each."""
    for V in (128000, 131073, 262147):
        logits, index, values, labels, dloss = make(256, V, 33, dtype, seed=1)
        check(tr, logits, index, values, labels, dloss, 3.0, 1.0, 0.5)
        check(tr, logits, index, values, None, dloss, 2.0, 1.0, 0.0)


@pytest.mark.parametrize("T,kl,ce", [(1.0, 1.0, 0.0), (1.0, 0.5, 0.5), (0.5, 1.0, 0.2), (4.0, 1.0, 1.0), (2.0, 0.0, 1.0), (2.0, 1.0, 0.0), (3.0, 0.0, 0.0),
                                     (100.0, 1.0, 0.1), (0.01, 1.0, 0.1)])
def test_weights_and_temperatures(tr, T, kl, ce):
    for N in (5, 300):
        check(tr, *make(N, 3001, 20, torch.bfloat16, seed=2), T, kl, ce)


@pytest.mark.parametrize("index_type", [torch.int32, torch.int64])
@pytest.mark.parametrize("top_type", TYPES)
def test_types_of_the_entries(tr, index_type, top_type):
    check(tr, *make(9, 5000, 40, torch.bfloat16, seed=3, index_type=index_type, top_type=top_type), 2.0, 1.0, 0.5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad", [1, 8])
def test_rows_apart(tr, dtype, pad):
    for N in (4, 300):
        check(tr, *make(N, 3333, 17, dtype, seed=4, pad=pad), 2.0, 1.0, 0.5)


@pytest.mark.parametrize("N", [4, 300])
def test_entries_of_one_place_add_up(tr, N):
    logits, index, values, labels, dloss = make(N, 500, 64, torch.float32, seed=5, padding=False)
    index[:, 10:20] = index[:, 9:10]
    index[:, 63] = labels.clamp(min=0)
    index[:, 62] = labels.clamp(min=0)
    check(tr, logits, index, values, labels, dloss, 2.0, 1.0, 0.5)


@pytest.mark.parametrize("N,V,K", [(5, 40, 1000), (300, 3000, 300), (130, 20000, 64), (3, 90000, 1024)])
def test_few_and_many_entries_of_one_place(tr, N, V, K):
    """A few indices twice, more than a list of such has room for, all of one; labels at such places."""
    logits, index, values, labels, dloss = make(N, V, K, torch.bfloat16, seed=12, padding=False)
    index[1::3, 5] = index[1::3, 17]
    index[2::3, :K // 2] = index[2::3, K - K // 2:]
    index[0] = index[0, 3]
    labels = torch.where(torch.arange(N, device="cuda") % 2 == 0, index[:, 5].long().clamp(min=-1), labels)
    check(tr, logits, index, values, labels, dloss, 2.0, 0.75, 0.5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V", [(140, 1), (140, 4099), (140, 8200), (140, 33000), (520, 33001), (140, 70003), (100, 140001)])
def test_rows_of_every_workgroup(tr, N, V, dtype):
    check(tr, *make(N, V, min(V, 20), dtype, seed=13), 1.5, 0.75, 0.5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [4, 300])
def test_masked_places(tr, dtype, N):
    """Places masked with -inf or with the type's lowest value, outside the entries; a row of which one place is left; rows of one value."""
    for mask in (float("-inf"), torch.finfo(dtype).min):
        logits, index, values, labels, dloss = make(N, 2000, 16, dtype, seed=6)
        hit = torch.rand((N, 2000), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)) < 0.5
        hit.scatter_(1, index.clamp(min=0), False)
        hit[torch.arange(N, device="cuda"), labels.clamp(min=0)] = False
        logits[hit] = mask
        logits[0] = mask
        logits[0, 77] = 1.5
        index[0] = -1
        index[0, 3] = 77
        labels[0] = 77
        logits[1] = 3.0
        check(tr, logits, index, values, labels, dloss, 2.0, 1.0, 0.5)
    lowest = torch.full((N, 300), torch.finfo(dtype).min, dtype=dtype, device="cuda")      # nothing but the lowest value: p = 1 / V
    index = torch.arange(8, device="cuda").repeat(N, 1)
    loss, grad, _ = tr.ebsp_distill_loss_grad(lowest, index, torch.zeros((N, 8), dtype=dtype, device="cuda"), torch.ones(N, device="cuda"))
    want = -1 / 8 + 1 / 300
    assert torch.allclose(loss, torch.full_like(loss, torch.log(torch.tensor(300 / 8)).item()), rtol=1e-5)
    assert torch.allclose(grad[:, :8].float(), torch.full((N, 8), want, device="cuda"), rtol=2 ** -7)
    assert torch.allclose(grad[:, 8:].float(), torch.full((N, 292), 1 / 300, device="cuda"), rtol=2 ** -7)


@pytest.mark.parametrize("N", [3, 300])
def test_weight_on_a_masked_place(tr, N):
    """The teacher wants what the mask forbids: the loss is +inf, the gradient finite; a row without any place left likewise."""
    logits, index, values, labels, dloss = make(N, 100, 4, torch.float32, seed=7, padding=False)
    dloss[:] = 1.0
    logits[0, index[0, 1]] = float("-inf")
    logits[1] = float("-inf")
    loss, grad, _ = tr.ebsp_distill_loss_grad(logits, index, values, dloss)
    assert torch.isinf(loss[:2]).all() and (loss[:2] > 0).all() and torch.isfinite(loss[2:]).all()
    assert torch.isfinite(grad).all()
    assert bool((grad[1][index[1]] < 0).all()) and grad[1].sum().item() == pytest.approx(-1.0, rel=1e-5)
    index[1] = -1                                                            # nor entries: nothing at all
    loss, grad, _ = tr.ebsp_distill_loss_grad(logits, index, values, dloss)
    assert loss[1].item() == 0 and bool((grad[1] == 0).all())


@pytest.mark.parametrize("N", [6, 300])
def test_not_finite_stays_in_its_row(tr, N):
    logits, index, values, labels, dloss = make(N, 700, 12, torch.bfloat16, seed=8, padding=False)
    clean = tr.ebsp_distill_loss_grad(logits, index, values, dloss, 2.0, 1.0, labels, 0.5)
    logits[1, 40] = float("nan")
    logits[2, 41] = float("inf")
    values[3, 5] = float("nan")
    loss, grad, _ = tr.ebsp_distill_loss_grad(logits, index, values, dloss, 2.0, 1.0, labels, 0.5)
    assert torch.isnan(loss[1:4]).all()
    keep = torch.ones(N, dtype=torch.bool, device="cuda")
    keep[1:4] = False
    assert torch.equal(loss[keep], clean[0][keep]) and torch.equal(grad[keep], clean[1][keep])


@pytest.mark.parametrize("N", [4, 300])
def test_places_beyond_the_vocabulary_are_flagged(tr, N):
    logits, index, values, labels, dloss = make(N, 600, 12, torch.float16, seed=9, padding=False)
    labels[:] = 5
    kept, kept_labels = index.clone(), labels.clone()
    index[0, 3], kept[0, 3] = 600, -1
    index[1, 0], kept[1, 0] = 1 << 40, -1
    labels[2], kept_labels[2] = 600, -1
    index[3, 2], kept[3, 2] = -(1 << 40), -1                                 # padding, whatever the number
    want = tr.ebsp_distill_loss_grad(logits, kept, values, dloss, 2.0, 1.0, kept_labels, 0.5)
    loss, grad, status = tr.ebsp_distill_loss_grad(logits, index, values, dloss, 2.0, 1.0, labels, 0.5)
    assert status[:4].tolist() == [4, 4, 4, 0] and bool((status[4:] == 0).all())
    assert torch.equal(loss, want[0]) and torch.equal(grad, want[1])
    loss, stats, status = tr.ebsp_distill_forward(logits, index, values, 2.0, 1.0, labels, 0.5)
    assert status[:4].tolist() == [4, 4, 4, 0]
    assert torch.equal(tr.ebsp_distill_backward(logits, index, values, stats, dloss, 2.0, 1.0, labels, 0.5).isnan(), grad.isnan())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V", [(3, 40000), (300, 5000), (256, 70001)])
def test_in_place(tr, N, V, dtype):
    for pad in (0, 3):
        logits, index, values, labels, dloss = make(N, V, 50, dtype, seed=10, pad=pad)
        args = dict(temperature=2.0, kl_weight=1.0, labels=labels, ce_weight=0.5)
        want_loss, want, _ = tr.ebsp_distill_loss_grad(logits, index, values, dloss, **args)
        loss, stats, _ = tr.ebsp_distill_forward(logits, index, values, **args)
        want2 = tr.ebsp_distill_backward(logits, index, values, stats, dloss, **args)
        mine = logits.clone() if pad == 0 else torch.zeros((N, V + 2 * pad), dtype=dtype, device="cuda")[:, pad:pad + V].copy_(logits)
        got_loss, got, _ = tr.ebsp_distill_loss_grad(mine, index, values, dloss, dlogits=mine, **args)
        assert got is mine and torch.equal(got, want) and torch.equal(got_loss, want_loss)
        mine.copy_(logits)
        assert torch.equal(tr.ebsp_distill_backward(mine, index, values, stats, dloss, dlogits=mine, **args), want2)


def test_rows_far_apart(tr):
    """Rows whose offsets pass 32 bits."""
    N, V, ld = 20, 1000, 1 << 28
    logits0, index, values, labels, dloss = make(N, V, 9, torch.bfloat16, seed=11)
    base = torch.empty(N * ld, dtype=torch.bfloat16, device="cuda")
    logits = base.view(N, ld)[:, :V]
    logits.copy_(logits0)
    check(tr, logits, index, values, labels, dloss, 2.0, 1.0, 0.5)


def test_differences(tr):
    """The gradient along a direction against differences of the 64-bit loss."""
    logits, index, values, labels, dloss = make(6, 400, 20, torch.float32, seed=12)
    T, kl, ce = 2.0, 0.8, 0.4
    _, _, _, tol = reference(logits, index, values, T, kl, labels, ce, dloss)
    _, grad, _ = tr.ebsp_distill_loss_grad(logits, index, values, dloss, T, kl, labels, ce)
    d = torch.randn((6, 400), device="cuda", dtype=torch.float64)

    def total(step):
        s = logits.double() + step * d
        q = torch.softmax(torch.where(index >= 0, values.double(), float("-inf")) / T, dim=1)
        lp = torch.log_softmax(s / T, dim=1).gather(1, index.clamp(min=0))
        first = torch.where((index >= 0) & (q > 0), q * (torch.log(q) - lp), 0.0).nansum(dim=1)
        nll = -torch.log_softmax(s, dim=1).gather(1, labels.clamp(min=0)[:, None])[:, 0]
        return ((kl * T * T * first + ce * torch.where(labels >= 0, nll, 0.0)) * dloss.double()).sum()
    eps = 1e-5
    slope = (total(eps) - total(-eps)) / (2 * eps)
    assert ((grad.double() * d).sum() - slope).abs().item() <= (tol * d.abs()).sum().item() + 1e-6 * abs(slope.item())


def test_autograd(tr):
    logits, index, values, labels, _ = make(12, 500, 10, torch.float32, seed=13)
    leaf = logits.reshape(3, 4, 500).clone().requires_grad_()
    loss = tr.distill_loss(leaf, index.reshape(3, 4, 10), values.reshape(3, 4, 10), 2.0, 0.7, labels.reshape(3, 4), 0.3)
    assert tuple(loss.shape) == (3, 4)
    loss.mean().backward()
    want_loss, loss_tol, want, tol = reference(logits, index, values, 2.0, 0.7, labels, 0.3, torch.full((12,), 1 / 12, device="cuda"))
    assert bool(((loss.detach().reshape(12).double() - want_loss).abs() <= loss_tol).all())
    assert bool(((leaf.grad.reshape(12, 500).double() - want).abs() <= tol).all())


@pytest.mark.parametrize("N,V", [(3, 40000), (300, 2000)])
def test_streams_and_graphs(tr, N, V):
    logits, index, values, labels, dloss = make(N, V, 20, torch.bfloat16, seed=14)

    def step():
        args = dict(temperature=2.0, kl_weight=1.0, labels=labels, ce_weight=0.5)
        loss, grad, status = tr.ebsp_distill_loss_grad(logits, index, values, dloss, **args)
        l2, stats, _ = tr.ebsp_distill_forward(logits, index, values, **args)
        return loss, grad, l2, tr.ebsp_distill_backward(logits, index, values, stats, dloss, **args)
    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in (20, 21, 22):
        for t, new in zip((logits, index, values, labels, dloss), make(N, V, 20, torch.bfloat16, seed=seed)):
            t.copy_(new)
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_no_rows(tr):
    logits, index = torch.empty((0, 10), device="cuda"), torch.empty((0, 3), dtype=torch.int64, device="cuda")
    loss, grad, status = tr.ebsp_distill_loss_grad(logits, index, torch.empty((0, 3), device="cuda"), torch.empty(0, device="cuda"))
    assert loss.shape == (0,) and grad.shape == (0, 10) and status.shape == (0,)


def test_binding_refuses(tr):
    logits, index, values, labels, dloss = make(6, 50, 4, torch.bfloat16)
    good = dict(logits=logits, top_index=index, top_logit=values)
    for bad in (dict(logits=logits.double()), dict(logits=logits[0]), dict(logits=logits.cpu()), dict(logits=logits[:5]), dict(logits=logits.t()),
                dict(logits=logits[:1].expand(6, 50)), dict(logits=logits[:, :0]), dict(top_index=index.short()), dict(top_index=index[:, :3]),
                dict(top_index=index[0]), dict(top_logit=values[:4]), dict(top_logit=values.double()), dict(labels=labels.int()),
                dict(labels=labels[:3]), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")),
                dict(temperature=float("inf")), dict(loss=torch.empty(5, device="cuda")), dict(stats=torch.empty((6, 2), device="cuda")),
                dict(top_index=torch.zeros((6, 1025), dtype=torch.int64, device="cuda"), top_logit=torch.zeros((6, 1025), device="cuda"))):
        with pytest.raises(ValueError):
            tr.ebsp_distill_forward(**{**good, **bad})
    for bad in (dict(dloss=dloss.double()), dict(dloss=dloss[:3]), dict(dlogits=logits.float()), dict(dlogits=logits[:, :49])):
        with pytest.raises(ValueError):
            tr.ebsp_distill_loss_grad(**{**good, "dloss": dloss, **bad})
    long = make(2, 40000, 4, torch.bfloat16)
    with pytest.raises(ValueError):
        tr.ebsp_distill_forward(*long[:3], workspace=torch.empty(256, dtype=torch.uint8, device="cuda")[:128])
