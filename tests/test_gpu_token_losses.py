"""Log-probabilities of tokens, the clipped policy loss and the preference loss, with their gradients, against the definitions in 64 bits (needs an MI355X).

Tolerances.  An exponent (s - m) c - log2(sum) is off by at most 2^-22 of the sizes that go into it (two roundings of each, and the exponential's own), which is
the relative error ``rp`` of one p (ln 2 < 1); their sum is off by the mean of that, and by 2^-24 for every addition in a chain of no more than V / 64 + 64.  A logp is
off by what its two terms are, each of three roundings, and by its sum.  The ratio e^(logp - old) is off by that error of logp and four roundings, and every loss by
its slope times the error of logp beside its own roundings.  A gradient is rounded once to its type: half a step of its size."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = [torch.bfloat16, torch.float16, torch.float32]
LOG2E = 1.4426950408889634
STEP = 2.0 ** -22
U = 2.0 ** -24
SIZES = [(1, 1), (1, 7), (2, 9), (5, 100), (300, 257), (3, 1001), (128, 4099), (1, 32000), (3, 40000), (97, 40001), (130, 70003), (7, 131072), (100, 131080), (2, 260007),
         (1030, 33), (1029, 500), (1030, 2000), (1026, 4095), (1025, 8190), (1027, 18000), (400, 8190), (200, 16001)]


@pytest.fixture(scope="module")
def tr():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2001_01347_amd import training
    training.load()
    return training


def make(N, V, dtype, seed=0, pad=0, masked=0, spread=2.5):
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + N + 31 * V)
    full = torch.full((N, V + 2 * pad), float("nan"), dtype=dtype, device="cuda")
    logits = full[:, pad:pad + V]
    logits.copy_((torch.randn((N, V), generator=gen, device="cuda") * spread).to(dtype))
    tokens = torch.randint(0, V - masked, (N,), generator=gen, device="cuda")
    if masked:
        logits[:, V - masked:] = float("-inf")
    if N > 2:
        tokens[N // 2] = -100
    return logits, tokens, gen


class Reference:
    """p, logp and their errors for every row that has a token."""

    def __init__(self, logits, tokens, T, some=None):
        self.logits, self.T = logits, T
        self.has = ((tokens >= 0) & (tokens < logits.shape[1])) if some is None else some
        self.at = torch.where(self.has, tokens, torch.zeros_like(tokens))
        s = logits.double() / T
        V = s.shape[1]
        m = s.amax(dim=1, keepdim=True)
        m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
        z = s - m
        e = torch.exp(z)
        total = e.sum(dim=1, keepdim=True)
        logsum = torch.where(total > 0, torch.log(total), torch.zeros_like(total))
        self.p = e * torch.exp(-logsum)
        size = torch.where(self.p > 0, z.abs(), torch.zeros_like(z)) * LOG2E + logsum.abs() * LOG2E + 8
        esum = STEP * (self.p * size).sum(dim=1, keepdim=True) + (V / 64 + 64) * U
        self.rp = STEP * size + esum
        zt = z.gather(1, self.at[:, None])
        none = torch.zeros((), dtype=torch.float64, device="cuda")
        self.logp = torch.where(self.has, (zt - logsum)[:, 0], none)
        finite = torch.where(torch.isinf(zt), torch.zeros_like(zt), zt)
        self.elogp = torch.where(self.has, (esum + (finite.abs() + logsum.abs() + (finite - logsum).abs()) * 3 * U)[:, 0], none)

    def gradient(self, slope, eslope):
        """From every row's dL/dlogp and its error: the logits' gradient and its tolerance."""
        c, ec = torch.where(self.has, slope / self.T, 0.0)[:, None], torch.where(self.has, eslope / self.T, 0.0)[:, None]
        hot = torch.zeros_like(self.p).scatter_(1, self.at[:, None], 1.0)
        grad = c * (hot - self.p)
        tol = ec * (hot - self.p).abs() + c.abs() * (self.p * (self.rp + 4 * U) + hot * 4 * U)
        half = torch.finfo(self.logits.dtype).eps / 2
        tiny = torch.finfo(self.logits.dtype).smallest_normal * half
        return grad, tol * (1 + 2 * half) + half * grad.abs() + tiny * (1 + half) + (1e-37 if self.logits.dtype == torch.float32 else 0)


def close(got, want, tol, what):
    same = got.double() == want                                              # infinities
    off = torch.where(same, torch.zeros_like(want), (got.double() - want).abs())
    assert bool((off <= tol).all()), (what, (off - tol).max().item(), off.max().item())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V", SIZES)
def test_logp_and_its_gradient(tr, N, V, dtype):
    for T, pad in ((1.0, 0), (0.7, 3)):
        logits, tokens, gen = make(N, V, dtype, pad=pad, masked=V // 10)
        dlogp = torch.randn(N, generator=gen, device="cuda")
        ref = Reference(logits, tokens, T)
        logp, stats, status = tr.ebsp_token_logp(logits, tokens, T)
        close(logp, ref.logp, ref.elogp + 1e-37, "logp")
        assert bool((status == 0).all())
        grad, tol = ref.gradient(dlogp.double(), dlogp.double().abs() * 2 * U)
        close(tr.ebsp_token_logp_backward(logits, tokens, stats, dlogp, T), grad, tol, "gradient")
        place = tr.ebsp_token_logp_backward(logits, tokens, stats, dlogp, T, dlogits=logits)
        assert place is logits
        close(place, grad, tol, "in place")


def policy(ref, old, advantage, low, high, kl, other):
    """Loss and slope over logp in 64 bits, and their errors; ratios are kept away from the borders."""
    x = torch.exp(ref.logp - old.double())
    ex = x * (ref.elogp + (ref.logp.abs() + old.double().abs()) * U + 8 * U)
    a = advantage.double()
    cut = x.clamp(1 - low, 1 + high)
    first = x * a <= cut * a
    loss = -torch.minimum(x * a, cut * a)
    eloss = torch.where(first, ex, cut * 2 * U) * a.abs() + loss.abs() * 2 * U
    slope, eslope = torch.where(first, -x * a, 0.0), torch.where(first, ex * a.abs() + (x * a).abs() * 2 * U, 0.0)
    if other is not None and kl != 0:
        g = other.double() - ref.logp
        up = torch.expm1(g)
        term = up - g
        eg = ref.elogp + g.abs() * 2 * U
        eloss = eloss + abs(kl) * (up.abs() * eg + (up.abs() + g.abs()) * 6 * U) + (loss.abs() + abs(kl) * term) * 2 * U
        loss = loss + kl * term
        eslope = eslope + abs(kl) * ((up + 1) * eg + up.abs() * 6 * U) + (slope.abs() + abs(kl) * up.abs()) * 2 * U
        slope = slope - kl * up
    zero = torch.zeros_like(loss)
    return [torch.where(ref.has, t, zero) for t in (loss, eloss, slope, eslope)]


def policy_inputs(ref, gen, low, high):
    N = ref.logp.shape[0]
    moved = 0.25 * torch.randn(N, generator=gen, device="cuda", dtype=torch.float64)
    for border in (math.log(1 - low) if low < 1 else -60.0, math.log(1 + high)):
        moved = torch.where((moved - border).abs() < 1e-2, moved + 0.03, moved)
    logp = torch.where(torch.isinf(ref.logp), torch.zeros_like(ref.logp), ref.logp)
    other = logp + 0.3 * torch.randn(N, generator=gen, device="cuda", dtype=torch.float64)
    other[::5] = logp[::5] + 1e-3                                            # nearly the same: the KL term by its series
    return (logp - moved).float(), torch.randn(N, generator=gen, device="cuda"), other.float(), torch.randn(N, generator=gen, device="cuda")


def check_policy(tr, logits, tokens, old, advantage, other, dloss, T, low, high, kl):
    ref = Reference(logits, tokens, T)
    args = dict(temperature=T, clip_low=low, clip_high=high, ref_logp=other, kl_weight=kl)
    want, tol, slope, eslope = policy(ref, old, advantage, low, high, kl, other)
    loss, logp, stats, status = tr.ebsp_policy_forward(logits, tokens, old, advantage, **args)
    close(loss, want, tol + 1e-37, "loss")
    close(logp, ref.logp, ref.elogp + 1e-37, "logp")
    w = dloss.double()
    grad, gtol = ref.gradient(slope * w, (eslope + slope.abs() * 3 * U) * w.abs())
    close(tr.ebsp_policy_backward(logits, tokens, old, advantage, stats, dloss, **args), grad, gtol, "gradient")
    both, both_grad, both_logp, both_status = tr.ebsp_policy_loss_grad(logits, tokens, old, advantage, dloss, **args)
    close(both, want, tol + 1e-37, "loss of both")
    close(both_logp, ref.logp, ref.elogp + 1e-37, "logp of both")
    close(both_grad, grad, gtol, "gradient of both")
    assert bool((status == 0).all()) and bool((both_status == 0).all())
    copy = logits.clone()
    assert tr.ebsp_policy_loss_grad(copy, tokens, old, advantage, dloss, dlogits=copy, **args)[1] is copy
    assert torch.equal(copy, both_grad)
    return both, both_grad


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V", SIZES)
def test_policy_loss_and_its_gradient(tr, N, V, dtype):
    for T, low, high, kl, pad in ((1.0, 0.2, 0.28, 0.05, 0), (0.8, 0.1, 0.2, 0.0, 3)):
        logits, tokens, gen = make(N, V, dtype, seed=1, pad=pad, masked=V // 10)
        old, advantage, other, dloss = policy_inputs(Reference(logits, tokens, T), gen, low, high)
        check_policy(tr, logits, tokens, old, advantage, other if kl else None, dloss, T, low, high, kl)


def test_policy_without_borders_and_with_none_left(tr):
    logits, tokens, gen = make(200, 1000, torch.float32, seed=2)
    ref = Reference(logits, tokens, 1.0)
    inf = float("inf")
    for low, high in ((inf, inf), (1.0, 3.0), (0.0, 0.0)):
        old, advantage, other, dloss = policy_inputs(ref, gen, min(low, 1.0), min(high, 50.0))
        if low == inf:                                                       # the plain gradient of policies, nothing clipped
            want = -torch.exp(ref.logp - old.double()) * advantage.double()
            loss = tr.ebsp_policy_forward(logits, tokens, old, advantage, clip_low=low, clip_high=high)[0]
            tol = (ref.elogp + (ref.logp.abs() + old.abs()) * U + 12 * U) * want.abs() + 1e-37
            close(loss, torch.where(ref.has, want, 0.0), tol, "loss")
        else:
            check_policy(tr, logits, tokens, old, advantage, other, dloss, 1.0, low, high, 0.1)


def test_zero_weight_leaves_zeros_whatever_the_logits(tr):
    logits, tokens, gen = make(4, 3000, torch.bfloat16, seed=3)
    old, advantage = torch.zeros(4, device="cuda"), torch.ones(4, device="cuda")
    grad = tr.ebsp_policy_loss_grad(logits, tokens, old, advantage, torch.zeros(4, device="cuda"))[1]
    assert bool((grad == 0).all())


@pytest.mark.parametrize("N", [3, 300])
@pytest.mark.parametrize("V", [50, 40000])
def test_rows_without_a_token_are_not_read(tr, N, V):
    """Their logits, old_logp and advantage may be anything; tokens beyond the vocabulary are flagged and count as none."""
    for dtype in TYPES:
        logits, tokens, gen = make(N, V, dtype, seed=4)
        tokens[0], tokens[1], tokens[2] = -1, V, 1 << 40
        logits[:3] = float("nan")
        some = (tokens >= 0) & (tokens < V)
        old, advantage, other = (torch.where(some, torch.randn(N, generator=gen, device="cuda"), float("nan")) for _ in range(3))
        flags = torch.where(tokens >= V, 4, 0).int()
        logp, stats, status = tr.ebsp_token_logp(logits, tokens)
        assert torch.equal(status, flags) and bool((logp[~some] == 0).all()) and bool(torch.isfinite(logp).all())
        one = torch.ones(N, device="cuda")
        grad = tr.ebsp_token_logp_backward(logits, tokens, stats, one)
        assert bool((grad[~some] == 0).all()) and bool(torch.isfinite(grad).all())
        args = dict(ref_logp=other, kl_weight=0.1)
        loss, grad, logp, status = tr.ebsp_policy_loss_grad(logits, tokens, old, advantage, one, **args)
        assert torch.equal(status, flags) and bool((loss[~some] == 0).all()) and bool((grad[~some] == 0).all())
        # with logp down to -16 and ref near 0 the KL term's slope, 0.1 e^(ref - logp), passes 65504 from ref - logp = 13.4 on: infinite in fp16
        assert not bool(torch.isnan(grad[some]).any()) and (dtype == torch.float16 or bool(torch.isfinite(grad[some]).all()))
        loss, logp, stats, status = tr.ebsp_policy_forward(logits, tokens, old, advantage, **args)
        assert torch.equal(status, flags) and bool((loss[~some] == 0).all()) and bool((logp[~some] == 0).all())
        assert bool((tr.ebsp_policy_backward(logits, tokens, old, advantage, stats, one, **args)[~some] == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V", [(4, 500), (4, 50000), (200, 500)])
def test_masked_places(tr, N, V, dtype):
    """Places of the lowest value, a token at one, a token masked with -inf, a row masked throughout, and one that is no number."""
    logits, tokens, gen = make(N, V, dtype, seed=5)
    low = torch.finfo(dtype).min
    tokens[:] = 5
    logits[0, 20:] = low
    logits[1] = low                                                          # equal places: logp is -log V
    logits[2, 5] = float("-inf")
    logits[3] = float("-inf")
    logp, stats, _ = tr.ebsp_token_logp(logits, tokens)
    ref = Reference(logits, tokens, 1.0)
    rows = [i for i in range(N) if i != 3]
    close(logp[rows], ref.logp[rows], ref.elogp[rows] + 1e-37, "logp")
    assert abs(logp[1].item() + math.log(V)) < 1e-5 and logp[2].item() == logp[3].item() == float("-inf")
    one = torch.ones(N, device="cuda")
    grad = tr.ebsp_token_logp_backward(logits, tokens, stats, one)
    want, tol = ref.gradient(one.double(), one.double() * U)
    close(grad[rows], want[rows], tol[rows], "gradient")
    assert bool((grad[3, 6:] == 0).all())
    zero = torch.zeros(N, device="cuda")
    loss, grad, _, _ = tr.ebsp_policy_loss_grad(logits, tokens, zero, one, one)
    assert loss[2].item() == 0 and bool(torch.isfinite(grad[:3]).all())      # a ratio of 0
    assert tr.ebsp_policy_forward(logits, tokens, zero, one, ref_logp=zero, kl_weight=0.1)[0][2].item() == float("inf")
    logits[0, 7] = float("nan")
    loss, grad, logp, _ = tr.ebsp_policy_loss_grad(logits, tokens, zero, one, one)
    assert math.isnan(logp[0].item()) and math.isnan(loss[0].item()) and bool(torch.isnan(grad[0]).all()) and bool(torch.isfinite(grad[1:3]).all())
    assert bool(torch.isfinite(logp[4:]).all())


@pytest.mark.parametrize("N,V", [(3, 900), (3, 50000), (200, 900), (97, 50000)])
@pytest.mark.parametrize("T", [1e-30, 1e-6, 0.003, 1.0, 300.0, 1e30])
def test_large_logits_and_far_temperatures(tr, N, V, T):
    """Rows whose exponents are of any size: some of their sums are taken from differences, some of their threads' sums are and others are not."""
    logits, tokens, gen = make(N, V, torch.float32, seed=12, spread=1.0)
    logits[0] += 30000.0
    logits[1] = -logits[1].abs() * 1e25                                      # most places weigh nothing
    logits[2, ::7] *= 1e4 * min(T, 1.0)                                      # around the border between the two ways, for T of 0.003 and 1
    ref = Reference(logits, tokens, T)
    logp, stats, _ = tr.ebsp_token_logp(logits, tokens, T)
    ok = ref.logp.abs() < 1e38                                               # a smaller one is -inf in 32 bits
    # c = log2(e) / T is off by 2^-24 of itself, and so is every exponent; the sum's weights move by as much
    more = U * ((ref.p * (logits.double() / T - (logits.double() / T).amax(dim=1, keepdim=True)).abs().nan_to_num(0, 0, 0)).sum(dim=1) + ref.logp.abs()) * 2
    close(logp[ok], ref.logp[ok], (ref.elogp + more)[ok] + 1e-37, "logp")
    assert not bool(torch.isnan(logp).any())
    slope = torch.full((N,), min(T, 1.0), device="cuda")                     # (a gradient is a slope over T)
    grad = tr.ebsp_token_logp_backward(logits, tokens, stats, slope, T)
    want, tol = ref.gradient(slope.double(), slope.double() * 4 * U)
    z = ((logits.double() / T) - (logits.double() / T).amax(dim=1, keepdim=True)).abs()
    tol = tol + (slope.double() / T)[:, None].abs() * ref.p * (z * 2 + more[:, None] / U) * U
    assert bool(torch.isfinite(grad).all())
    close(grad, want, tol, "gradient")
    old, advantage = torch.where(ok, ref.logp, 0.0).float(), torch.ones(N, device="cuda")
    loss, both, again, _ = tr.ebsp_policy_loss_grad(logits, tokens, old, advantage, slope, T, 0.9, 9.0)
    assert torch.equal(again, logp) or bool(((again - logp).abs()[ok] <= 2 * (ref.elogp + more)[ok]).all())


def preference(sums, other, beta, kind, smoothing):
    m = sums if other is None else sums - other
    h = m[0::2] - m[1::2]
    logsigmoid = torch.nn.functional.logsigmoid
    if kind == "sigmoid":
        return h, -(1 - smoothing) * logsigmoid(beta * h) - smoothing * logsigmoid(-beta * h)
    return h, torch.relu(1 - beta * h) if kind == "hinge" else (h - 1 / (2 * beta)) ** 2


def check_preference(tr, logits, tokens, starts, other, dloss, beta=0.3, kind="sigmoid", smoothing=0.0, mean=False):
    at = starts.tolist()
    N = logits.shape[0]
    rows = torch.arange(N, device="cuda")
    some = (tokens >= 0) & (rows >= at[0]) & (rows < at[-1])
    ref = Reference(logits, tokens, 1.0, some)
    leaf = ref.logp.clone().requires_grad_()
    share = [1 / max(1, int(some[a:b].sum())) if mean else 1.0 for a, b in zip(at, at[1:])]
    sums = torch.stack([leaf[a:b].sum() * c for a, b, c in zip(at, at[1:], share)])
    esums = torch.stack([ref.elogp[a:b].sum() * c for a, b, c in zip(at, at[1:], share)]) + 0.0
    h, want = preference(sums, None if other is None else other.double(), beta, kind, smoothing)
    (slope,) = torch.autograd.grad(want, leaf, dloss.double())
    want, sums, h = want.detach(), sums.detach(), h.detach()
    eh = esums[0::2] + esums[1::2] + (sums[0::2].abs() + sums[1::2].abs() + h.abs()) * 2.0 ** -50
    per = {"sigmoid": beta, "hinge": beta, "square": 2 * (h.abs() + 0.5 / beta)}[kind]   # most of the loss' slope, and of the slope's own
    bend = {"sigmoid": beta * beta / 4, "hinge": 0.0, "square": 2.0}[kind]
    # parameters are kept in 32 bits: beta and the smoothing are off by half a step each
    eloss = per * eh + bend * eh * eh + U * (want.abs() + per * (h.abs() + 1 / beta) + 1e-30) * 4
    args = dict(ref=other, beta=beta, kind=kind, smoothing=smoothing, mean=mean)
    loss, got_sums, saved, status = tr.ebsp_preference_forward(logits, tokens, starts, **args)
    close(loss, want, eloss, "loss")
    close(got_sums, sums, esums + sums.abs() * 2 * U + 1e-37, "sums")
    base = per if kind != "square" else per
    eslope = (bend * eh + U * 8 * (torch.zeros_like(h) + base)) * dloss.double().abs()
    of = (torch.bucketize(rows, starts, right=True) - 1).clamp(0, len(at) - 2)
    erow = eslope[of // 2] * torch.tensor(share, device="cuda", dtype=torch.float64)[of] + slope.abs() * 4 * U
    grad, tol = ref.gradient(slope, erow)
    close(tr.ebsp_preference_backward(logits, tokens, starts, saved, dloss), grad, tol, "gradient")
    both, both_grad, both_sums, both_status = tr.ebsp_preference_loss_grad(logits, tokens, starts, dloss, **args)
    close(both, want, eloss, "loss of both")
    close(both_grad, grad, tol, "gradient of both")
    assert bool((status == 0).all()) and bool((both_status == 0).all()) and torch.equal(both_sums, got_sums)
    copy = logits.clone()
    assert tr.ebsp_preference_loss_grad(copy, tokens, starts, dloss, dlogits=copy, **args)[1] is copy and torch.equal(copy, both_grad)
    return both, both_grad


def answers(lengths, V, dtype, seed=0, before=0, behind=0, pad=0):
    N = before + sum(lengths) + behind
    logits, tokens, gen = make(N, V, dtype, seed, pad)
    starts = [before]
    for n in lengths:
        tokens[starts[-1]:starts[-1] + n // 4] = -100
        starts.append(starts[-1] + n)
    other = -torch.rand(len(lengths), generator=gen, device="cuda") * 4 * torch.tensor([n + 1 for n in lengths], device="cuda")
    return logits, tokens, torch.tensor(starts, device="cuda"), other, torch.randn(len(lengths) // 2, generator=gen, device="cuda")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths,V", [((1, 1), 7), ((3, 5), 100), ((9, 2, 1, 30), 1003), ((40, 33), 4100), ((20, 31, 60, 4, 7, 7), 40001), ((2, 1), 70000),
                                       ((5,) * 140, 300), ((300, 500), 129)])
def test_preference_loss_and_its_gradient(tr, lengths, V, dtype):
    for kind, smoothing, mean, before, behind, pad in (("sigmoid", 0.0, False, 0, 0, 0), ("sigmoid", 0.1, True, 3, 5, 3), ("hinge", 0.0, True, 0, 2, 0),
                                                       ("square", 0.0, False, 1, 0, 0)):
        logits, tokens, starts, other, dloss = answers(lengths, V, dtype, 6, before, behind, pad)
        check_preference(tr, logits, tokens, starts, other, dloss, 0.3, kind, smoothing, mean)
        if kind != "hinge":
            check_preference(tr, logits, tokens, starts, None, dloss, 0.01, kind, smoothing, mean)


def test_empty_answers_and_no_pairs(tr):
    logits, tokens, starts, other, dloss = answers((4, 0, 0, 6, 0, 0), 200, torch.float32, 7)
    _, grad = check_preference(tr, logits, tokens, starts, other, dloss, 0.3)
    check_preference(tr, logits, tokens, starts, other, dloss, 0.3, mean=True)
    one = torch.tensor([2], device="cuda")
    loss, grad, sums, status = tr.ebsp_preference_loss_grad(logits, tokens, one, torch.empty(0, device="cuda"))
    assert loss.shape == (0,) and sums.shape == (0,) and status.shape == (0,) and bool((grad == 0).all())
    starts = torch.zeros(5, dtype=torch.int64, device="cuda")
    loss, grad, sums, status = tr.ebsp_preference_loss_grad(logits[:0], tokens[:0], starts, torch.ones(2, device="cuda"))
    assert bool((sums == 0).all()) and bool(((loss - math.log(2)).abs() < 1e-6).all()) and grad.shape == (0, 200) and bool((status == 0).all())


def test_rows_outside_all_answers_are_not_read(tr):
    logits, tokens, starts, other, dloss = answers((4, 6), 3000, torch.bfloat16, 8, before=3, behind=4)
    logits[:3], logits[-4:] = float("nan"), float("nan")
    tokens[0] = 1 << 40                                                      # outside: not looked at
    loss, grad, _, status = tr.ebsp_preference_loss_grad(logits, tokens, starts, dloss, ref=other)
    assert bool(torch.isfinite(loss).all()) and bool(torch.isfinite(grad).all()) and bool((grad[:3] == 0).all()) and bool((grad[-4:] == 0).all())
    assert status.tolist() == [0]


def test_starts_and_tokens_out_of_range_are_flagged(tr):
    logits, tokens, starts, other, dloss = answers((4, 6, 5, 5, 3, 3), 300, torch.float32, 9)
    tokens[12] = 300
    _, grad, _, status = tr.ebsp_preference_loss_grad(logits, tokens, starts, dloss, ref=other)
    assert status.tolist() == [0, 4, 0] and bool((grad[12] == 0).all()) and bool(torch.isfinite(grad).all())
    tokens[12] = 0
    for bad in ([0, 4, 10, 15, 20, 23, 27], [-1, 4, 10, 15, 20, 23, 26], [0, 4, 10, 9, 20, 23, 26], [0, 1 << 62, 10, 15, 20, 23, 26],
                [-(1 << 63), 4, 10, 15, 20, 23, (1 << 63) - 1], [26, 23, 20, 15, 10, 4, 0]):
        loss, grad, sums, status = tr.ebsp_preference_loss_grad(logits, tokens, torch.tensor(bad, device="cuda"), dloss, ref=other)
        assert status.max().item() == 4 and bool(torch.isfinite(grad).all()), bad
    assert status.tolist() == [4, 4, 4]


def test_far_margins_and_masked_answers(tr):
    """A loss of a large margin is its linear part, and of one to the other side nothing; a masked token in an answer makes the margin infinite."""
    logits, tokens, starts, other, dloss = answers((8, 8), 100, torch.float32, 10)
    far = torch.tensor([1e4, -1e4], device="cuda")
    check_preference(tr, logits, tokens, starts, far, dloss, 1.0)
    check_preference(tr, logits, tokens, starts, -far, dloss, 1.0)
    logits[5, tokens[5]] = float("-inf")
    loss, grad, sums, _ = tr.ebsp_preference_loss_grad(logits, tokens, starts, torch.ones(1, device="cuda"))
    assert loss.item() == float("inf") and sums[0].item() == float("-inf") and bool(torch.isfinite(grad).all())
    turned = torch.cat([logits[8:], logits[:8]])
    loss, grad, _, _ = tr.ebsp_preference_loss_grad(turned, torch.cat([tokens[8:], tokens[:8]]), starts, torch.ones(1, device="cuda"))
    assert loss.item() == 0 and bool((grad == 0).all())


def test_autograd(tr):
    """Leading dimensions, rows apart, transposed logits, expanded weights; against the losses' own gradients in 64 bits."""
    logits = torch.randn((2, 6, 70), device="cuda", requires_grad=True)
    tokens = torch.randint(0, 70, (2, 6), device="cuda")
    tokens[0, 3] = -100
    has = tokens >= 0
    exact = logits.detach().double().requires_grad_()
    logp64 = torch.where(has, torch.log_softmax(exact / 0.7, dim=-1).gather(-1, tokens.clamp(min=0)[..., None])[..., 0], 0.0)
    tr.token_logp(logits, tokens, 0.7).sum().backward()
    logp64.sum().backward(retain_graph=True)
    assert torch.allclose(logits.grad.double(), exact.grad, rtol=1e-4, atol=1e-6)
    old = (logp64.detach() - 0.05).float()
    advantage, other = torch.randn((2, 6), device="cuda"), old - 0.1
    logits.grad = exact.grad = None
    turned = logits.detach().reshape(12, 70).t().contiguous().t().requires_grad_()
    for leaf, lead in ((logits, (2, 6)), (turned, (12,))):
        tr.policy_loss(leaf, tokens.reshape(lead), old.reshape(lead), advantage.reshape(lead), 0.7, ref_logp=other.reshape(lead), kl_weight=0.1).mean().backward()
    x, g = torch.exp(logp64 - old.double()), other.double() - logp64
    loss = -torch.minimum(x * advantage, x.clamp(0.8, 1.2) * advantage) + 0.1 * (torch.exp(g) - g - 1)
    torch.where(has, loss, 0.0).mean().backward()
    assert torch.allclose(logits.grad.double(), exact.grad, rtol=1e-4, atol=1e-6)
    assert torch.allclose(turned.grad.double().reshape(2, 6, 70), exact.grad, rtol=1e-4, atol=1e-6)
    rows, starts = logits.detach().reshape(12, 70).clone().requires_grad_(), torch.tensor([0, 2, 6, 9, 12], device="cuda")
    tr.preference_loss(rows, tokens.reshape(12), starts, beta=0.5).mean().backward()
    exact = rows.detach().double().requires_grad_()
    logp64 = torch.where(has.reshape(12), torch.log_softmax(exact, dim=1).gather(1, tokens.reshape(12, 1).clamp(min=0))[:, 0], 0.0)
    sums = torch.stack([logp64[a:b].sum() for a, b in ((0, 2), (2, 6), (6, 9), (9, 12))])
    preference(sums, None, 0.5, "sigmoid", 0.0)[1].mean().backward()
    assert torch.allclose(rows.grad.double(), exact.grad, rtol=1e-4, atol=1e-6)


def test_gradients_against_differences(tr):
    """Central differences of the losses in 64-bit sums of the kernel's values.  The truncation is that of the same difference in 64 bits; the rounding 2^-19 of the terms over h
    (logp of a V of 60: STEP times 16, and its own roundings)."""
    h = 2.0 ** -6
    logits, tokens, starts, other, _ = answers((5, 4, 6, 3), 60, torch.float32, 11)
    N = logits.shape[0]
    step = torch.randn((N, 60), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(torch.bfloat16).float()
    logits = logits.to(torch.bfloat16).float()
    ref = Reference(logits, tokens, 1.0)
    old, advantage = (ref.logp - 0.02).float(), torch.randn(N, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    one, two = torch.ones(N, device="cuda"), torch.ones(2, device="cuda")

    def logp64(s):
        return torch.where(ref.has, torch.log_softmax(s, dim=1).gather(1, ref.at[:, None])[:, 0], 0.0)

    def policy64(s):
        x = torch.exp(logp64(s) - old.double())
        return torch.where(ref.has, -x * advantage.double(), 0.0)

    def pairs64(s):
        at = starts.tolist()
        return preference(torch.stack([logp64(s)[a:b].sum() for a, b in zip(at, at[1:])]), other.double(), 0.1, "sigmoid", 0.0)[1]
    wide = dict(clip_low=float("inf"), clip_high=float("inf"))
    _, stats, _ = tr.ebsp_token_logp(logits, tokens)
    for value, plain, grad in ((lambda s: tr.ebsp_token_logp(s, tokens)[0], logp64, tr.ebsp_token_logp_backward(logits, tokens, stats, one)),
                               (lambda s: tr.ebsp_policy_forward(s, tokens, old, advantage, **wide)[0], policy64,
                                tr.ebsp_policy_loss_grad(logits, tokens, old, advantage, one, **wide)[1]),
                               (lambda s: tr.ebsp_preference_forward(s, tokens, starts, other)[0], pairs64,
                                tr.ebsp_preference_loss_grad(logits, tokens, starts, two, ref=other)[1])):
        up, down = value(logits + h * step).double(), value(logits - h * step).double()
        leaf = logits.double().requires_grad_()
        (slope,) = torch.autograd.grad(plain(leaf).sum(), leaf)
        slope = (slope * step.double()).sum()
        exact = (plain(logits.double() + h * step.double()).sum() - plain(logits.double() - h * step.double()).sum()) / (2 * h)
        size = ref.logp.abs().sum() + up.abs().sum() + advantage.abs().sum() * 2
        tol = (exact - slope).abs() + size * 2.0 ** -19 / h + (grad.double() * step.double()).abs().sum() * 2.0 ** -18
        assert ((up - down).sum() / (2 * h) - (grad.double() * step.double()).sum()).abs() <= tol


def test_refusals(tr):
    logits, tokens = torch.zeros((4, 8), device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    f, starts = torch.zeros(4, device="cuda"), torch.tensor([0, 2, 4], device="cuda")
    common = (dict(logits=logits.double()), dict(logits=logits[0]), dict(logits=None), dict(logits=logits[:, :0]), dict(logits=logits[:1].expand(4, 8)),
              dict(logits=logits.t()), dict(tokens=tokens.int()), dict(tokens=tokens[:3]), dict(tokens=tokens.cpu()), dict(tokens=None))
    for bad in common + (dict(temperature=0.0), dict(temperature=float("nan")), dict(logp=f.half()), dict(stats=f), dict(status=f)):
        with pytest.raises(ValueError):
            tr.ebsp_token_logp(**{**dict(logits=logits, tokens=tokens), **bad})
    for bad in common + (dict(old_logp=f.half()), dict(advantage=f[:3]), dict(ref_logp=f.cpu()), dict(kl_weight=0.1), dict(clip_low=-0.1), dict(clip_high=-1.0),
                         dict(clip_low=float("nan")), dict(dloss=f.double()), dict(dlogits=f), dict(old_logp=None), dict(dloss=None)):
        with pytest.raises(ValueError):
            tr.ebsp_policy_loss_grad(**{**dict(logits=logits, tokens=tokens, old_logp=f, advantage=f, dloss=f), **bad})
    two = torch.zeros(1, device="cuda")
    for bad in common + (dict(starts=starts[:2]), dict(starts=starts.int()), dict(starts=starts.cpu()), dict(starts=None), dict(starts=starts[None]),
                         dict(ref=f[:1]), dict(beta=0.0), dict(beta=float("nan")), dict(kind="other"), dict(smoothing=-0.1), dict(smoothing=float("nan")),
                         dict(kind="hinge", smoothing=0.1), dict(dloss=f), dict(dloss=None)):
        with pytest.raises(ValueError):
            tr.ebsp_preference_loss_grad(**{**dict(logits=logits, tokens=tokens, starts=starts, dloss=two), **bad})
    for bad in (dict(logits=logits[0]), dict(starts=starts[:2]), dict(tokens=tokens[:2])):
        with pytest.raises(ValueError):
            tr.preference_loss(**{**dict(logits=logits, tokens=tokens, starts=starts), **bad})
    for bad in (dict(tokens=None), dict(tokens=tokens[:2]), dict(tokens=tokens.reshape(2, 2)), dict(old_logp=None), dict(advantage=None), dict(ref_logp=f[:2]),
                dict(logits=torch.zeros((), device="cuda"))):
        with pytest.raises(ValueError):
            tr.policy_loss(**{**dict(logits=logits, tokens=tokens, old_logp=f, advantage=f), **bad})
    with pytest.raises(ValueError):
        tr.token_logp(logits, None)
