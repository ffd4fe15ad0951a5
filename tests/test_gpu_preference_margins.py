"""The sigmoid preference loss with smoothing at margins of any size, infinite ones too (needs an MI355X).

Tolerance, with u = 2^-24: the margin is made of sums that are exact here but for the rows' own logp, which the kernel gives too (so they are taken from it, each rounded once);
beta and the smoothing are kept in 32 bits, half a step of each; the loss is rounded once: five steps of u of the sizes beta |h| and 1 that it is made of."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24


@pytest.fixture(scope="module")
def tr():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2001_01347_amd import training
    training.load()
    return training


def batch(seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    logits = torch.randn((8, 50), generator=gen, device="cuda")
    tokens = torch.randint(0, 50, (8,), generator=gen, device="cuda")
    return logits, tokens, torch.tensor([0, 2, 4, 6, 8], device="cuda")


def plain(h, beta, e):
    """-(1 - e) log sigmoid(beta h) - e log sigmoid(-beta h), a term of weight 0 left out."""
    def minus_log_sigmoid(z):
        return max(-z, 0.0) + math.log1p(math.exp(-abs(z)))
    return sum(w * minus_log_sigmoid(z) for w, z in ((1 - e, beta * h), (e, -beta * h)) if w > 0)


@pytest.mark.parametrize("smoothing", [0.0, 0.125, 0.5, 1.0])
def test_masked_answers(tr, smoothing):
    """A token masked in the preferred answer of one pair, in the other answer of the next: margins of -inf and +inf."""
    logits, tokens, starts = batch()
    for row in (1, 6):
        logits[row, tokens[row]] = float("-inf")
    weight = torch.tensor([1.0, -2.0], device="cuda")
    loss, sums, saved, status = tr.ebsp_preference_forward(logits, tokens, starts, beta=0.5, smoothing=smoothing)
    both, grad, _, _ = tr.ebsp_preference_loss_grad(logits, tokens, starts, weight, beta=0.5, smoothing=smoothing)
    assert sums[0].item() == sums[3].item() == float("-inf") and status.tolist() == [0, 0]
    assert loss.tolist() == [plain(-math.inf, 0.5, smoothing), plain(math.inf, 0.5, smoothing)] and torch.equal(both, loss)
    assert loss.tolist() == [0.0 if smoothing == 1 else math.inf, 0.0 if smoothing == 0 else math.inf]
    # slopes of -inf and inf: -(1 - e) beta and e beta, exact in 32 bits; the rows' own gradients as with these slopes given
    slopes = torch.tensor([-(1 - smoothing) * 0.5, (1 - smoothing) * 0.5, smoothing * 0.5 * -2, -smoothing * 0.5 * -2], device="cuda").repeat_interleave(2)
    _, stats, _ = tr.ebsp_token_logp(logits, tokens)
    assert torch.equal(grad, tr.ebsp_token_logp_backward(logits, tokens, stats, slopes)) and bool(torch.isfinite(grad).all())
    assert torch.equal(grad, tr.ebsp_preference_backward(logits, tokens, starts, saved, weight))


@pytest.mark.parametrize("smoothing", [0.0, 0.125, 0.3, 1.0])
def test_margins_of_any_size(tr, smoothing):
    logits, tokens, starts = batch(1)
    logp = tr.ebsp_token_logp(logits, tokens)[0].double().reshape(4, 2).sum(dim=1)
    for beta in (0.1, 2.0):
        for far in (0.0, 1e-3, 1.0, 40.0, 1e4, 1e30, 3e38):
            ref = torch.tensor([far, -far, -far, far], device="cuda") / 2
            loss, sums, saved, _ = tr.ebsp_preference_forward(logits, tokens, starts, ref, beta=beta, smoothing=smoothing)
            margins = (logp - ref.double()).reshape(2, 2)
            for got, h in zip(loss.tolist(), (margins[:, 0] - margins[:, 1]).tolist()):
                want = plain(h, beta, smoothing)
                assert got == want or abs(got - want) <= 5 * U * (beta * abs(h) + 1) or abs(want) > 3.4e38, (beta, far, got, want)


def test_margins_that_are_no_number(tr):
    logits, tokens, starts = batch(2)
    for row in (0, 2):
        logits[row, tokens[row]] = float("-inf")                             # -inf less -inf
    for smoothing in (0.0, 0.1, 1.0):
        loss = tr.ebsp_preference_forward(logits, tokens, starts, smoothing=smoothing)[0]
        assert math.isnan(loss[0].item()) and math.isfinite(loss[1].item())
