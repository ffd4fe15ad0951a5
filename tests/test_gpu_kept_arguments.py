"""What a program changes between the passes is what it was to the backward pass: places in the random numbers, and numbers that are not plain ones (needs an MI355X)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

SEED, OFFSET = 11, 22


@pytest.fixture(scope="module")
def tr():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2001_01347_amd import training
    training.load()
    return training


PLACES = {"list": lambda: [SEED, OFFSET], "tuple": lambda: (SEED, OFFSET), "array": lambda: np.array([SEED, OFFSET]), "iterator": lambda: iter([SEED, OFFSET]),
          "device": lambda: torch.tensor([SEED, OFFSET], device="cuda")}


def moved_on(rng):
    if not isinstance(rng, tuple) and hasattr(rng, "__setitem__"):
        rng[1] += 1


@pytest.mark.parametrize("kind", list(PLACES))
def test_place_in_the_random_numbers(tr, kind):
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, b = (torch.randn((6, 300), generator=gen, device="cuda").requires_grad_() for _ in range(2))
    w = torch.ones(300, device="cuda")

    def grads(rng):
        out = tr.dropout(x, 0.5, rng)
        moved_on(rng)
        return out.detach(), *torch.autograd.grad(out, x, torch.ones_like(out))

    def norm_grads(rng):
        y, n = tr.residual_norm(x, b, w, p=0.5, rng=rng)
        moved_on(rng)
        return y.detach(), n.detach(), *torch.autograd.grad((y.sum() + n.square().sum()), [x, b])
    for f in (grads, norm_grads):
        want = f((SEED, OFFSET))
        assert all(torch.equal(s, t) for s, t in zip(f(PLACES[kind]()), want))
    kept = tr.dropout(torch.ones_like(x), 0.5, (SEED, OFFSET)) != 0
    assert torch.equal(grads(PLACES[kind]())[1] != 0, kept)


def test_numbers(tr):
    """0-dimensional arrays and tensors in the places of numbers."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((5, 40), generator=gen, device="cuda").requires_grad_()
    w, f = torch.ones(40, device="cuda"), torch.full((5,), -3.5, device="cuda")
    tokens, advantage = torch.arange(5, device="cuda"), torch.tensor([1.0, -1.0, 2.0, -2.0, 0.5], device="cuda")
    for form in (lambda v: np.array(v), lambda v: torch.tensor(v, dtype=torch.float64)):
        for call, value in ((lambda v: tr.dropout(x, v, (1, 2)), 0.5), (lambda v: tr.residual_norm(x, x.detach(), w, p=v, rng=(1, 2))[1], 0.5),
                            (lambda v: tr.residual_norm(x, x.detach() * 2, w, scale=v)[1], 0.5), (lambda v: tr.token_logp(x, tokens, v), 0.5),
                            (lambda v: tr.policy_loss(x, tokens, f, advantage, v), 0.5), (lambda v: tr.policy_loss(x, tokens, f, advantage, clip_low=v), 0.5),
                            (lambda v: tr.policy_loss(x, tokens, f, advantage, clip_high=v), 0.5),
                            (lambda v: tr.policy_loss(x, tokens, f, advantage, ref_logp=f, kl_weight=v), 0.5)):
            (want,) = torch.autograd.grad(call(value).square().sum(), x)
            given = form(value)
            out = call(given)
            given[...] = 0.25
            (got,) = torch.autograd.grad(out.square().sum(), x)
            assert torch.equal(got, want)
