"""Starts of the preference loss that are no starts of rows one behind the other: no pair's results pass for right ones (needs an MI355X).

A row's answer is found among all starts, so one that is out of order misleads rows of other pairs than its own: every pair is flagged, and there is no gradient.  Results of good
starts are held against those of each pair by itself, bit for bit: its rows' log-probabilities are the same numbers, added in the same order."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def tr():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2001_01347_amd import training
    training.load()
    return training


def batch(N, V, dtype=torch.float32, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed + N + 31 * V)
    logits = torch.randn((N, V), generator=gen, device="cuda").to(dtype)
    return logits, torch.randint(0, V, (N,), generator=gen, device="cuda")


def calls(tr, logits, tokens, starts, ref=None):
    """(loss, sums, status, gradient) by either way, which have to agree."""
    starts = torch.as_tensor(starts, device="cuda")
    weight = torch.ones(starts.shape[0] // 2, device="cuda")
    loss, sums, saved, status = tr.ebsp_preference_forward(logits, tokens, starts, ref)
    grad = tr.ebsp_preference_backward(logits, tokens, starts, saved, weight)
    both, both_grad, both_sums, both_status = tr.ebsp_preference_loss_grad(logits, tokens, starts, weight, ref)
    assert torch.equal(both_grad, grad) and torch.equal(status, both_status) and torch.equal(both.nan_to_num(), loss.nan_to_num()) and torch.equal(both_sums, sums)
    return loss, sums, status, grad


def spread(N, pairs):
    """Starts over N rows, every third answer empty."""
    answers = 2 * pairs
    at = [0]
    for a in range(answers):
        left = N - at[-1]
        at.append(at[-1] + (0 if a % 3 == 2 or left == 0 else max(1, min(left, N // answers))))
    return at


def check_flagged(tr, logits, tokens, starts):
    loss, sums, status, grad = calls(tr, logits, tokens, starts)
    assert bool((status == 4).all()), (starts[:20], status.tolist()[:20])
    assert bool((grad == 0).all())


@pytest.mark.parametrize("V", [60, 3000, 70000])
def test_any_start_astray_flags_every_pair(tr, V):
    """Short rows, long ones, and ones in several parts; a bad start at each place."""
    logits, tokens = batch(26, V)
    good = [0, 4, 10, 15, 20, 23, 26]
    assert calls(tr, logits, tokens, good)[2].tolist() == [0, 0, 0]
    for place in range(7):
        for value in (-1, 27, 1 << 62, -(1 << 63), good[place + 1] + 1 if place < 6 else 22, good[place - 1] - 1):
            bad = list(good)
            bad[place] = value
            if all(a <= b for a, b in zip([0] + bad, bad + [26])):
                continue                                                     # in order after all
            check_flagged(tr, logits, tokens, bad)
    check_flagged(tr, logits, tokens, good[::-1])


@pytest.mark.parametrize("N,pairs", [(600, 200), (3, 100), (70, 64), (1, 1), (130, 65), (64, 500), (2000, 1000)])
def test_many_pairs(tr, N, pairs):
    """Starts looked over in several slices, of several for a thread, and by fewer rows than pairs."""
    logits, tokens = batch(N, 40, torch.bfloat16)
    good = spread(N, pairs)
    assert bool((calls(tr, logits, tokens, good)[2] == 0).all())
    places = sorted({0, 1, 2, pairs, 2 * pairs - 1, 2 * pairs, 2 * pairs // 3, 127 % (2 * pairs), (2 * pairs + 64) // 64 % (2 * pairs)})
    for place in places:
        for value in (N + 1, -1):
            check_flagged(tr, logits, tokens, good[:place] + [value] + good[place + 1:])


def test_no_rows(tr):
    logits, tokens = batch(0, 40)
    for pairs in (1, 5, 64, 300):
        zeros = [0] * (2 * pairs + 1)
        loss, sums, status, grad = calls(tr, logits, tokens, zeros)
        assert bool((status == 0).all()) and bool((sums == 0).all()) and grad.shape == (0, 40)
        for place in (0, pairs, 2 * pairs):
            for value in (1, -1):
                check_flagged(tr, logits, tokens, zeros[:place] + [value] + zeros[place + 1:])


@pytest.mark.parametrize("V", [60, 70000])
def test_pairs_that_are_not_flagged_have_their_own_results(tr, V):
    """A token beyond the vocabulary flags its own pair alone; the others' loss, sums and gradients are those of each by itself."""
    logits, tokens = batch(28, V, seed=5)
    starts = [1, 4, 10, 15, 20, 23, 26]
    tokens[12] = V
    tokens[17] = -100
    ref = torch.tensor([-1.0, -2.0, 3.0, -4.0, 0.5, 0.0], device="cuda")
    loss, sums, status, grad = calls(tr, logits, tokens, starts, ref)
    assert status.tolist() == [0, 4, 0]
    assert bool((grad[:1] == 0).all()) and bool((grad[26:] == 0).all()) and bool((grad[12] == 0).all()) and bool((grad[17] == 0).all())
    for pair in range(3):
        alone = calls(tr, logits, tokens, starts[2 * pair:2 * pair + 3], ref[2 * pair:2 * pair + 2].contiguous())
        rows = slice(starts[2 * pair], starts[2 * pair + 2])
        assert torch.equal(alone[0], loss[pair:pair + 1]) and torch.equal(alone[1], sums[2 * pair:2 * pair + 2])
        assert torch.equal(alone[3][rows], grad[rows]) and bool((grad[rows][0] != 0).any())


def test_autograd(tr):
    logits, tokens = batch(12, 300, seed=6)
    logits.requires_grad_()
    (grad,) = torch.autograd.grad(tr.preference_loss(logits, tokens, torch.tensor([0, 3, 9, 6, 12], device="cuda")).sum(), logits)
    assert bool((grad == 0).all())
