"""Teacher's weight and labels at places that are masked with the type's lowest value (needs an MI355X).

The loss of such a row is of that value's size and finite.  Reference and tolerances are those of ``test_gpu_distill``."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import test_gpu_distill as base  # noqa: E402


@pytest.mark.parametrize("dtype", base.TYPES)
@pytest.mark.parametrize("T", [0.5, 1.0, 2.0, 4.0])
@pytest.mark.parametrize("N,V", [(4, 2000), (300, 2000), (3, 40000), (130, 70003)])
def test_entries_and_labels_at_the_lowest_value(N, V, T, dtype):
    from paper_2001_01347_amd import training as tr
    logits, index, values, labels, dloss = base.make(N, V, 8, dtype, seed=30, padding=False)
    low = torch.finfo(dtype).min
    labels[:] = 5
    logits[0, 5] = low                                                       # the label alone
    logits[1, index[1, 2]] = low                                             # an entry alone
    logits[2, index[2]] = low                                                # all entries, and the label at one of them
    labels[2] = index[2, 0]
    loss, grad = base.check(tr, logits, index, values, labels, dloss, T, 0.125, 0.25)
    assert torch.isfinite(loss).all() and torch.isfinite(grad).all()
    base.check(tr, logits, index, values, None, dloss, T, 0.125, 0.0)


@pytest.mark.parametrize("N", [4, 300])
def test_a_small_weight_at_a_forbidden_place_is_infinite_too(N):
    from paper_2001_01347_amd import training as tr
    logits, index, values, labels, dloss = base.make(N, 500, 2, torch.float32, seed=31, padding=False)
    logits[1, index[1, 1]] = float("-inf")
    values[1, 1] = values[1, 0] - 80                                         # q = e^-80, times 1e-10 below all 32-bit numbers
    loss, _, _ = tr.ebsp_distill_forward(logits, index, values, kl_weight=1e-10)
    assert loss[1].item() == float("inf") and torch.isfinite(loss[2:]).all() and torch.isfinite(loss[:1]).all()
