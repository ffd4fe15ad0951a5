"""Places and labels beyond the vocabulary in the loss by itself and in the gradient from its statistics (needs an MI355X).

An entry or a label that is left out gives what padding in its place gives, bit for bit."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import test_gpu_distill as base  # noqa: E402


@pytest.mark.parametrize("N,V", [(5, 600), (300, 600), (5, 40000), (130, 70003)])
@pytest.mark.parametrize("index_type", [torch.int32, torch.int64])
def test_what_is_left_out_is_as_padding(N, V, index_type):
    from paper_2001_01347_amd import training as tr
    logits, index, values, labels, dloss = base.make(N, V, 12, torch.float16, seed=32, padding=False, index_type=index_type)
    labels[:] = 5
    kept, kept_labels = index.clone(), labels.clone()
    index[0, 3], kept[0, 3] = V, -1
    index[1, 0], kept[1, 0] = (1 << 31) - 1, -1
    labels[2], kept_labels[2] = V, -100
    index[3, 2], kept[3, 2] = -(1 << 31), -1                                 # padding, whatever the number
    index[4], kept[4] = V + 7, -1                                            # no entry left, no label
    labels[4], kept_labels[4] = 1 << 40, -1
    if index_type == torch.int64:
        index[1, 1], kept[1, 1] = 1 << 40, -1
    args = dict(temperature=2.0, kl_weight=1.0, ce_weight=0.5)
    loss, stats, status = tr.ebsp_distill_forward(logits, index, values, labels=labels, **args)
    want_loss, want_stats, clean = tr.ebsp_distill_forward(logits, kept, values, labels=kept_labels, **args)
    assert status[:5].tolist() == [4, 4, 4, 0, 4] and bool((status[5:] == 0).all()) and bool((clean == 0).all())
    assert torch.equal(loss, want_loss) and torch.equal(stats, want_stats)
    grad = tr.ebsp_distill_backward(logits, index, values, stats, dloss, labels=labels, **args)
    assert torch.equal(grad, tr.ebsp_distill_backward(logits, kept, values, stats, dloss, labels=kept_labels, **args))
    assert bool((grad[4] == 0).all()) and bool((grad[:4] != 0).any(dim=1).all())
    want, want_tol = base.reference(logits, kept, values, 2.0, 1.0, kept_labels, 0.5, dloss)[2:]
    assert bool(((grad.double() - want).abs() <= want_tol).all())
