"""The training operators as parts of an autograd graph, on the CPU: the entry points are replaced by plain torch operations."""
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture
def calls(monkeypatch):
    from paper_2001_01347_amd import training
    seen = []

    def forward(x, wg, wu, act="silu", save=False, **_):
        seen.append(save)
        with torch.no_grad():
            g, u = x @ wg.t(), x @ wu.t()
            return torch.nn.functional.silu(g) * u, g if save else None, u if save else None
    monkeypatch.setattr(training, "ebsp_gated_ff_forward", forward)
    return seen


@pytest.mark.parametrize("place", range(3))
@pytest.mark.parametrize("mode", [torch.enable_grad, torch.no_grad])
def test_gated_ff_does_not_lose_a_tangent(calls, mode, place):
    """Forward mode does not depend on whether gradients are on: a tangent is refused in either case."""
    import torch.autograd.forward_ad as forward_ad
    from paper_2001_01347_amd import training
    args = [torch.randn(4, 16), torch.randn(8, 16), torch.randn(8, 16)]
    with mode(), forward_ad.dual_level():
        args[place] = forward_ad.make_dual(args[place], torch.ones_like(args[place]))
        with pytest.raises(NotImplementedError):
            training.gated_ff(*args)


def test_gated_ff_saves_the_products_for_a_backward_pass_alone(calls):
    from paper_2001_01347_amd import training
    x, wg, wu = torch.randn(2, 3, 16), torch.randn(8, 16), torch.randn(8, 16)
    for needed in (False, True):
        wg.requires_grad_(needed)
        assert training.gated_ff(x, wg, wu).requires_grad == needed
        with torch.no_grad():
            assert not training.gated_ff(x, wg, wu).requires_grad
        with torch.inference_mode():
            assert training.gated_ff(x, wg, wu).shape == (2, 3, 8)
    assert calls == [False, False, False, True, False, False]


@pytest.fixture
def losses(monkeypatch):
    from paper_2001_01347_amd import training

    def forward(logits, top_index, top_logit, temperature, kl_weight, labels, ce_weight):
        return logits.sum(dim=1), torch.zeros(logits.shape[0], 3), None
    monkeypatch.setattr(training, "ebsp_distill_forward", forward)


def test_distill_loss_takes_matching_rows_only(losses):
    """Entries and labels whose leading dimensions are others, though as many, belong to other rows."""
    from paper_2001_01347_amd import training
    logits, index, values, labels = torch.randn(2, 3, 50), torch.zeros(2, 3, 4, dtype=torch.int64), torch.randn(2, 3, 4), torch.zeros(2, 3, dtype=torch.int64)
    assert training.distill_loss(logits, index, values, 2.0, 0.5, labels, 0.5).shape == (2, 3)
    # the rows as one dimension, and dimensions of one, leave the order as it is
    assert training.distill_loss(logits, index.reshape(6, 4), values, 2.0, 0.5, labels.reshape(6), 0.5).shape == (2, 3)
    assert training.distill_loss(logits.reshape(2, 3, 1, 50), index, values.reshape(6, 4), 2.0, 0.5, labels.reshape(1, 2, 3), 0.5).shape == (2, 3, 1)
    assert training.distill_loss(logits[:0], index[:0], values[:0], labels=labels[:0], ce_weight=0.5).shape == (0, 3)
    assert training.distill_loss(logits[0, 0], index[0, 0], values[0, 0], labels=labels[0, 0], ce_weight=0.5).shape == ()
    for bad in (dict(top_index=index.transpose(0, 1)), dict(top_logit=values.transpose(0, 1)), dict(labels=labels.t()),
                dict(top_index=index.reshape(6, 4).t()), dict(top_index=None), dict(top_logit=[1.0]), dict(labels=7), dict(top_index=index[:1])):
        with pytest.raises(ValueError):
            training.distill_loss(**{**dict(logits=logits, top_index=index, top_logit=values, labels=labels, ce_weight=0.5), **bad})
