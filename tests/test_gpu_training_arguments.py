"""Arguments that are no tensors are refused by name (needs an MI355X)."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_gated_ff_operands_that_are_no_tensors():
    from paper_2001_01347_amd import training as tr
    x, w = torch.ones((4, 8), device="cuda"), torch.ones((6, 8), device="cuda")
    dh, g = torch.ones((4, 6), device="cuda"), torch.ones((4, 6), device="cuda")
    for bad in (None, 3, [[1.0] * 8] * 6):
        for args, name in (((bad, w, w), "x"), ((x, bad, w), "wg"), ((x, w, bad), "wu")):
            with pytest.raises(ValueError, match=name):
                tr.ebsp_gated_ff_forward(*args)
            with pytest.raises(ValueError, match=name):
                tr.ebsp_gated_ff_backward(dh, *args, g, g)
            with pytest.raises(ValueError, match=name):
                tr.gated_ff(*args)
