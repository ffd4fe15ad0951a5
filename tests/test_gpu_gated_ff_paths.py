"""Every way in which the gated feed-forward block is cut up, against the definition in 64 bits (needs an MI355X).

``test_ff_paths`` sees to it that the shapes take all of them.  Reference and tolerances are those of ``test_gpu_gated_ff``."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import ff_paths  # noqa: E402
import test_gpu_gated_ff as base  # noqa: E402

CASES = [(M, K, F, dtype, cut) for M, K, F, size, cut in ff_paths.SHAPES
         for dtype in ((torch.float32,) if size == 4 else (torch.bfloat16, torch.float16))]


@pytest.mark.parametrize("M,K,F,dtype,cut", CASES)
def test_every_way(M, K, F, dtype, cut):
    from paper_2001_01347_amd import training as tr
    if cut.split()[0] != "few1":
        assert (tr.ebsp_gated_ff_forward_workspace_bytes(M, K, F, dtype) > 0) == (cut.split()[1] != "1")
    room = tr.ebsp_gated_ff_split_workspace_bytes(M, K, F, dtype) - tr.ebsp_gated_ff_workspace_bytes(M, F, dtype)
    assert (room > 0) == (cut.split()[3] != "1" or cut.split()[5] != "1")
    x, wg, wu, dh = base._inputs(M, K, F, dtype, seed=40)
    ref = base.Reference("silu", x, wg, wu, dh)
    h, g, u = tr.ebsp_gated_ff_forward(x, wg, wu, save=True)
    base._compare((h, *tr.ebsp_gated_ff_backward(dh, x, wg, wu, g, u)), ref, ("h", "dx", "dwg", "dwu"))
    for got, w in ((g, wg), (u, wu)):
        bound = 2 * (K + 8) * 2.0 ** -24 * (x.double().abs() @ w.double().abs().t())
        assert bool(((got.double() - x.double() @ w.double().t()).abs() <= bound + 1e-37).all())
    assert torch.equal(tr.ebsp_gated_ff_forward(x, wg, wu)[0], h)
