"""Columns' gradients of rows that have more columns than a launch has workgroups for (needs an MI355X).

One row in fp32, so every column's sum is one product: dweight is dn times (y r), dgate is (scale b) times dx, rounded as 32-bit products are, and held to them bit for bit."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("K", [(1 << 26) + 3, (1 << 28) + 77])
def test_one_wide_row(K):
    from paper_2001_01347_amd import training as tr
    gen = torch.Generator(device="cuda").manual_seed(K)
    x, b, dn, dy = (torch.randn((1, K), generator=gen, device="cuda") for _ in range(4))
    w, g = (torch.randn(K, generator=gen, device="cuda") for _ in range(2))
    y, n, stats = tr.ebsp_residual_norm_forward(x, b, w, gate=g, scale=0.5)
    dx, db, dw, _, dg = tr.ebsp_residual_norm_backward(dy, dn, y, stats, b, w, gate=g, scale=0.5)
    assert torch.equal(dw, (dn * (y * stats[0, 0]))[0])
    assert torch.equal(dg, (b * 0.5 * dx)[0]) and torch.equal(db, 0.5 * g * dx)
    assert abs(stats[0, 0].item() * (y.double().square().mean().item() + 1e-6) ** 0.5 - 1) < (K / 1024 + 72) * 2.0 ** -24
