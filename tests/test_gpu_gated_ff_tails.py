"""Activations and their derivatives where they are small beside 1, relative to their own size (needs an MI355X).

With x = (g, 1), Wg = (1, 0) and Wu = (0, 1) the products are exact, h is act(g) and, for dh = 1, dx = (act'(g), act(g)).
Tolerances.  An exponential e^y or a tail like one is off by the rounding of y, a few steps of 2^-24 of its size, and by some units in the
last place of the function: ``2^-19 + 2^-21 |y|`` of its value.  A 16-bit result is rounded once more: half a step."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _results(act, g, dtype):
    from paper_2001_01347_amd import training as tr
    x = torch.stack([g, torch.ones_like(g)], dim=1).to(dtype)
    assert torch.equal(x[:, 0].to(g.dtype), g)                               # (the values are numbers of the type)
    wg, wu = torch.tensor([[1.0, 0.0]], device="cuda").to(dtype), torch.tensor([[0.0, 1.0]], device="cuda").to(dtype)
    h, p, u = tr.ebsp_gated_ff_forward(x, wg, wu, act, save=True)
    dx, _, _ = tr.ebsp_gated_ff_backward(torch.ones_like(h), x, wg, wu, p, u, act)
    return h[:, 0].double(), dx[:, 0].double(), dx[:, 1].double()


def _within(got, want, tol, dtype):
    tol = tol + torch.finfo(dtype).eps / 2 * (want.abs() + tol)
    off = (got - want).abs()
    assert bool((off <= tol).all()), f"{(off / tol).max().item():.3g} times its bound"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gelu_of_negative_numbers(dtype):
    g = -torch.arange(1, 97, device="cuda", dtype=torch.float64) / 8         # down to -12
    cdf, pdf = 0.5 * torch.special.erfc(-g / math.sqrt(2)), torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    rel = 2.0 ** -19 + 2.0 ** -21 * (g * g / 2)
    h, d, a = _results("gelu", g, dtype)
    _within(h, g * cdf, rel * (g * cdf).abs(), dtype)
    _within(a, g * cdf, rel * (g * cdf).abs(), dtype)
    _within(d, cdf + g * pdf, rel * (cdf + (g * pdf).abs()), dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sigmoid_of_large_numbers(dtype):
    g = torch.arange(-128, 129, device="cuda", dtype=torch.float64) / 2      # up to 64 either way
    g = g.to(dtype).double()
    s, other = torch.sigmoid(g), torch.sigmoid(-g)
    rel = 2.0 ** -19 + 2.0 ** -21 * g.abs()
    h, d, a = _results("sigmoid", g, dtype)
    _within(h, s, rel * s, dtype)
    _within(a, s, rel * s, dtype)
    _within(d, s * other, rel * s * other, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_gelu_around_nought(dtype):
    g = torch.arange(-24, 97, device="cuda", dtype=torch.float64) / 8        # -3 to 12: normal numbers in fp16 too
    cdf, pdf = 0.5 * torch.special.erfc(-g / math.sqrt(2)), torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    rel = 2.0 ** -19 + 2.0 ** -21 * (g * g / 2)
    h, d, a = _results("gelu", g, dtype)
    _within(h, g * cdf, rel * (g * cdf).abs(), dtype)
    _within(a, g * cdf, rel * (g * cdf).abs(), dtype)
    _within(d, cdf + g * pdf, rel * (cdf + (g * pdf).abs()), dtype)
