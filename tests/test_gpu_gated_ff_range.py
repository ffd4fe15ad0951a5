"""Gradients of the gated feed-forward block whose dg and du pass the range of fp16 while the results do not (needs an MI355X).

Tolerances.  dg and du are rounded to fp16 times a common power of two: half a step, ``U`` = 2^-11 of a value's size, or 2^-39 of the
largest of all.  A sum of n products is held in 32 bits: ``2 (n + 8) 2^-24`` of the sum of their sizes.  g and u are taken as the forward pass
saved them; activations are off by 2^-20 (1 + |g|).  A result is rounded once: half a step, or 2^-25 below the normal numbers."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -11


def _check(name, got, left, right, left_tol):
    want = left @ right
    n = left.shape[1]
    tol = left_tol @ right.abs() + 2 * (n + 8) * 2.0 ** -24 * (left.abs() @ right.abs())
    tol = tol * (1 + 2 * U) + U * want.abs() + 2.0 ** -25
    assert bool((want.abs() < 65000).all())                                  # what is asked for fits
    off = (got.double() - want).abs()
    assert bool((off <= tol).all()), f"{name}: {(off / tol).max().item():.3g} times its bound"


# Whole sums, dx in parts, dW in parts; rows of whole 16-byte chunks and others.
@pytest.mark.parametrize("M,K,F", [(33, 64, 128), (40, 72, 1600), (3000, 64, 72), (61, 67, 131)])
@pytest.mark.parametrize("case", ["dx high", "dw high", "dw low", "dx low"])
def test_range_of_fp16(M, K, F, case):
    from paper_2001_01347_amd import training as tr
    gen = torch.Generator(device="cuda").manual_seed(M + K + F)
    # sizes of x, Wg, Wu and dh: dg of some 1e5 and 1e-7, results that fit
    sx, sg, su, sd = {"dx high": (8.0, 2.0 ** -9, 4.0, 400.0), "dw high": (2.0 ** -8, 32.0, 8192.0, 100.0),
                      "dw low": (32.0, 2.0 ** -8, 2.0 ** -13, 2e-6), "dx low": (2.0 ** -8, 32.0, 32.0, 5e-7)}[case]

    def rand(r, c, size):
        return (torch.randn((r, c), generator=gen, device="cuda") * size).half()
    x, wg, wu, dh = rand(M, K, sx), rand(F, K, sg), rand(F, K, su), rand(M, F, sd)
    _, g, u = tr.ebsp_gated_ff_forward(x, wg, wu, "silu", save=True)
    dx, dwg, dwu = tr.ebsp_gated_ff_backward(dh, x, wg, wu, g, u, "silu")
    g, u, d = g.double(), u.double(), dh.double()
    s = torch.sigmoid(g)
    du, dg = d * g * s, d * u * (s + g * s * (1 - s))
    most = max(dg.abs().max(), du.abs().max()).item()
    assert most > 70000 if "high" in case else most < 2.0 ** -14
    soft = 2.0 ** -20 * (1 + g.abs())
    tol_u = d.abs() * soft + U * du.abs() + 2.0 ** -39 * most
    tol_g = d.abs() * u.abs() * soft + U * dg.abs() + 2.0 ** -39 * most
    if "dx" in case:
        _check("dx", dx, torch.cat([dg, du], 1), torch.cat([wg, wu]).double(), torch.cat([tol_g, tol_u], 1))
    else:
        _check("dwg", dwg, dg.t(), x.double(), tol_g.t())
        _check("dwu", dwu, du.t(), x.double(), tol_u.t())


def test_an_infinity_does_not_change_the_others():
    """A token whose dg is infinite reaches its own row of dx; the power of two is chosen from what is finite."""
    from paper_2001_01347_amd import training as tr
    gen = torch.Generator(device="cuda").manual_seed(5)
    x, wg, wu, dh = ((torch.randn(s, generator=gen, device="cuda") * k).half() for s, k in (((40, 64), 1.0), ((96, 64), 0.125), ((96, 64), 0.125), ((40, 96), 1.0)))
    _, g, u = tr.ebsp_gated_ff_forward(x, wg, wu, save=True)
    clean = tr.ebsp_gated_ff_backward(dh, x, wg, wu, g, u)[0]
    dh[7, 5], dh[8, 6] = float("inf"), float("nan")
    dx = tr.ebsp_gated_ff_backward(dh, x, wg, wu, g, u)[0]
    keep = torch.ones(40, dtype=torch.bool, device="cuda")
    keep[7:9] = False
    assert torch.equal(dx[keep], clean[keep]) and not torch.isfinite(dx[8]).any() and not torch.isfinite(dx[7]).all()


def test_in_a_graph_the_power_is_chosen_anew():
    """Replays with inputs of another size than the captured ones."""
    from paper_2001_01347_amd import training as tr
    gen = torch.Generator(device="cuda").manual_seed(6)
    x, wg, wu, dh = ((torch.randn(s, generator=gen, device="cuda") * k).half() for s, k in (((70, 64), 8.0), ((96, 64), 2.0 ** -9), ((96, 64), 4.0), ((70, 96), 1.0)))

    def step():
        _, g, u = tr.ebsp_gated_ff_forward(x, wg, wu, save=True)
        return tr.ebsp_gated_ff_backward(dh, x, wg, wu, g, u)
    base = dh.clone()
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for size in (400.0, 1.0, 1e-6, 400.0):
        dh.copy_(base * size)
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        assert torch.isfinite(want[0]).all()
