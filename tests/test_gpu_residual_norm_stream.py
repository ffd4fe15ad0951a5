"""The backward pass of a stream of 16 bits, from x: its results are those of the stream before it was rounded (needs an MI355X).

Tolerances as for the backward pass from y, with u = 2^-24: a chain of ``C`` = K / 1024 + 72 additions over a row, M / 256 + 128 over a column, up to eight roundings of the
sizes that go into anything else, half a step of the result's type.  Beside them the stream that the kernel forms is off by at most eight roundings of what the branch adds
and two of itself (``ev``, times the inverse root), which goes into everything that it is a factor of.  Read from a rounded y, every term of dweight would be off by half a step of
the type instead, 2^15 (bf16) or 2^12 (fp16) times as much."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_residual_norm import EPS, U, close, make, parts  # noqa: E402


@pytest.fixture(scope="module")
def tr():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2001_01347_amd import training
    training.load()
    return training


def arguments(a):
    return a["weight"], a["post_weight"], a["gate"], a["scale"], a["p"], a["rng"]


def check(a, dy, dn, stats, out):
    """dx, dbranch, dweight, dpost_weight and dgate against the formulas on the unrounded stream and the inverse roots that the forward pass left."""
    M, K = dn.shape
    C, R = K / 1024 + 72, M / 256 + 128
    r, w = stats[:, :1].double(), a["weight"].double()
    rb, h, d, fg, f = parts(a, stats[:, 1:].double())
    y = a["x"].double() + fg * d
    ev = r * ((fg * d).abs() * 8 * U + y.abs() * 2 * U)
    gy, gn = dy.double(), dn.double()
    v, gw = y * r, gn * w
    c1 = (gw * v).mean(dim=1, keepdim=True)
    ec1 = (gw * v).abs().mean(dim=1, keepdim=True) * C * U + (gw.abs() * ev).mean(dim=1, keepdim=True)
    dx = gy + r * (gw - v * c1)
    edx = r * v.abs() * ec1 + r * ev * c1.abs() + (gy.abs() + r * (gw.abs() + (v * c1).abs())) * 8 * U
    close(out[0], dx, edx, "dx")
    close(out[2], (gn * v).sum(dim=0), (gn * v).abs().sum(dim=0) * (R + 4) * U + (gn.abs() * ev).sum(dim=0), "dweight")
    dd, edd = fg * dx, fg.abs() * edx + (fg * dx).abs() * 8 * U
    if a["post_weight"] is not None:
        wp = a["post_weight"].double()
        q = (fg * wp * h).abs()
        big, small = (q * (gy.abs() + r * gw.abs())).mean(dim=1, keepdim=True), r * (q * v.abs()).mean(dim=1, keepdim=True)
        c2 = (dd * wp * h).mean(dim=1, keepdim=True)
        ec2 = big * C * U + small * (c1.abs() * C * U + ec1) + r * c1.abs() * (q * ev).mean(dim=1, keepdim=True)
        close(out[1], rb * (dd * wp - h * c2), rb * (wp.abs() * edd + h.abs() * ec2) + rb * ((dd * wp).abs() + (h * c2).abs()) * 8 * U, "dbranch")
        close(out[3], (dd * h).sum(dim=0), (dd * h).abs().sum(dim=0) * (R + 4) * U + (h.abs() * edd).sum(dim=0), "dpost_weight")
    else:
        close(out[1], dd, edd, "dbranch")
    if a["gate"] is not None:
        dg, edg = f * d * dx, (f * d).abs() * edx + (f * d * dx).abs() * 8 * U
        if a["gate"].dim() == 1:
            close(out[4], dg.sum(dim=0), dg.abs().sum(dim=0) * (R + 4) * U + edg.sum(dim=0), "dgate")
        else:
            close(out[4], dg, edg, "dgate")


def by_autograd(tr, a, dy, dn):
    leaf = {k: a[k].detach().clone().requires_grad_() for k in ("x", "branch", "weight", "post_weight", "gate") if a[k] is not None}
    y, n = tr.residual_norm(leaf["x"], leaf["branch"], leaf["weight"], leaf.get("post_weight"), leaf.get("gate"), a["scale"], a["p"], a["rng"], EPS)
    grads = dict(zip(leaf, torch.autograd.grad([y, n], list(leaf.values()), [dy, dn])))
    return [grads.get(k) for k in ("x", "branch", "weight", "post_weight", "gate")]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,K,gate,post,p,pad", [(1, 8, "channel", True, 0.0, 0), (1, 4096, "none", False, 0.0, 0), (3, 7, "token", True, 0.0, 0), (70, 64, "channel", True, 0.1, 0),
                                                 (33, 500, "token", False, 0.5, 3), (19, 1003, "none", True, 0.0, 0), (9, 300, "channel", True, 1.0, 0),
                                                 (700, 2041, "token", True, 0.2, 0), (600, 4096, "channel", True, 0.1, 0), (2100, 1000, "channel", False, 0.0, 1),
                                                 (2, 8193, "token", True, 0.1, 0), (300, 12000, "channel", True, 0.1, 0), (2, 16390, "channel", True, 0.1, 1),
                                                 (300, 16390, "channel", True, 0.0, 0)])
def test_results_are_those_of_the_unrounded_stream(tr, M, K, gate, post, p, pad, dtype):
    a, dy, dn = make(M, K, dtype, dtype, True, post, gate, p, seed=11, pad=pad)
    y, n, stats = tr.ebsp_residual_norm_forward(a["x"], a["branch"], *arguments(a), EPS)
    out = tr.ebsp_residual_norm_backward(dy, dn, None, stats, a["branch"], *arguments(a), x=a["x"])
    check(a, dy, dn, stats, out)
    for s, t in zip(out, by_autograd(tr, a, dy, dn)):
        assert (s is None) == (t is None) and (s is None or torch.equal(s, t))


def test_streams_in_fp32_and_without_a_branch_take_y(tr):
    for stream, dtype, branch in ((torch.float32, torch.bfloat16, True), (torch.float32, torch.float32, True), (torch.bfloat16, torch.bfloat16, False)):
        a, dy, dn = make(11, 300, stream, dtype, branch, branch, "channel" if branch else "none", seed=12)
        y, n, stats = tr.ebsp_residual_norm_forward(a["x"], a["branch"], *arguments(a), EPS)
        want = tr.ebsp_residual_norm_backward(dy, dn, y, stats, a["branch"], *arguments(a))
        got = tr.ebsp_residual_norm_backward(dy, dn, y, stats, a["branch"], *arguments(a), x=a["x"])
        assert all(s is None and t is None or torch.equal(s, t) for s, t in zip(want, got))


def test_dropped_infinities_and_either_gradient(tr):
    """What a dropped element holds goes nowhere, in the stream that is formed again either; dx over dy, and one gradient alone."""
    a, dy, dn = make(40, 520, torch.bfloat16, torch.bfloat16, True, False, "none", 0.5, seed=13)
    y, n, stats = tr.ebsp_residual_norm_forward(a["x"], a["branch"], *arguments(a), EPS)
    clean = tr.ebsp_residual_norm_backward(dy, dn, None, stats, a["branch"], *arguments(a), x=a["x"])
    rb, h, d, fg, f = parts(a)
    dirty = torch.where(fg == 0, torch.full_like(a["branch"], float("inf")), a["branch"])
    again = tr.ebsp_residual_norm_backward(dy, dn, None, stats, dirty, *arguments(a), x=a["x"])
    assert all(s is None and t is None or torch.equal(s, t) for s, t in zip(clean, again))
    zero = torch.zeros_like(dn)
    for one, two in (((dy, zero), (dy, None)), ((torch.zeros_like(dy), dn), (None, dn))):
        s, t = (tr.ebsp_residual_norm_backward(*g, None, stats, a["branch"], *arguments(a), x=a["x"]) for g in (one, two))
        assert all(p is None and q is None or torch.equal(p, q) for p, q in zip(s, t))
    place = dy.clone()
    over = tr.ebsp_residual_norm_backward(place, dn, None, stats, a["branch"], *arguments(a), x=a["x"], dx=place)
    assert over[0] is place and all(s is None and t is None or torch.equal(s, t) for s, t in zip(clean, over))


def test_what_the_graph_keeps(tr):
    """Of 16 bits x, which must not change before the backward pass; y is the program's own then."""
    x, b = (torch.randn((6, 64), device="cuda").bfloat16() for _ in range(2))
    w = torch.ones(64, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    y, n = tr.residual_norm(x, b, w)
    (want,) = torch.autograd.grad(n.float().square().sum(), w)
    y, n = tr.residual_norm(x, b, w)
    with torch.no_grad():
        y.zero_()
    (got,) = torch.autograd.grad(n.float().square().sum(), w)
    assert torch.equal(got, want)
    y, n = tr.residual_norm(x, b, w)
    x.zero_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        n.float().sum().backward()


def test_refusals(tr):
    x, b, w = (torch.zeros((4, 8), device="cuda", dtype=torch.bfloat16) for _ in range(3))
    w, stats = w[0].contiguous(), torch.ones((4, 2), device="cuda")
    for bad in (dict(x=x[:3]), dict(x=x.half()), dict(x=x.cpu()), dict(x=x[0]), dict(x=3), dict(x=None), dict(branch=None)):
        with pytest.raises(ValueError):
            tr.ebsp_residual_norm_backward(**{**dict(dy=x, dn=x, y=None, stats=stats, branch=b, weight=w, x=x), **bad})


def test_x_that_was_joined_in_place_is_refused(tr):
    a, dy, dn = make(6, 64, torch.bfloat16, torch.bfloat16, seed=14)
    x = a["x"].clone()
    y, n, stats = tr.ebsp_residual_norm_forward(x, a["branch"], *arguments(a), EPS, y=x)
    with pytest.raises(ValueError, match="overwritten"):
        tr.ebsp_residual_norm_backward(dy, dn, y, stats, a["branch"], *arguments(a), x=x)
    from_y = tr.ebsp_residual_norm_backward(dy, dn, y, stats, a["branch"], *arguments(a))
    kept = tr.ebsp_residual_norm_forward(a["x"], a["branch"], *arguments(a), EPS)
    assert all(s is None or torch.equal(s, t) for s, t in zip(from_y, tr.ebsp_residual_norm_backward(dy, dn, kept[0], kept[2], a["branch"], *arguments(a))))
