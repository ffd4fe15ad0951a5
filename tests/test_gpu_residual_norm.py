"""The residual stream around a block and its backward pass against the formulas in 64 bits (needs an MI355X).

Tolerances, with u = 2^-24.  A sum over a row is a chain of at most K / 1024 + 64 additions, each of relative error u, and every term of it a product or two:
``C`` = K / 1024 + 72 steps of the sum of sizes.  An inverse root halves the relative error of its sum and adds four roundings.  Everything else is products and
fused sums of at most eight roundings of the sizes that go in.  A result is rounded once to its type: half a step of its size, and half
a step of the smallest normal number below that.  The backward pass is held to its formula on the y and the inverse roots that it is given, which are the
forward pass' own; columns are sums over at most M / 256 + 128 additions."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import philox  # noqa: E402

TYPES = [torch.bfloat16, torch.float16, torch.float32]
PAIRS = [(t, t) for t in TYPES] + [(torch.float32, torch.bfloat16), (torch.float32, torch.float16)]
U = 2.0 ** -24
RNG = (1234567890123456789, 42)
EPS = 1e-6


@pytest.fixture(scope="module")
def tr():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2001_01347_amd import training
    training.load()
    return training


def close(got, want, tol, what):
    dtype = got.dtype
    half = torch.finfo(dtype).eps / 2
    tol = tol * (1 + half) + want.abs() * half + torch.finfo(dtype).smallest_normal * half
    off = (got.double() - want).abs()
    assert bool((off <= tol).all()), (what, (off - tol).max().item(), off.max().item())


def make(M, K, stream, dtype, branch=True, post=False, gate="none", p=0.0, seed=0, pad=0):
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + M + 31 * K)

    def rows(scale, dt):
        full = torch.full((M, K + 2 * pad), float("nan"), dtype=dt, device="cuda")
        full[:, pad:pad + K] = (torch.randn((M, K), generator=gen, device="cuda") * scale).to(dt)
        return full[:, pad:pad + K]

    def vector(scale, shift=0.0):
        return (shift + torch.randn((K,), generator=gen, device="cuda") * scale).to(dtype)
    a = {"x": rows(1.5, stream), "branch": rows(0.7, dtype) if branch else None, "weight": vector(0.2, 1.0),
         "post_weight": vector(0.2, 1.0) if post else None, "gate": None, "scale": 0.5 if branch else 1.0, "p": p, "rng": RNG if p else None}
    if gate == "channel":
        a["gate"] = vector(0.5)
    elif gate == "token":
        a["gate"] = rows(0.5, dtype)
    return a, rows(0.3, stream), rows(0.3, dtype)


def parts(a, rb=None):
    """What the branch adds, in 64 bits: b r', d, f g and f."""
    x = a["x"].double()
    M, K = x.shape
    b = a["branch"].double()
    if a["post_weight"] is not None:
        if rb is None:
            rb = (b.square().mean(dim=1, keepdim=True) + EPS) ** -0.5
        h = b * rb
        d = h * a["post_weight"].double()
    else:
        rb, h, d = torch.zeros((M, 1), dtype=torch.float64, device="cuda"), b, b
    f = torch.full((M, K), float(a["scale"]), dtype=torch.float64, device="cuda")
    if a["p"] > 0:
        keep = torch.from_numpy(philox.keep(M, K, a["p"], *a["rng"])).cuda()
        f = torch.where(keep, f * philox.kept_factor(a["p"]), 0.0)
    fg = f if a["gate"] is None else f * a["gate"].double()
    return rb, h, d, fg, f


def check_forward(tr, a):
    x = a["x"].double()
    M, K = x.shape
    C = K / 1024 + 72
    y, n, stats = tr.ebsp_residual_norm_forward(a["x"], a["branch"], a["weight"], a["post_weight"], a["gate"], a["scale"], a["p"], a["rng"], EPS)
    eb = (C / 2 + 4) * U
    want, dy = x, torch.zeros_like(x)
    if a["branch"] is not None:
        rb, _, d, fg, _ = parts(a)
        want = x + fg * d
        dy = (fg * d).abs() * (eb + 8 * U) + want.abs() * U
        close(y, want, dy, "y")
        if a["post_weight"] is not None:
            assert bool(((stats[:, 1:].double() - rb).abs() <= rb * eb).all())
    else:
        assert y is a["x"]
    r = (want.square().mean(dim=1, keepdim=True) + EPS) ** -0.5
    er = eb + (want.abs() * dy).sum(dim=1, keepdim=True) / (want.square().sum(dim=1, keepdim=True) + K * EPS)
    w = a["weight"].double()
    close(n, want * r * w, (want * r * w).abs() * (er + 4 * U) + r * w.abs() * dy, "n")
    assert bool(((stats[:, :1].double() - r).abs() <= r * er * 1.01).all())
    return y, n, stats


def check_backward(tr, a, dy, dn, y, stats):
    """Against the formula on this y and these inverse roots; every size that a sum or difference is made of is kept beside it."""
    M, K = y.shape
    C, R = K / 1024 + 72, M / 256 + 128
    out = tr.ebsp_residual_norm_backward(dy, dn, y, stats, a["branch"], a["weight"], a["post_weight"], a["gate"], a["scale"], a["p"], a["rng"])
    r, w = stats[:, :1].double(), a["weight"].double()
    zero = torch.zeros((M, K), dtype=torch.float64, device="cuda")
    gy, gn = zero if dy is None else dy.double(), zero if dn is None else dn.double()
    v = y.double() * r
    gw = gn * w
    c1 = (gw * v).mean(dim=1, keepdim=True)
    ec1 = (gw * v).abs().mean(dim=1, keepdim=True) * C * U
    dx = gy + r * (gw - v * c1)
    edx = r * v.abs() * ec1 + (gy.abs() + r * (gw.abs() + (v * c1).abs())) * 8 * U
    close(out[0], dx, edx, "dx")
    close(out[2], (gn * v).sum(dim=0), (gn * v).abs().sum(dim=0) * (R + 4) * U, "dweight")
    assert (out[1] is None) == (a["branch"] is None) and (out[3] is None) == (a["post_weight"] is None) and (out[4] is None) == (a["gate"] is None)
    if a["branch"] is None:
        return out
    rb, h, d, fg, f = parts(a, stats[:, 1:].double())
    dd, edd = fg * dx, fg.abs() * edx + (fg * dx).abs() * 8 * U
    if a["post_weight"] is not None:
        wp = a["post_weight"].double()
        q = (fg * wp * h).abs()
        big, small = (q * (gy.abs() + r * gw.abs())).mean(dim=1, keepdim=True), r * (q * v.abs()).mean(dim=1, keepdim=True)
        c2 = (dd * wp * h).mean(dim=1, keepdim=True)
        ec2 = big * C * U + small * (c1.abs() * C * U + ec1)
        db = rb * (dd * wp - h * c2)
        close(out[1], db, rb * (wp.abs() * edd + h.abs() * ec2) + rb * ((dd * wp).abs() + (h * c2).abs()) * 8 * U, "dbranch")
        close(out[3], (dd * h).sum(dim=0), (dd * h).abs().sum(dim=0) * (R + 4) * U + (h.abs() * edd).sum(dim=0), "dpost_weight")
    else:
        close(out[1], dd, edd, "dbranch")
    if a["gate"] is not None:
        dg, edg = f * d * dx, (f * d).abs() * edx + (f * d * dx).abs() * 8 * U
        if a["gate"].dim() == 1:
            close(out[4], dg.sum(dim=0), dg.abs().sum(dim=0) * (R + 4) * U + edg.sum(dim=0), "dgate")
        else:
            close(out[4], dg, edg, "dgate")
    return out


@pytest.mark.parametrize("stream,dtype", PAIRS)
@pytest.mark.parametrize("M,K", [(1, 1), (1, 8), (3, 7), (70, 64), (5, 65), (9, 127), (33, 128), (6, 500), (7, 513), (4, 1024), (37, 1003), (3, 2048), (2, 2056), (5, 4096),
                                 (3, 4104), (2, 8192), (2, 8193), (3, 16384), (2, 16390), (3, 40001)])
def test_all_parts_at_every_width(tr, M, K, stream, dtype):
    a, dy, dn = make(M, K, stream, dtype, post=True, gate="channel", p=0.1)
    y, n, stats = check_forward(tr, a)
    check_backward(tr, a, dy, dn, y, stats)


@pytest.mark.parametrize("stream,dtype", PAIRS)
@pytest.mark.parametrize("gate", ["none", "channel", "token"])
@pytest.mark.parametrize("branch,post,p", [(False, False, 0.0), (True, False, 0.0), (True, True, 0.0), (True, False, 0.5), (True, True, 0.3), (True, True, 1.0)])
def test_combinations(tr, branch, post, gate, p, stream, dtype):
    if not branch:
        gate = "none"                                                        # (it needs a branch)
    for M, K, pad in ((19, 300, 3), (3, 20000, 1)):
        a, dy, dn = make(M, K, stream, dtype, branch, post, gate, p, seed=1, pad=pad)
        y, n, stats = check_forward(tr, a)
        check_backward(tr, a, dy, dn, y, stats)


@pytest.mark.parametrize("M,K", [(2000, 64), (1300, 200), (600, 1000), (1100, 4096), (5000, 8)])
def test_many_rows(tr, M, K):
    a, dy, dn = make(M, K, torch.bfloat16, torch.bfloat16, post=True, gate="channel", p=0.1, seed=2)
    y, n, stats = check_forward(tr, a)
    first = check_backward(tr, a, dy, dn, y, stats)
    again = tr.ebsp_residual_norm_backward(dy, dn, y, stats, a["branch"], a["weight"], a["post_weight"], a["gate"], a["scale"], a["p"], a["rng"])
    assert all(torch.equal(s, t) for s, t in zip(first, again))


@pytest.mark.parametrize("stream,dtype", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float16), (torch.float32, torch.float32)])
@pytest.mark.parametrize("M,K", [(131073, 50), (65541, 120), (32769, 255), (16385, 500), (8193, 1000), (4099, 2041), (2051, 4090), (600, 8190)])
def test_rows_enough_for_whole_cus(tr, M, K, stream, dtype):
    """A backward pass in its larger workgroups, for every number of threads a row."""
    a, dy, dn = make(M, K, stream, dtype, post=True, gate="channel", seed=10)
    y, n, stats = check_forward(tr, a)
    check_backward(tr, a, dy, dn, y, stats)


def test_either_gradient_may_be_missing(tr):
    for K in (100, 4096, 20000):
        a, dy, dn = make(11, K, torch.float32, torch.bfloat16, post=True, gate="token", p=0.2, seed=3)
        y, n, stats = check_forward(tr, a)
        check_backward(tr, a, None, dn, y, stats)
        check_backward(tr, a, dy, None, y, stats)


def test_only_what_is_wanted(tr):
    a, dy, dn = make(11, 300, torch.float32, torch.float32, post=True, gate="channel", seed=4)
    y, n, stats = check_forward(tr, a)
    args = (dy, dn, y, stats, a["branch"], a["weight"], a["post_weight"], a["gate"], a["scale"])
    whole = tr.ebsp_residual_norm_backward(*args)
    for i in range(5):
        for alone in (True, False):
            want = [alone == (j == i) for j in range(5)]
            some = tr.ebsp_residual_norm_backward(*args, want=want)
            for j in range(5):
                assert some[j] is None if not want[j] else torch.equal(some[j], whole[j]), (i, j)


def test_in_place(tr):
    for K in (300, 4096, 20000):
        a, dy, dn = make(9, K, torch.float32, torch.bfloat16, post=True, gate="token", p=0.3, seed=5, pad=2)
        y, n, stats = tr.ebsp_residual_norm_forward(a["x"], a["branch"], a["weight"], a["post_weight"], a["gate"], a["scale"], a["p"], a["rng"])
        want = tr.ebsp_residual_norm_backward(dy, dn, y, stats, a["branch"], a["weight"], a["post_weight"], a["gate"], a["scale"], a["p"], a["rng"])
        got = tr.ebsp_residual_norm_backward(dy, dn, y, stats, a["branch"], a["weight"], a["post_weight"], a["gate"], a["scale"], a["p"], a["rng"], dx=dy)
        assert got[0] is dy and all(torch.equal(s, t) for s, t in zip(want, got))
        x = a["x"]
        y2, n2, stats2 = tr.ebsp_residual_norm_forward(x, a["branch"], a["weight"], a["post_weight"], a["gate"], a["scale"], a["p"], a["rng"], y=x)
        assert y2 is x and torch.equal(y2, y) and torch.equal(n2, n) and torch.equal(stats2, stats)


def test_no_rows(tr):
    a, dy, dn = make(0, 24, torch.float32, torch.float32, post=True, gate="channel")
    y, n, stats = tr.ebsp_residual_norm_forward(a["x"], a["branch"], a["weight"], a["post_weight"], a["gate"])
    out = tr.ebsp_residual_norm_backward(dy, dn, y, stats, a["branch"], a["weight"], a["post_weight"], a["gate"])
    assert y.shape == n.shape == out[0].shape == out[1].shape == (0, 24)
    assert all(t.shape == (24,) and bool((t == 0).all()) for t in out[2:])


def test_rows_of_zeros_and_of_large_numbers(tr):
    a, dy, dn = make(6, 500, torch.bfloat16, torch.bfloat16, post=True, seed=6)
    a["x"][0] = 0
    a["branch"][0] = 0
    a["branch"][1] *= 1e15
    a["x"][2] *= 1e15
    y, n, stats = check_forward(tr, a)
    out = check_backward(tr, a, dy, dn, y, stats)
    assert bool((n[0] == 0).all()) and all(bool(torch.isfinite(t).all()) for t in out if t is not None)


def test_a_row_that_is_no_number_stays_alone(tr):
    a, dy, dn = make(6, 500, torch.bfloat16, torch.bfloat16, post=True, seed=7)
    clean = tr.ebsp_residual_norm_forward(a["x"], a["branch"], a["weight"], a["post_weight"])[1].clone()
    a["branch"][2, 17] = float("nan")
    n = tr.ebsp_residual_norm_forward(a["x"], a["branch"], a["weight"], a["post_weight"])[1]
    others = [0, 1, 3, 4, 5]
    assert torch.equal(n[others], clean[others]) and bool(torch.isnan(n[2]).all())


def plain(x, b, w, wp, g, scale, p, rng):
    """The formulas on 64-bit leaves, for autograd."""
    def normed(v):
        return v * (v.square().mean(dim=1, keepdim=True) + EPS) ** -0.5
    if b is None:
        return x, normed(x) * w
    d = b if wp is None else normed(b) * wp
    if g is not None:
        d = d * g
    if p > 0:
        d = torch.where(torch.from_numpy(philox.keep(*x.shape, p, *rng)).cuda(), d * philox.kept_factor(p), torch.zeros_like(d))
    y = x + scale * d
    return y, normed(y) * w


@pytest.mark.parametrize("gate", ["none", "channel", "token"])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("K", [40, 1003])
def test_autograd_against_the_formulas_gradient(tr, K, post, gate):
    """In float32 throughout.  Every result is a sum of terms that hold y, r and r' in at most three places each, so their relative errors,
    (C / 2 + 12) u each, come in at most 8 times beside the passes' own C u; the terms' sizes are bounded by the gradient of the sums of sizes: every row's largest."""
    a, dy, dn = make(23, K, torch.float32, torch.float32, True, post, gate, 0.2, seed=8)
    names = [k for k in ("x", "branch", "weight", "post_weight", "gate") if a[k] is not None]
    leaf = {k: a[k].detach().clone().requires_grad_() for k in names}
    y, n = tr.residual_norm(leaf["x"], leaf["branch"], leaf["weight"], leaf.get("post_weight"), leaf.get("gate"), a["scale"], a["p"], a["rng"], EPS)
    got = torch.autograd.grad([y, n], [leaf[k] for k in names], [dy, dn])
    exact = {k: a[k].double().requires_grad_() for k in names}
    wy, wn = plain(exact["x"], exact["branch"], exact["weight"], exact.get("post_weight"), exact.get("gate"), a["scale"], a["p"], a["rng"])
    want = torch.autograd.grad([wy, wn], [exact[k] for k in names], [dy.double(), dn.double()])
    C = K / 1024 + 72
    r = (wy.detach().square().mean(dim=1, keepdim=True) + EPS) ** -0.5
    v, gw = wy.detach() * r, dn.double() * a["weight"].double()
    size = dy.double().abs() + r * (gw.abs() + v.abs() * (gw * v).abs().mean(dim=1, keepdim=True))      # of dx' terms
    rb, h, d, fg, f = parts(a)
    sizes = {"x": size, "weight": (dn.double() * v).abs().sum(dim=0)}
    if post:
        wp = a["post_weight"].double().abs()
        inner = fg.abs() * size * wp
        sizes["branch"] = rb * (inner + h.abs() * (inner * h.abs()).mean(dim=1, keepdim=True))
        sizes["post_weight"] = (fg.abs() * size * h.abs()).sum(dim=0)
    else:
        sizes["branch"] = fg.abs() * size
    if gate != "none":
        sizes["gate"] = (f * d).abs() * size if gate == "token" else ((f * d).abs() * size).sum(dim=0)
    for k, g, t in zip(names, got, want):
        off = (g.double() - t).abs()
        assert bool((off <= sizes[k] * (8 * (C / 2 + 12) + C + 200) * U + 1e-37).all()), (k, (off / (sizes[k] + 1e-37)).max().item())


def test_gradient_against_differences(tr):
    """L(h) = sum y dy + n dn along a direction.  The central difference of the exact function differs from its derivative by what the same difference in 64 bits shows;
    that of the kernel's by the rounding of its terms besides, (C + 16) u of their sizes, over h."""
    K, M, h = 300, 7, 2.0 ** -7
    a, dy, dn = make(M, K, torch.float32, torch.float32, True, True, "channel", 0.2, seed=9)
    names = ("x", "branch", "weight", "post_weight", "gate")
    y, n, stats = tr.ebsp_residual_norm_forward(*(a[k] for k in names[:2]), a["weight"], a["post_weight"], a["gate"], a["scale"], a["p"], a["rng"], EPS)
    grads = tr.ebsp_residual_norm_backward(dy, dn, y, stats, a["branch"], a["weight"], a["post_weight"], a["gate"], a["scale"], a["p"], a["rng"])
    for name, grad in zip(names, grads):
        step = (torch.randn(a[name].shape, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda") * 0.5).to(torch.bfloat16).float()

        def loss(sign, kernel):
            t = {k: a[k] if k != name else (a[k] + sign * h * step) for k in names}
            if kernel:
                y, n, _ = tr.ebsp_residual_norm_forward(t["x"], t["branch"], t["weight"], t["post_weight"], t["gate"], a["scale"], a["p"], a["rng"], EPS)
            else:
                y, n = plain(*(t[k].double() for k in names), a["scale"], a["p"], a["rng"])
            terms = torch.cat([(y.double() * dy.double()).reshape(-1), (n.double() * dn.double()).reshape(-1)])
            return terms.sum(), terms.abs().sum()
        (up, size), (down, _) = loss(1, True), loss(-1, True)
        exact = (loss(1, False)[0] - loss(-1, False)[0]) / (2 * h)
        leaf = {k: a[k].double().requires_grad_(k == name) for k in names}
        wy, wn = plain(*(leaf[k] for k in names), a["scale"], a["p"], a["rng"])
        (slope,) = torch.autograd.grad((wy * dy.double()).sum() + (wn * dn.double()).sum(), leaf[name])
        slope = (slope * step.double()).sum()
        rounding = (K / 1024 + 88) * U * size / h
        tol = (exact - slope).abs() + rounding + (grad.double() * step.double()).abs().sum() * 2000 * U
        assert ((up - down) / (2 * h) - (grad.double() * step.double()).sum()).abs() <= tol, name


def test_autograd_of_parts(tr):
    """Leading dimensions, broadcast gates, transposed operands, only some leaves, the first norm of a model."""
    x, b = torch.randn((2, 5, 96), device="cuda", requires_grad=True), torch.randn((2, 5, 96), device="cuda", requires_grad=True)
    w, g = torch.randn(96, device="cuda", requires_grad=True), torch.randn((2, 1, 96), device="cuda", requires_grad=True)
    y, n = tr.residual_norm(x, b, w, gate=g)
    (y.sum() + (n * n).sum()).backward()
    ref = [t.detach().double().requires_grad_() for t in (x, b, w, g)]
    wy = ref[0] + ref[3] * ref[1]
    wn = wy * (wy.square().mean(dim=-1, keepdim=True) + EPS) ** -0.5 * ref[2]
    (wy.sum() + (wn * wn).sum()).backward()
    for t, s in zip((x, b, w, g), ref):
        assert t.grad.shape == t.shape and torch.allclose(t.grad.double(), s.grad, rtol=1e-4, atol=1e-4)
    first, normed = tr.residual_norm(x, None, w)
    assert first is x
    normed.sum().backward()
    turned = torch.randn((96, 10), device="cuda").t().requires_grad_()
    y, n = tr.residual_norm(turned, torch.ones((10, 96), device="cuda"), w.detach())
    n.sum().backward()                                                       # y has no gradient then
    z = turned.detach().double().requires_grad_()
    s = z + 1
    (s * (s.square().mean(dim=-1, keepdim=True) + EPS) ** -0.5 * w.detach().double()).sum().backward()
    assert torch.allclose(turned.grad.double(), z.grad, rtol=1e-4, atol=1e-5)
    with torch.no_grad():
        y, n = tr.residual_norm(x, b, w)
        assert not y.requires_grad and not n.requires_grad


def test_forward_mode_is_refused(tr):
    import torch.autograd.forward_ad as forward_ad
    x, w = torch.randn((4, 16), device="cuda"), torch.ones(16, device="cuda")
    for mode in (torch.enable_grad, torch.no_grad):
        with mode(), forward_ad.dual_level():
            dual = forward_ad.make_dual(x, torch.ones_like(x))
            with pytest.raises(NotImplementedError):
                tr.residual_norm(dual, x, w)
            with pytest.raises(NotImplementedError):
                tr.dropout(dual, 0.5, (1, 2))


def test_refusals(tr):
    x, b, w = torch.zeros((4, 8), device="cuda"), torch.zeros((4, 8), device="cuda"), torch.ones(8, device="cuda")
    half = torch.zeros((4, 8), device="cuda", dtype=torch.float16)
    for bad in (dict(x=half), dict(x=x[0]), dict(x=None), dict(branch=half), dict(branch=x[:3]), dict(weight=w[:7]), dict(weight=w.double()), dict(weight=None),
                dict(post_weight=w[:7]), dict(post_weight=w.half()), dict(gate=w[:7]), dict(gate=half), dict(gate=3.0), dict(p=0.5), dict(p=-1.0),
                dict(branch=None, gate=w), dict(branch=None, post_weight=w), dict(branch=None, p=0.5, rng=(1, 2)), dict(y=half), dict(n=half),
                dict(stats=torch.zeros((4, 1), device="cuda")), dict(gate=w[None].expand(4, 8))):
        with pytest.raises(ValueError):
            tr.ebsp_residual_norm_forward(**{**dict(x=x, branch=b, weight=w), **bad})
    stats = torch.ones((4, 2), device="cuda")
    for bad in (dict(dy=half), dict(dn=half), dict(y=None), dict(stats=stats[:3]), dict(branch=half), dict(workspace=torch.zeros(8, device="cuda", dtype=torch.uint8)),
                dict(dx=half)):
        with pytest.raises(ValueError):
            tr.ebsp_residual_norm_backward(**{**dict(dy=x, dn=x, y=x, stats=stats, branch=b, weight=w), **bad})
    for bad in (dict(branch=x[:1]), dict(gate=torch.ones((3, 8), device="cuda")), dict(gate=1.0), dict(x=torch.zeros((), device="cuda"))):
        with pytest.raises(ValueError):
            tr.residual_norm(**{**dict(x=x, branch=b, weight=w), **bad})
    from paper_2001_01347_amd.zipline import ZipLineError
    for bad in (dict(scale=float("nan")), dict(eps=-1.0)):
        with pytest.raises(ZipLineError):
            tr.ebsp_residual_norm_forward(x, b, w, **bad)
