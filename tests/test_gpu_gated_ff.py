"""The gated feed-forward block and its backward pass against the definition in 64 bits (needs an MI355X).

Tolerances.  A result is rounded once to its type: half a step, ``finfo.eps / 2`` of its size, ``u`` below.  Sums of n
products are held in 32 bits: an error of at most ``2 (n + 8) 2^-24`` of the sum of the products' sizes (each addition rounds
once, the matrix cores may round twice).  The activations are off by at most ``2^-20 (1 + |g|)``.  The backward pass starts from g and u
as they were summed (an error of g goes through the activation's curvature, at most 1 in size for all of them) and rounds dg and
du to the type: half a step each.  These bounds hold element by element; as rounding errors are of either sign, their sums' norm is also held to a few u."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = [torch.bfloat16, torch.float16, torch.float32]
ACTS = ["silu", "gelu", "gelu_tanh", "relu", "sigmoid"]


@pytest.fixture(scope="module")
def tr():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2001_01347_amd import training
    training.load()
    return training


def _both(act, g):
    """act(g) and act'(g) in 64 bits."""
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s + g * s * (1 - s)
    if act == "sigmoid":
        s = torch.sigmoid(g)
        return s, s * (1 - s)
    if act == "relu":
        return g.clamp(min=0), (g > 0).double()
    if act == "gelu":
        cdf = 0.5 * torch.special.erfc(-g / math.sqrt(2))
        return g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


class Reference:
    """Results in 64 bits and, beside each, how far off a result may be."""

    def __init__(self, act, x, wg, wu, dh=None):
        u_t = torch.finfo(x.dtype).eps / 2
        tiny = 2.0 ** -24 if x.dtype == torch.float16 else 1e-37            # half a step of the smallest numbers
        x, wg, wu = x.double(), wg.double(), wu.double()
        M, K = x.shape
        F = wg.shape[0]

        def gamma(n):
            return 2 * (n + 8) * 2.0 ** -24
        g, u = x @ wg.t(), x @ wu.t()
        eg, eu = gamma(K) * (x.abs() @ wg.abs().t()), gamma(K) * (x.abs() @ wu.abs().t())
        a, d = _both(act, g)
        ea = 1.2 * eg + 2.0 ** -20 * (1 + g.abs())
        self.h = a * u
        self.h_tol = ea * u.abs() + a.abs() * eu + ea * eu + u_t * (1 + 1e-3) * self.h.abs() + tiny
        if dh is None:
            return
        dh = dh.double()
        rg, ru = eg, eu
        ed = rg + 2.0 ** -20 * (1 + g.abs())
        if act == "relu":
            ed = torch.where(g.abs() <= rg, 1.0, 0.0)                       # the step may be taken on either side
        du, dg = dh * a, dh * u * d
        edu = dh.abs() * (1.2 * rg + 2.0 ** -20 * (1 + g.abs()))
        edg = dh.abs() * (ru * d.abs() + u.abs() * ed + ru * ed)
        edu, edg = edu + u_t * (du.abs() + edu) + tiny, edg + u_t * (dg.abs() + edg) + tiny
        self.dx = dg @ wg + du @ wu
        self.dx_tol = (edg @ wg.abs() + edu @ wu.abs()) * (1 + 1e-3) + gamma(2 * F) * (dg.abs() @ wg.abs() + du.abs() @ wu.abs()) \
            + u_t * (1 + 1e-3) * self.dx.abs() + tiny
        self.dwg, self.dwu = dg.t() @ x, du.t() @ x
        self.dwg_tol = edg.t() @ x.abs() * (1 + 1e-3) + gamma(M) * (dg.abs().t() @ x.abs()) + u_t * (1 + 1e-3) * self.dwg.abs() + tiny
        self.dwu_tol = edu.t() @ x.abs() * (1 + 1e-3) + gamma(M) * (du.abs().t() @ x.abs()) + u_t * (1 + 1e-3) * self.dwu.abs() + tiny


def _compare(got, ref, names, norms=True):
    for name, value in zip(names, got):
        want, tol = getattr(ref, name), getattr(ref, name + "_tol")
        assert value.shape == want.shape
        off = (value.double() - want).abs()
        assert bool((off <= tol).all()), f"{name}: {(off / tol).max().item():.3g} times its bound"
        if norms and value.dtype != torch.float32 and want.numel() > 64:
            u_t = torch.finfo(value.dtype).eps / 2
            rel = (off.norm() / want.norm().clamp(min=1e-30)).item()
            assert rel <= (1.1 if name == "h" else 2.0) * u_t, f"{name}: the error's norm is {rel / u_t:.3g} half steps"


def _inputs(M, K, F, dtype, seed=0, pad=0):
    gen = torch.Generator(device="cuda").manual_seed(1000 * seed + M + 7 * K + 31 * F)

    def matrix(r, c, scale):
        full = torch.full((r, c + 2 * pad), float("nan"), device="cuda", dtype=dtype)     # what lies beside a row must not be read
        full[:, pad:pad + c] = (torch.randn((r, c), generator=gen, device="cuda") * scale).to(dtype)
        return full[:, pad:pad + c]
    return matrix(M, K, 1.0), matrix(F, K, K ** -0.5), matrix(F, K, K ** -0.5), matrix(M, F, 1.0)


def _step(tr, act, x, wg, wu, dh):
    h, g, u = tr.ebsp_gated_ff_forward(x, wg, wu, act, save=True)
    return (h, *tr.ebsp_gated_ff_backward(dh, x, wg, wu, g, u, act))


SHAPES = [(1, 1, 1), (1, 64, 64), (1, 4096, 200), (2, 7, 3), (5, 200, 1000), (15, 8, 40), (16, 64, 16), (17, 130, 65), (31, 513, 96),
          (33, 72, 129), (64, 96, 24), (65, 31, 200), (100, 1000, 330), (130, 64, 128), (257, 520, 70), (300, 128, 514), (1021, 72, 34)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,F", SHAPES)
def test_shapes(tr, M, K, F, dtype):
    act = ACTS[(M + K + F) % len(ACTS)]
    x, wg, wu, dh = _inputs(M, K, F, dtype)
    ref = Reference(act, x, wg, wu, dh)
    _compare(_step(tr, act, x, wg, wu, dh), ref, ("h", "dx", "dwg", "dwu"))
    _compare((tr.ebsp_gated_ff_forward(x, wg, wu, act)[0],), ref, ("h",))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,F", [(512, 512, 640), (1000, 264, 1032), (2050, 520, 390), (1, 520, 2048), (48, 1032, 512)])
def test_larger(tr, M, K, F, dtype):
    x, wg, wu, dh = _inputs(M, K, F, dtype)
    ref = Reference("silu", x, wg, wu, dh)
    _compare(_step(tr, "silu", x, wg, wu, dh), ref, ("h", "dx", "dwg", "dwu"))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTS)
def test_activations(tr, act, dtype):
    x, wg, wu, dh = _inputs(40, 48, 56, dtype, seed=3)
    x = x * 4                                                                # well into both tails
    _compare(_step(tr, act, x, wg, wu, dh), Reference(act, x, wg, wu, dh), ("h", "dx", "dwg", "dwu"), norms=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad", [1, 3, 8])
@pytest.mark.parametrize("M,K,F", [(1, 100, 70), (70, 100, 36), (300, 256, 130), (520, 264, 520)])
def test_rows_apart(tr, M, K, F, dtype, pad):
    """Operands are columns of wider matrices, aligned to 16 bytes or to nothing; NaN lies beside them."""
    x, wg, wu, dh = _inputs(M, K, F, dtype, seed=1, pad=pad)
    ref = Reference("silu", x, wg, wu, dh)
    _compare(_step(tr, "silu", x, wg, wu, dh), ref, ("h", "dx", "dwg", "dwu"))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,F", [(5, 128, 200), (70, 256, 320), (300, 200, 136), (260, 99, 77), (800, 1032, 1304)])
def test_weights_of_different_strides(tr, M, K, F, dtype):
    x, wg, wu, dh = _inputs(M, K, F, dtype, seed=14)
    wide = torch.full((F, K + 40), float("nan"), device="cuda", dtype=dtype)
    for width in (8, 5):                                                     # rows of wu at multiples of 16 bytes and at others
        wide[:, width:width + K] = wu
        ref = Reference("silu", x, wg, wu, dh)
        _compare(_step(tr, "silu", x, wg, wide[:, width:width + K], dh), ref, ("h", "dx", "dwg", "dwu"))
        _compare(_step(tr, "silu", x, wide[:, width:width + K], wg, dh)[1:2], Reference("silu", x, wu, wg, dh), ("dx",))
        wide.fill_(float("nan"))


@pytest.mark.parametrize("M", [3, 40, 200])
def test_not_finite_stays_where_it_belongs(tr, M):
    """An infinity or a NaN in one token, or in one unit's weights, reaches the results that it is part of and no other."""
    K, F = 72, 90
    x, wg, wu, dh = _inputs(M, K, F, torch.bfloat16, seed=2)
    clean = _step(tr, "silu", x, wg, wu, dh)
    x2 = x.clone()
    x2[1, 5], x2[2, 70] = float("inf"), float("nan")
    h, dx, dwg, dwu = _step(tr, "silu", x2, wg, wu, dh)
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    keep[1:3] = False
    assert torch.equal(h[keep], clean[0][keep]) and torch.equal(dx[keep], clean[1][keep])
    assert not torch.isfinite(h[2]).any()
    wg2 = wg.clone()
    wg2[89, 71] = float("nan")
    h = tr.ebsp_gated_ff_forward(x, wg2, wu)[0]
    assert torch.equal(h[:, :89], clean[0][:, :89]) and torch.isnan(h[:, 89]).all()


def test_rows_far_apart(tr):
    """Rows whose offsets pass 32 bits, in elements and in bytes."""
    K, F = 64, 48
    for M, ld in ((17, 1 << 27), (300, 1 << 23)):
        base = torch.empty(M * ld, dtype=torch.bfloat16, device="cuda")
        x0, wg, wu, dh = _inputs(M, K, F, torch.bfloat16, seed=4)
        x = base.view(M, ld)[:, :K]
        x.copy_(x0)
        ref = Reference("silu", x0, wg, wu, dh)
        _compare(_step(tr, "silu", x, wg, wu, dh), ref, ("h", "dx", "dwg", "dwu"))
        del base, x


@pytest.mark.parametrize("dtype", TYPES)
def test_nothing_to_sum(tr, dtype):
    for M, K, F in ((0, 8, 8), (4, 0, 8), (4, 8, 0), (0, 8, 0), (0, 0, 0)):
        x, wg = torch.ones((M, K), dtype=dtype, device="cuda"), torch.ones((F, K), dtype=dtype, device="cuda")
        dh = torch.ones((M, F), dtype=dtype, device="cuda")
        h, dx, dwg, dwu = _step(tr, "sigmoid", x, wg, wg, dh)
        for t, shape in ((h, (M, F)), (dx, (M, K)), (dwg, (F, K)), (dwu, (F, K))):
            assert tuple(t.shape) == shape and bool((t == 0).all())


def test_parts_of_the_backward_pass(tr):
    x, wg, wu, dh = _inputs(50, 64, 72, torch.bfloat16, seed=5)
    h, g, u = tr.ebsp_gated_ff_forward(x, wg, wu, save=True)
    whole = tr.ebsp_gated_ff_backward(dh, x, wg, wu, g, u)
    dx, a, b = tr.ebsp_gated_ff_backward(dh, x, wg, wu, g, u, want_dw=False)
    assert a is None and b is None and torch.equal(dx, whole[0])
    none, dwg, dwu = tr.ebsp_gated_ff_backward(dh, x, wg, wu, g, u, want_dx=False)
    assert none is None and torch.equal(dwg, whole[1]) and torch.equal(dwu, whole[2])


@pytest.mark.parametrize("dtype", TYPES)
def test_differences(tr, dtype):
    """The gradients along a direction against differences of the 64-bit forward pass."""
    for act in ("silu", "gelu", "gelu_tanh", "sigmoid"):
        x, wg, wu, dh = _inputs(33, 40, 50, dtype, seed=6)
        ref = Reference(act, x, wg, wu, dh)
        grads = _step(tr, act, x, wg, wu, dh)[1:]
        gen = torch.Generator(device="cuda").manual_seed(9)
        args = [t.double() for t in (x, wg, wu)]
        for i, name in enumerate(("dx", "dwg", "dwu")):
            d = torch.randn(args[i].shape, generator=gen, device="cuda", dtype=torch.float64)

            def loss(step):
                p = list(args)
                p[i] = p[i] + step * d
                return ((_both(act, p[0] @ p[1].t())[0] * (p[0] @ p[2].t())) * dh.double()).sum()
            eps = 1e-5
            slope = (loss(eps) - loss(-eps)) / (2 * eps)
            off = ((grads[i].double() * d).sum() - slope).abs().item()
            room = (getattr(ref, name + "_tol") * d.abs()).sum().item() + 1e-6 * (getattr(ref, name) * d).abs().sum().item()
            assert off <= room


def test_autograd(tr):
    """As part of a graph: leading dimensions, a gradient that arrives transposed or expanded, parts that need none."""
    x, wg, wu, _ = _inputs(24, 40, 56, torch.float32, seed=7)
    leaves = [t.clone().requires_grad_() for t in (x.reshape(2, 3, 4, 40), wg, wu)]
    out = tr.gated_ff(*leaves, act="gelu")
    assert tuple(out.shape) == (2, 3, 4, 56)
    out.sum().backward()                                                     # an expanded gradient
    ref = Reference("gelu", x, wg, wu, torch.ones((24, 56), device="cuda"))
    _compare([leaves[0].grad.reshape(24, 40), leaves[1].grad, leaves[2].grad], ref, ("dx", "dwg", "dwu"))
    w2 = wg.clone().requires_grad_()
    d = torch.randn((56, 24), device="cuda")
    (tr.gated_ff(x, w2, wu).t() * d).sum().backward()                        # a transposed one
    _compare([w2.grad], Reference("silu", x, wg, wu, d.t()), ("dwg",))
    with torch.no_grad():
        assert not tr.gated_ff(x, w2, wu).requires_grad


def test_streams_and_graphs(tr):
    x, wg, wu, dh = _inputs(70, 128, 96, torch.bfloat16, seed=8)
    want = _step(tr, "silu", x, wg, wu, dh)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _step(tr, "silu", x, wg, wu, dh)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _step(tr, "silu", x, wg, wu, dh)
    for seed in (10, 11, 12):
        for t, new in zip((x, wg, wu, dh), _inputs(70, 128, 96, torch.bfloat16, seed=seed)):
            t.copy_(new)
        want = _step(tr, "silu", x, wg, wu, dh)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


# Few tokens or few units (sums shared out inside a workgroup), gradients whose sums are cut (dx of few tokens, weights' gradients of many),
# large tiles of cut sums.
@pytest.mark.parametrize("M,K,F", [(9, 1024, 48), (16, 1000, 160), (24, 640, 2000), (64, 200, 6000), (80, 2050, 500), (129, 90, 1500), (3000, 64, 72),
                                   (2100, 130, 200), (6000, 40, 9), (4200, 1030, 300)])
@pytest.mark.parametrize("dtype", TYPES)
def test_cut_sums(tr, M, K, F, dtype):
    x, wg, wu, dh = _inputs(M, K, F, dtype, seed=20)
    ref = Reference("silu", x, wg, wu, dh)
    h, g, u = tr.ebsp_gated_ff_forward(x, wg, wu, save=True)
    whole = torch.empty(max(tr.ebsp_gated_ff_workspace_bytes(M, F, dtype), 256), dtype=torch.uint8, device="cuda")
    for workspace in (None, whole):                                          # in parts, and with room for none
        _compare((h, *tr.ebsp_gated_ff_backward(dh, x, wg, wu, g, u, workspace=workspace)), ref, ("h", "dx", "dwg", "dwu"))


@pytest.mark.parametrize("M,K,F", [(40, 2100, 3000), (70, 4096, 1024), (100, 2048, 1001), (129, 2056, 515), (341, 3981, 286), (700, 2049, 70), (2000, 4096, 33),
                                   (513, 1030, 514)])
@pytest.mark.parametrize("dtype", TYPES)
def test_cut_sums_forward(tr, M, K, F, dtype):
    x, wg, wu, dh = _inputs(M, K, F, dtype, seed=22)
    ref = Reference("gelu_tanh", x, wg, wu)
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    saved = []
    for workspace in (None, small):                                          # in parts, and without room for them
        h, g, u = tr.ebsp_gated_ff_forward(x, wg, wu, "gelu_tanh", save=True, workspace=workspace)
        _compare((h,), ref, ("h",))
        for got, w in ((g, wg), (u, wu)):
            bound = 2 * (K + 8) * 2.0 ** -24 * (x.double().abs() @ w.double().abs().t())
            assert bool(((got.double() - x.double() @ w.double().t()).abs() <= bound + 1e-37).all())
        alone = tr.ebsp_gated_ff_forward(x, wg, wu, "gelu_tanh", workspace=workspace)[0]
        assert torch.equal(alone, h)


def test_cut_sums_large_tiles(tr):
    for M, K, F in ((1300, 1300, 6200), (16400, 1032, 770)):                 # 36 large tiles of dx, 40 of dW
        x, wg, wu, dh = _inputs(M, K, F, torch.bfloat16, seed=21)
        ref = Reference("gelu", x, wg, wu, dh)
        _compare(_step(tr, "gelu", x, wg, wu, dh), ref, ("h", "dx", "dwg", "dwu"))


def test_binding_refuses(tr):
    x, wg, wu, dh = _inputs(8, 16, 24, torch.bfloat16)
    h, g, u = tr.ebsp_gated_ff_forward(x, wg, wu, save=True)
    bad = [(x.double(), wg, wu), (x, wg.float(), wu), (x, wg, wu[:8]), (x.t(), wg, wu), (x[0], wg, wu), (x.cpu(), wg, wu),
           (x[:, :8], wg, wu), (x[:1].expand(8, 16), wg, wu), (torch.randn((16, 8), device="cuda").bfloat16().t(), wg, wu)]
    for args in bad:
        with pytest.raises(ValueError):
            tr.ebsp_gated_ff_forward(*args)
    with pytest.raises(ValueError):
        tr.ebsp_gated_ff_forward(x, wg, wu, "tanh")
    with pytest.raises(ValueError):
        tr.ebsp_gated_ff_forward(x, wg, wu, h=torch.empty((8, 25), dtype=torch.bfloat16, device="cuda"))
    for args in ((dh[:, :8], x, wg, wu, g, u), (dh, x, wg, wu, g.half(), u), (dh, x, wg, wu, g, u[:4])):
        with pytest.raises(ValueError):
            tr.ebsp_gated_ff_backward(*args)
    with pytest.raises(ValueError):
        tr.ebsp_gated_ff_backward(dh, x, wg, wu, g, u, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
