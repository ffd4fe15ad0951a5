"""Dropout against the generator written out in Python (needs an MI355X).

A kept element is one product in 32 bits, x times the rounded 65536 / (65536 - t), rounded once to the type: within 2^-23 relative of the exact quotient and half a step."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import philox  # noqa: E402

TYPES = [torch.bfloat16, torch.float16, torch.float32]
RNG = (0x0123456789ABCDEF, 0xFEDCBA9876543210)


@pytest.fixture(scope="module")
def tr():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2001_01347_amd import training
    training.load()
    return training


def expected(x, p, rng):
    keep = torch.from_numpy(philox.keep(x.shape[0], x.shape[1], p, *rng)).to(x.device)
    return torch.where(keep, x.double() * philox.kept_factor(p), 0.0), keep


def check(got, x, p, rng):
    want, keep = expected(x, p, rng)
    u = torch.finfo(x.dtype).eps / 2
    tiny = torch.finfo(x.dtype).smallest_normal * u
    off = (got.double() - want).abs()
    assert bool((off <= want.abs() * (u + 2.0 ** -23) * (1 + u) + tiny).all()), off.max()
    assert bool((got[~keep] == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K", [(1, 1), (1, 7), (1, 8), (1, 9), (3, 64), (61, 1001), (5, 2048), (300, 63), (1000, 8), (2, 70001), (70001, 3), (1029, 2050)])
def test_kept_elements_and_their_values(tr, M, K, dtype):
    gen = torch.Generator(device="cuda").manual_seed(M + 7 * K)
    x = torch.randn((M, K), generator=gen, device="cuda").to(dtype)
    for p in (0.0, 0.1, 0.5, 1.0):
        check(tr.ebsp_dropout(x, p, RNG), x, p, RNG)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_apart_and_in_place(tr, dtype):
    full = torch.full((37, 110), float("nan"), dtype=dtype, device="cuda")
    x = full[:, 3:104]
    x.copy_(torch.randn((37, 101), device="cuda"))
    before = x.clone()
    check(tr.ebsp_dropout(x, 0.3, RNG), before, 0.3, RNG)
    got = tr.ebsp_dropout(x, 0.3, RNG, out=x)
    assert got is x
    check(x, before, 0.3, RNG)
    assert bool(torch.isnan(full[:, :3]).all()) and bool(torch.isnan(full[:, 104:]).all())           # nothing beside the rows


def test_dropped_infinities_and_nan_leave_zeros(tr):
    x = torch.full((16, 256), float("inf"), device="cuda")
    x[::2] = float("nan")
    keep = torch.from_numpy(philox.keep(16, 256, 0.5, 1, 2)).cuda()
    got = tr.ebsp_dropout(x, 0.5, (1, 2))
    assert bool((got[~keep] == 0).all()) and not bool(torch.isfinite(got[keep]).any())


def test_empty(tr):
    assert tr.ebsp_dropout(torch.empty((0, 8), device="cuda"), 0.5, RNG).shape == (0, 8)
    assert tr.ebsp_dropout(torch.empty((8, 0), device="cuda"), 0.5, RNG).shape == (8, 0)
    assert tr.dropout(torch.empty((2, 0, 8), device="cuda"), 0.5, RNG).shape == (2, 0, 8)


def test_gradient_drops_the_same_elements(tr):
    x = torch.randn((4, 5, 96), device="cuda", requires_grad=True)
    dy = torch.randn((4, 5, 96), device="cuda")
    y = tr.dropout(x, 0.25, RNG)
    y.backward(dy)
    keep = torch.from_numpy(philox.keep(20, 96, 0.25, *RNG)).cuda().reshape(4, 5, 96)
    assert torch.equal(y != 0, keep & (x != 0)) and torch.equal(x.grad != 0, keep & (dy != 0))
    check(x.grad.reshape(20, 96), dy.reshape(20, 96), 0.25, RNG)


def test_place_on_the_device_and_in_a_graph(tr):
    """Seed and offset from the device; a replayed graph that moves the offset on draws anew, and the backward pass keeps the forward pass' place."""
    x = torch.randn((33, 200), device="cuda")
    place = torch.tensor([7, 100], dtype=torch.int64, device="cuda")
    assert torch.equal(tr.ebsp_dropout(x, 0.5, place), tr.ebsp_dropout(x, 0.5, (7, 100)))
    high = torch.tensor([-2, -1], dtype=torch.int64, device="cuda")          # the same bits as numbers without a sign
    assert torch.equal(tr.ebsp_dropout(x, 0.5, high), tr.ebsp_dropout(x, 0.5, (2 ** 64 - 2, 2 ** 64 - 1)))
    leaf = x.clone().requires_grad_()
    y = tr.dropout(leaf, 0.5, place)
    place[1] += 1
    y.sum().backward()
    assert torch.equal(leaf.grad != 0, y != 0)
    place[1] = 100
    out = torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        tr.ebsp_dropout(x, 0.5, place, out=out)
        place[1:] += 1
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, tr.ebsp_dropout(x, 0.5, (7, 100 + i))), i
    assert place.tolist() == [7, 104]


def test_refusals(tr):
    x = torch.zeros((4, 8), device="cuda")
    for bad in (dict(p=-0.1), dict(p=1.5), dict(p=float("nan")), dict(rng=None), dict(rng=(-1, 0)), dict(rng=(0, 1 << 64)), dict(x=x[0]), dict(x=x.double()),
                dict(x=None), dict(x=x.t()[:, :2]), dict(x=x[:1].expand(4, 8)), dict(rng=torch.zeros(2, dtype=torch.int64)),
                dict(rng=torch.zeros(3, dtype=torch.int64, device="cuda")), dict(rng=torch.zeros(2, device="cuda")), dict(out=torch.zeros((4, 9), device="cuda")),
                dict(out=torch.zeros((4, 8), device="cuda", dtype=torch.float16))):
        with pytest.raises(ValueError):
            tr.ebsp_dropout(**{**dict(x=x, p=0.5, rng=(1, 2)), **bad})
    with pytest.raises(TypeError):
        tr.ebsp_dropout(x, 0.5, (1.5, 2))
    with pytest.raises(ValueError):
        tr.dropout(torch.zeros((), device="cuda"), 0.5, (1, 2))


@pytest.mark.parametrize("dtype,M,K", [(torch.bfloat16, 8200, 8192), (torch.float32, 4100, 8200), (torch.bfloat16, 8200, 8195), (torch.float32, 40000, 300)])
def test_large_matrices_in_part(tr, dtype, M, K):
    """Those that go past the caches, and those of as many that do not; some rows looked at."""
    x = torch.randn((M, K), device="cuda", dtype=dtype)
    got = tr.ebsp_dropout(x, 0.25, RNG)
    for first in (0, M // 2, M - 3):
        keep = torch.from_numpy(philox.keep(3, K, 0.25, *RNG, first_row=first)).cuda()
        assert torch.equal(got[first:first + 3] != 0, keep & (x[first:first + 3] != 0))
        assert torch.equal(got[first:first + 3], torch.where(keep, (x[first:first + 3].float() * philox.kept_factor(0.25)).to(dtype), 0.0))
