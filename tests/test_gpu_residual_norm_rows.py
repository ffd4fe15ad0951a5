"""The backward pass of the residual norm where a workgroup takes several rows one after the other: wide rows, a gate for every element, dx in the place of dy (needs an MI355X).

Checks and tolerances are those of the other tests of the backward pass, from y and, for streams of 16 bits, from x."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_residual_norm import EPS, check_backward, make  # noqa: E402
from test_gpu_residual_norm_stream import arguments, check  # noqa: E402

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def tr():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2001_01347_amd import training
    training.load()
    return training


def same(a, b):
    return all(s is None and t is None or torch.equal(s, t) for s, t in zip(a, b))


def check_both_ways(tr, a, dy, dn):
    y, n, stats = tr.ebsp_residual_norm_forward(a["x"], a["branch"], *arguments(a), EPS)
    from_y = check_backward(tr, a, dy, dn, y, stats)
    ways = [(y, None, from_y)]
    if a["x"].dtype != F32:
        from_x = tr.ebsp_residual_norm_backward(dy, dn, None, stats, a["branch"], *arguments(a), x=a["x"])
        check(a, dy, dn, stats, from_x)
        ways.append((None, a["x"], from_x))
    for y, x, want in ways:
        place = dy.clone()
        over = tr.ebsp_residual_norm_backward(place, dn, y, stats, a["branch"], *arguments(a), x=x, dx=place)
        assert over[0] is place and same(over, want)
        assert same(tr.ebsp_residual_norm_backward(dy, dn, y, stats, a["branch"], *arguments(a), x=x), want)


@pytest.mark.parametrize("stream,dtype", [(BF16, BF16), (F16, F16), (F32, BF16), (F32, F32)])
@pytest.mark.parametrize("M,K,gate", [(300, 8193, "channel"), (600, 9000, "token"), (700, 12000, "channel"), (300, 16384, "channel"), (300, 16390, "channel"), (600, 16390, "token"),
                                      (300, 20000, "channel")])
def test_wide_rows(tr, M, K, gate, stream, dtype):
    a, dy, dn = make(M, K, stream, dtype, post=True, gate=gate, p=0.1, seed=21)
    check_both_ways(tr, a, dy, dn)


@pytest.mark.parametrize("stream,dtype", [(BF16, BF16), (F32, F16), (F32, F32)])
@pytest.mark.parametrize("M,K", [(70001, 50), (40000, 120), (20001, 255), (16385, 500), (8193, 1000), (4099, 2041), (2051, 4090), (700, 4096), (1300, 200), (700, 8190)])
def test_a_gate_for_every_element(tr, M, K, stream, dtype):
    """In either size of workgroup, for every number of threads a row; the gate comes with each row."""
    a, dy, dn = make(M, K, stream, dtype, post=True, gate="token", p=0.1, seed=22, pad=1)
    check_both_ways(tr, a, dy, dn)


@pytest.mark.parametrize("M,K", [(2051, 4096), (9000, 64)])
def test_without_the_norm_behind_the_block(tr, M, K):
    for gate in ("none", "channel", "token"):
        a, dy, dn = make(M, K, BF16, BF16, post=False, gate=gate, p=0.5, seed=23)
        check_both_ways(tr, a, dy, dn)
