"""The merge of the workers' pushes against the definition in 64 bits (needs an MI355X).

Tolerances.  The sum over P workers is held in 32 bits, one rounding a worker, and the shares are rounded once: at most
(P + 2) 2^-24 of the sum of the terms' sizes.  Momentum, step and weight round once each."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = [torch.bfloat16, torch.float16, torch.float32]
U = 2.0 ** -24


@pytest.fixture(scope="module")
def tr():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2001_01347_amd import training
    training.load()
    return training


def make(P, n, dtype, seed=0, stride=None):
    gen = torch.Generator(device="cuda").manual_seed(seed * 101 + P * 13 + n)
    w, v = torch.randn(n, generator=gen, device="cuda"), torch.randn(n, generator=gen, device="cuda")
    pushes = torch.full((P, stride or n), float("nan"), dtype=dtype, device="cuda")[:, :n]
    pushes.copy_(torch.randn((P, n), generator=gen, device="cuda"))
    iters = torch.randint(0, 30, (P,), generator=gen, device="cuda", dtype=torch.int32)
    iters[P // 2] = 7                                                        # somebody has worked
    return w, v, pushes, iters


def check(tr, w, v, pushes, iters, lr, mu, nesterov, pull):
    P = pushes.shape[0]
    on = iters > 0
    c = (iters.clamp(min=0).double() / iters.clamp(min=0).sum())[on][:, None]
    d = pushes[on].double()
    avg, size = (c * d).sum(dim=0), (c * d.abs()).sum(dim=0)
    tol = (P + 2) * U * size + 1e-37
    want_v, v_tol, step = None, None, avg
    if v is not None:
        want_v = mu * v.double() + avg
        v_tol = tol + U * want_v.abs() * 1.001 + 1e-37
        step = avg + mu * want_v if nesterov else want_v
        tol = (tol + mu * v_tol + U * step.abs()) if nesterov else v_tol
    want = w.double() + lr * step
    tol = lr * tol * 1.001 + U * want.abs() + U * (lr * step).abs() + 1e-37
    out, v2, pulled = tr.ebsp_merge_pushes(w, pushes, iters, lr, mu, nesterov, v, pull=pull)
    assert bool(((out.double() - want).abs() <= tol).all())
    if v is not None:
        assert bool(((v2.double() - want_v).abs() <= v_tol).all())
    else:
        assert v2 is None
    assert (pulled is None) if pull is None else torch.equal(pulled, out.to(pull))
    return out, v2, pulled


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("P,n", [(1, 1), (1, 7), (2, 8), (3, 64), (4, 2049), (16, 100003), (17, 5000), (64, 3333), (100, 4096), (1000, 1001), (4096, 70)])
def test_shapes(tr, P, n, dtype):
    w, v, pushes, iters = make(P, n, dtype)
    check(tr, w, None, pushes, iters, 1.0, 0.0, False, None)
    check(tr, w, v, pushes, iters, 0.7, 0.9, False, torch.bfloat16)
    check(tr, w, v, pushes, iters, 0.7, 0.9, True, dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_many_weights(tr, dtype):
    w, v, pushes, iters = make(5, (1 << 22) + 3, dtype, seed=1)
    check(tr, w, v, pushes, iters, 0.5, 0.8, True, torch.float16)


@pytest.mark.parametrize("dtype", TYPES)
def test_workers_far_apart(tr, dtype):
    """Offsets beyond 32 bits, and NaN between the pushes."""
    w, v, pushes, iters = make(9, 3000, dtype, seed=2, stride=(1 << 29) + 1)
    check(tr, w, v, pushes, iters, 1.0, 0.9, False, None)


def test_workers_without_iterations_are_not_read(tr):
    w, v, pushes, iters = make(8, 1000, torch.bfloat16, seed=3)
    iters[2], iters[5], iters[6] = 0, -3, 0
    pushes[2], pushes[5], pushes[6] = float("nan"), float("inf"), float("nan")
    out, v2, _ = check(tr, w, v, pushes, iters, 1.0, 0.5, False, None)
    assert torch.isfinite(out).all()
    iters[:] = 0                                                             # nobody: nothing changes
    out, v2, pulled = tr.ebsp_merge_pushes(w, pushes, iters, 1.0, 0.5, True, v, pull=torch.float16)
    assert torch.equal(out, w) and torch.equal(v2, v) and torch.equal(pulled, w.half())


def test_large_iterations(tr):
    w, v, pushes, iters = make(300, 50, torch.float32, seed=4)
    iters[:] = 2 ** 31 - 1
    check(tr, w, v, pushes, iters, 1.0, 0.0, False, None)


def test_in_place_and_results_that_do_not_vary(tr):
    w, v, pushes, iters = make(33, 10007, torch.bfloat16, seed=5)
    want = tr.ebsp_merge_pushes(w, pushes, iters, 0.7, 0.9, True, v, pull=torch.bfloat16)
    for _ in range(3):
        w2, v2, pull = w.clone(), v.clone(), torch.empty(10007, dtype=torch.bfloat16, device="cuda")
        got = tr.ebsp_merge_pushes(w2, pushes, iters, 0.7, 0.9, True, v2, out=w2, velocity_out=v2, pull=pull)
        assert got[0] is w2 and got[1] is v2 and got[2] is pull
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_any_alignment(tr):
    w, v, pushes, iters = make(6, 1005, torch.bfloat16, seed=6)
    check(tr, w[1:], v[1:], pushes[:, 1:], iters, 0.7, 0.9, False, torch.bfloat16)


def test_streams_and_graphs_with_a_search(tr):
    """The merge takes the iterations where a search leaves them, on the search's stream and inside one graph with it."""
    from paper_2001_01347_amd import workloads, zipline
    ts = torch.from_numpy(workloads.make(2, instances=range(1))).cuda()
    w, v, pushes, _ = make(16, 4099, torch.bfloat16, seed=7)

    def step():
        barrier, iters, wait, status = zipline.ebsp_zipline_batch(ts)
        return tr.ebsp_merge_pushes(w, pushes, iters[0], 0.7, 0.9, False, v)[:2] + (iters,)
    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    check(tr, w, v, pushes, want[2][0].contiguous(), 0.7, 0.9, False, None)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in (1, 2, 3):
        ts.copy_(torch.from_numpy(workloads.make(2, instances=range(seed, seed + 1))))
        pushes.copy_(make(16, 4099, torch.bfloat16, seed=20 + seed)[2])
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_nothing_to_merge(tr):
    out, v, pull = tr.ebsp_merge_pushes(torch.empty(0, device="cuda"), torch.empty((3, 0), device="cuda"),
                                        torch.ones(3, dtype=torch.int32, device="cuda"), pull=torch.float16)
    assert out.shape == (0,) and v is None and pull.shape == (0,)


def test_binding_refuses(tr):
    w, v, pushes, iters = make(4, 100, torch.bfloat16)
    for bad in (dict(weights=w.half()), dict(weights=w[:50]), dict(pushes=pushes.double()), dict(pushes=pushes[0]), dict(pushes=pushes.cpu()),
                dict(pushes=pushes[:1].expand(4, 100)), dict(iters=iters.long()), dict(iters=iters[:3]), dict(velocity=v[:3]), dict(momentum=0.9),
                dict(nesterov=True), dict(pull=torch.int32), dict(pull=torch.empty(99, device="cuda")), dict(out=torch.empty(99, device="cuda")),
                dict(velocity_out=v)):
        with pytest.raises(ValueError):
            tr.ebsp_merge_pushes(**{**dict(weights=w, pushes=pushes, iters=iters), **bad})
    with pytest.raises(RuntimeError):
        big = torch.empty((4097, 4), device="cuda")
        tr.ebsp_merge_pushes(torch.empty(4, device="cuda"), big, torch.ones(4097, dtype=torch.int32, device="cuda"))
