"""Loss and gradient in one pass where other tests do not go: rows longer than what a workgroup keeps of them, and rows whose exponents are taken from differences (needs an MI355X).

Checks and tolerances are those of the other tests of these losses.  For rows of far exponents the factor log2(e) / T is off by a step of 2^-24 of itself, and every exponent with it:
``more`` is what that moves logp by, and a gradient's weights move by twice as much of their exponent."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_token_losses import TYPES, U, Reference, check_policy, close, make, policy_inputs  # noqa: E402


@pytest.fixture(scope="module")
def tr():
    assert torch.cuda.is_available(), "these tests need a GPU"
    from paper_2001_01347_amd import training
    training.load()
    return training


# 16-byte words a row: 31 x 512 are kept by one kind of workgroup, 24 x 1024 by the next; what lies behind is read twice
@pytest.mark.parametrize("dtype,N,V", [(torch.bfloat16, 130, 128000), (torch.float16, 97, 127001), (torch.bfloat16, 97, 131072), (torch.float32, 97, 64000), (torch.float32, 130, 65536),
                                       (torch.float32, 97, 63493), (torch.bfloat16, 97, 196609), (torch.float16, 97, 220000), (torch.float32, 97, 100003)])
def test_rows_longer_than_what_is_kept(tr, dtype, N, V):
    for T, low, high, kl, pad in ((1.0, 0.2, 0.28, 0.05, 0), (0.8, 0.1, 0.2, 0.0, 3)):
        logits, tokens, gen = make(N, V, dtype, seed=31, pad=pad, masked=V // 10)
        old, advantage, other, dloss = policy_inputs(Reference(logits, tokens, T), gen, low, high)
        check_policy(tr, logits, tokens, old, advantage, other if kl else None, dloss, T, low, high, kl)


def far_rows(N, V, dtype, T):
    """Rows of exponents around 0, and around 2^21 either way; rows where those are mixed, masked with -inf or with the type's lowest value."""
    gen = torch.Generator(device="cuda").manual_seed(N + 31 * V)
    shift = 2.0 ** 21 * T / 1.4426950408889634
    noise = torch.randn((N, V), generator=gen, device="cuda") * 2.5 * T
    kind = torch.arange(N, device="cuda") % 6
    moved = torch.where((kind == 1) | (kind == 3) | (kind == 5), shift, 0.0) + torch.where(kind == 2, -shift, 0.0)
    logits = (noise + moved[:, None]).to(dtype)
    logits[3::6, ::3] = 0.0                                                  # far below the row's others
    logits[4::6, V // 2:] = float("-inf")
    logits[5::6, 1::2] = torch.finfo(dtype).min
    tokens = torch.randint(0, (V + 3) // 4, (N,), generator=gen, device="cuda") * 2
    tokens[kind == 3] += (tokens[kind == 3] % 3 == 0).long()                 # one that weighs something
    tokens[kind == 3] += (tokens[kind == 3] % 3 == 0).long()
    tokens[N // 2] = -100
    return logits, tokens, gen


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V", [(12, 900), (200, 900), (1030, 900), (1030, 2500), (200, 9000), (97, 24000), (97, 50000), (97, 65000), (97, 127500), (97, 200000), (6, 90000)])
def test_far_rows(tr, N, V, dtype):
    """Every kind of workgroup; the gradient from statistics beside the one of the step."""
    T = 0.01
    logits, tokens, gen = far_rows(N, V, dtype, T)
    ref = Reference(logits, tokens, T)
    z = logits.double() / T
    z = (z - z.amax(dim=1, keepdim=True)).abs().nan_to_num(0, 0, 0)          # (places of -inf weigh nothing)
    more = 2 * U * ((ref.p * z).sum(dim=1) + ref.logp.abs())
    assert bool((ref.logp.abs() < 40).all())
    old, advantage, dloss = (ref.logp - 0.1).float(), torch.randn(N, generator=gen, device="cuda"), torch.randn(N, generator=gen, device="cuda")
    advantage += 0.01 * advantage.sign()
    wide = dict(temperature=T, clip_low=0.9, clip_high=9.0)                  # ratios are e^0.1: inside
    x = torch.exp(ref.logp - old.double())
    elogp = ref.elogp + torch.where(ref.has, more, 0.0)
    slope = torch.where(ref.has, -x * advantage.double(), 0.0)
    eslope = slope.abs() * (elogp + (ref.logp.abs() + old.double().abs()) * U + 12 * U)
    w = dloss.double()
    grad, tol = ref.gradient(slope * w, (eslope + slope.abs() * 4 * U) * w.abs())
    tol = tol + (slope * w / T).abs()[:, None] * ref.p * (z * 2 + more[:, None] / U) * U
    loss, both, logp, status = tr.ebsp_policy_loss_grad(logits, tokens, old, advantage, dloss, **wide)
    one, first, stats, _ = tr.ebsp_policy_forward(logits, tokens, old, advantage, **wide)
    apart = tr.ebsp_policy_backward(logits, tokens, old, advantage, stats, dloss, **wide)
    for l, p, g, what in ((loss, logp, both, "step"), (one, first, apart, "apart")):
        close(p, ref.logp, elogp + 1e-37, "logp, " + what)
        close(l, slope, eslope + slope.abs() * 2 * U + 1e-37, "loss, " + what)
        close(g, grad, tol, "gradient, " + what)
    assert bool((status == 0).all())
    copy = logits.clone()
    assert torch.equal(tr.ebsp_policy_loss_grad(copy, tokens, old, advantage, dloss, dlogits=copy, **wide)[1], both)
