"""Host-side checks of the C ABI of the operators of tuning that need no GPU: workspace sizes, and the refusal of bad arguments
before anything touches a device."""
import ctypes
import os

import pytest

NULL = ctypes.c_void_p(0)
ONE = ctypes.c_void_p(256)           # never dereferenced: every call below fails validation first
TWO = ctypes.c_void_p(512)
ODD = ctypes.c_void_p(257)
BF16, F16, F32 = 0, 1, 2
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    from paper_2001_01347_amd import build, training, zipline
    if not os.path.exists(zipline.LIB_PATH):
        build.build()
    return training.load()


def _error():
    from paper_2001_01347_amd import zipline
    return zipline.ebsp_last_error()


def _norm(lib, x=ONE, ldx=64, branch=ONE, ldb=64, M=4, K=64, stream=BF16, dtype=BF16, weight=ONE, post=NULL, gate=NULL, ldgate=0, scale=1.0,
          eps=1e-6, p=0.0, rng=NULL, y=TWO, ldy=64, n=TWO, ldn=64, stats=ONE):
    return lib.ebsp_residual_norm_forward(x, ldx, branch, ldb, M, K, stream, dtype, weight, post, gate, ldgate, scale, eps, p, 1, 2, rng, y, ldy,
                                          n, ldn, stats, NULL)


def test_residual_norm_forward_refuses(lib):
    for bad, rc in ((dict(M=-1), -2), (dict(K=-1), -2), (dict(M=1 << 31), -2), (dict(K=1 << 30), -2), (dict(dtype=3), -6), (dict(stream=F16), -6),
                    (dict(dtype=F32), -6), (dict(scale=NAN), -6), (dict(scale=INF), -6), (dict(eps=-1.0), -6), (dict(eps=NAN), -6), (dict(p=-0.1), -6),
                    (dict(p=1.1), -6), (dict(p=NAN), -6), (dict(x=NULL), -1), (dict(n=NULL), -1), (dict(y=NULL), -1), (dict(weight=NULL), -1),
                    (dict(branch=NULL, post=ONE), -6), (dict(branch=NULL, gate=ONE), -6), (dict(branch=NULL, p=0.5), -6), (dict(ldx=63), -6),
                    (dict(ldb=63), -6), (dict(ldy=63), -6), (dict(ldn=63), -6), (dict(gate=ONE, ldgate=63), -6), (dict(gate=ONE, ldgate=-1), -6),
                    (dict(y=ONE, ldy=65), -6), (dict(x=ODD), -6), (dict(branch=ODD), -6), (dict(weight=ODD), -6), (dict(post=ODD), -6),
                    (dict(gate=ODD), -6), (dict(y=ODD), -6), (dict(n=ODD), -6), (dict(stats=ctypes.c_void_p(258)), -6),
                    (dict(rng=ctypes.c_void_p(260), p=0.5), -6), (dict(x=ctypes.c_void_p(258), stream=F32), -6),
                    (dict(M=1 << 30, K=20000, ldx=20000, ldb=20000, ldy=20000, ldn=20000), -2)):
        assert _norm(lib, **bad) == rc, bad
        assert _error()
    assert _norm(lib, M=0, x=NULL, n=NULL) == 0 and _norm(lib, K=0, x=NULL, n=NULL) == 0             # nothing to do


def _norm_backward(lib, dy=ONE, lddy=64, dn=ONE, lddn=64, y=ONE, ldy=64, branch=ONE, ldb=64, M=4, K=64, stream=BF16, dtype=BF16, weight=ONE, post=ONE,
                   gate=ONE, ldgate=0, scale=1.0, p=0.0, rng=NULL, stats=ONE, dx=TWO, lddx=64, db=TWO, lddb=64, dw=TWO, dpost=TWO, dgate=TWO, lddgate=64,
                   workspace=ONE, nbytes=1 << 20):
    return lib.ebsp_residual_norm_backward(dy, lddy, dn, lddn, y, ldy, branch, ldb, M, K, stream, dtype, weight, post, gate, ldgate, scale, p, 1, 2, rng,
                                           stats, dx, lddx, db, lddb, dw, dpost, dgate, lddgate, workspace, nbytes, NULL)


def test_residual_norm_backward_refuses(lib):
    need = lib.ebsp_residual_norm_workspace_bytes(4, 64)
    for bad, rc in ((dict(M=-1), -2), (dict(K=1 << 30), -2), (dict(dtype=3), -6), (dict(stream=F16), -6), (dict(scale=NAN), -6), (dict(p=2.0), -6),
                    (dict(y=NULL), -1), (dict(stats=NULL), -1), (dict(weight=NULL), -1), (dict(workspace=NULL), -1), (dict(nbytes=need - 1), -3),
                    (dict(workspace=ctypes.c_void_p(264)), -3), (dict(post=NULL), -6), (dict(gate=NULL), -6), (dict(lddy=63), -6), (dict(lddn=63), -6),
                    (dict(ldy=63), -6), (dict(ldb=63), -6), (dict(lddx=63), -6), (dict(lddb=63), -6), (dict(ldgate=64, lddgate=63), -6),
                    (dict(dx=ONE, lddx=65), -6), (dict(dw=ODD), -6), (dict(dpost=ODD), -6), (dict(dgate=ODD), -6), (dict(dx=ODD), -6),
                    (dict(branch=NULL, post=NULL, gate=NULL, dpost=NULL, dgate=NULL), -6), (dict(p=0.5, branch=NULL, post=NULL, gate=NULL, db=NULL, dpost=NULL,
                                                                                                dgate=NULL), -6)):
        assert _norm_backward(lib, **bad) == rc, bad
        assert _error()
    assert _norm_backward(lib, dx=NULL, db=NULL, dw=NULL, dpost=NULL, dgate=NULL) == 0 and _norm_backward(lib, K=0) == 0      # nothing to do


def test_residual_norm_workspace(lib):
    from paper_2001_01347_amd import training
    ws = lib.ebsp_residual_norm_workspace_bytes
    assert ws(0, 64) == 0 and ws(4, 0) == 0 and ws(-1, 64) == 0 and ws(1 << 31, 64) == 0 and ws(4, 1 << 30) == 0
    for M in (1, 5, 100, 8192, (1 << 31) - 1):
        for K in (1, 8, 9, 1000, 4096, 16384, 16385, (1 << 30) - 1):
            assert ws(M, K) >= 3 * 4 * K and ws(M, K) <= 3 * 4 * (K + 7) * min(M, 1024)
    assert training.ebsp_residual_norm_workspace_bytes(4, 64) == ws(4, 64)


def _dropout(lib, x=ONE, ldx=64, M=4, K=64, dtype=BF16, p=0.5, rng=NULL, out=TWO, ldout=64):
    return lib.ebsp_dropout(x, ldx, M, K, dtype, p, 1, 2, rng, out, ldout, NULL)


def test_dropout_refuses(lib):
    for bad, rc in ((dict(M=-1), -2), (dict(K=-1), -2), (dict(M=1 << 31), -2), (dict(K=1 << 30), -2), (dict(dtype=3), -6), (dict(p=-0.1), -6),
                    (dict(p=1.5), -6), (dict(p=NAN), -6), (dict(x=NULL), -1), (dict(out=NULL), -1), (dict(ldx=63), -6), (dict(ldout=63), -6),
                    (dict(out=ONE, ldout=65), -6), (dict(x=ODD), -6), (dict(out=ODD), -6), (dict(rng=ctypes.c_void_p(260)), -6),
                    (dict(M=(1 << 31) - 1, K=1 << 20, ldx=1 << 20, ldout=1 << 20), -2)):
        assert _dropout(lib, **bad) == rc, bad
        assert _error()
    assert _dropout(lib, M=0, x=NULL) == 0 and _dropout(lib, K=0, x=NULL) == 0


def _tokens(lib, name, logits=ONE, ld=100, N=4, V=100, dtype=BF16, tokens=ONE, T=1.0, old=ONE, advantage=ONE, ref=NULL, low=0.2, high=0.2, kl=0.0,
            loss=ONE, logp=ONE, stats=ONE, status=NULL, outer=ONE, grad=ONE, ldd=100, workspace=NULL, nbytes=0):
    common = (logits, ld, N, V, dtype, tokens, T)
    if name == "logp":
        return lib.ebsp_token_logp(*common, logp, stats, status, workspace, nbytes, NULL)
    if name == "logp_backward":
        return lib.ebsp_token_logp_backward(*common, stats, outer, grad, ldd, NULL)
    common += (old, advantage, ref, low, high, kl)
    if name == "policy":
        return lib.ebsp_policy_forward(*common, loss, logp, stats, status, workspace, nbytes, NULL)
    if name == "policy_backward":
        return lib.ebsp_policy_backward(*common, stats, outer, grad, ldd, NULL)
    return lib.ebsp_policy_loss_grad(*common, outer, loss, logp, grad, ldd, status, workspace, nbytes, NULL)


CALLS = ("logp", "logp_backward", "policy", "policy_backward", "policy_both")


def test_token_losses_refuse(lib):
    need, both_need = lib.ebsp_token_logp_workspace_bytes(2, 100000, BF16), lib.ebsp_policy_workspace_bytes(2, 100000, BF16)
    assert need > 0 and need % 256 == 0 and both_need >= need + 2 * 3 * 4 and both_need % 256 == 0
    wide = dict(N=2, V=100000, ld=100000, ldd=100000)
    for bad, rc in ((dict(N=-1), -2), (dict(V=0), -2), (dict(V=1 << 31), -2), (dict(dtype=3), -6), (dict(T=0.0), -6), (dict(T=-1.0), -6), (dict(T=NAN), -6),
                    (dict(T=INF), -6), (dict(T=1e-39), -6), (dict(logits=NULL), -1), (dict(tokens=NULL), -1), (dict(ld=99), -6), (dict(logits=ODD), -6),
                    (dict(tokens=ctypes.c_void_p(260)), -6), (dict(N=(1 << 31) - 1, V=2, ld=2, ldd=2), -2)):
        for name in CALLS:
            assert _tokens(lib, name, **bad) == rc, (name, bad)
            assert _error()
    for bad, rc in ((dict(old=NULL), -1), (dict(advantage=NULL), -1), (dict(low=-0.1), -6), (dict(low=NAN), -6), (dict(high=-0.1), -6), (dict(high=NAN), -6),
                    (dict(kl=NAN), -6), (dict(kl=INF), -6), (dict(old=ctypes.c_void_p(258)), -6), (dict(ref=ctypes.c_void_p(258)), -6)):
        for name in CALLS[2:]:
            assert _tokens(lib, name, **bad) == rc, (name, bad)
    for name in ("logp_backward", "policy_backward", "policy_both"):
        for bad, rc in ((dict(outer=NULL), -1), (dict(grad=NULL), -1), (dict(ldd=99), -6), (dict(logits=ONE, grad=ONE, ldd=101), -6), (dict(grad=ODD), -6)):
            assert _tokens(lib, name, **bad) == rc, (name, bad)
    for name, size in (("logp", need), ("policy", need), ("policy_both", both_need)):
        assert _tokens(lib, name, **wide) == -1
        assert _tokens(lib, name, workspace=ONE, nbytes=size - 1, **wide) == -3
        assert _tokens(lib, name, workspace=ctypes.c_void_p(264), nbytes=size, **wide) == -3
    for name, bad in (("logp", dict(logp=NULL)), ("policy", dict(loss=NULL)), ("policy_both", dict(loss=NULL)), ("logp_backward", dict(stats=NULL)),
                      ("policy_backward", dict(stats=NULL))):
        assert _tokens(lib, name, **bad) == -1, (name, bad)
    for name in CALLS:
        assert _tokens(lib, name, N=0, logits=NULL, tokens=NULL, grad=NULL, loss=NULL, old=NULL, advantage=NULL) == 0
    for ws in (lib.ebsp_token_logp_workspace_bytes, lib.ebsp_policy_workspace_bytes):
        assert ws(4096, 128000, BF16) == 0 and ws(0, 1000, BF16) == 0 and ws(1, 100, BF16) == 0 and ws(1, 0, BF16) == 0 and ws(1, 100, 3) == 0


def _preference(lib, name, logits=ONE, ld=100, N=4, V=100, dtype=BF16, tokens=ONE, starts=ONE, pairs=2, ref=NULL, beta=0.1, kind=0, smoothing=0.0, mean=0,
                loss=ONE, sums=ONE, saved=ONE, status=NULL, dloss=ONE, grad=ONE, ldd=100, workspace=ONE, nbytes=1 << 20):
    common = (logits, ld, N, V, dtype, tokens, starts, pairs)
    more = (ref, beta, kind, smoothing, mean)
    if name == "forward":
        return lib.ebsp_preference_forward(*common, *more, loss, sums, saved, status, workspace, nbytes, NULL)
    if name == "backward":
        return lib.ebsp_preference_backward(*common, saved, dloss, grad, ldd, NULL)
    return lib.ebsp_preference_loss_grad(*common, *more, dloss, loss, sums, grad, ldd, status, workspace, nbytes, NULL)


def test_preference_loss_refuses(lib):
    from paper_2001_01347_amd import training
    ws = lib.ebsp_preference_workspace_bytes
    need = ws(4, 2, 100, BF16)
    assert need >= 6 * 3 * 4 and need % 256 == 0 and training.ebsp_preference_workspace_bytes(4, 2, 100, __import__("torch").bfloat16) == need
    assert ws(0, 2, 100, BF16) >= 24 and ws(4, -1, 100, BF16) == 0 and ws(4, 2, 100, 3) == 0 and ws(4, 2, 0, BF16) == 0
    for bad, rc in ((dict(N=-1), -2), (dict(V=0), -2), (dict(dtype=3), -6), (dict(logits=NULL), -1), (dict(tokens=NULL), -1), (dict(starts=NULL), -1),
                    (dict(pairs=-1), -2), (dict(pairs=1 << 30), -2), (dict(ld=99), -6), (dict(starts=ctypes.c_void_p(260)), -6), (dict(logits=ODD), -6)):
        for name in ("forward", "backward", "both"):
            assert _preference(lib, name, **bad) == rc, (name, bad)
            assert _error()
    for bad, rc in ((dict(beta=0.0), -6), (dict(beta=-1.0), -6), (dict(beta=INF), -6), (dict(beta=NAN), -6), (dict(kind=3), -6), (dict(kind=-1), -6),
                    (dict(smoothing=-0.1), -6), (dict(smoothing=1.1), -6), (dict(smoothing=NAN), -6), (dict(smoothing=0.1, kind=1), -6),
                    (dict(loss=NULL), -1), (dict(ref=ctypes.c_void_p(258)), -6), (dict(sums=ctypes.c_void_p(258)), -6),
                    (dict(pairs=1 << 29), -2)):
        for name in ("forward", "both"):
            assert _preference(lib, name, **bad) == rc, (name, bad)
    for name in ("backward", "both"):
        for bad, rc in ((dict(dloss=NULL), -1), (dict(grad=NULL), -1), (dict(ldd=99), -6), (dict(logits=ONE, grad=ONE, ldd=101), -6)):
            assert _preference(lib, name, **bad) == rc, (name, bad)
    for name, bad, rc in (("both", dict(nbytes=need - 1), -3), ("both", dict(workspace=NULL), -1), ("forward", dict(saved=NULL, nbytes=need - 1), -3),
                          ("forward", dict(saved=NULL, workspace=NULL), -1), ("backward", dict(saved=NULL), -1),
                          ("both", dict(workspace=ctypes.c_void_p(264)), -3)):
        assert _preference(lib, name, **bad) == rc, (name, bad)
    for name in ("forward", "backward", "both"):
        assert _preference(lib, name, N=0, pairs=0, logits=NULL, tokens=NULL, starts=NULL, grad=NULL) == 0


def test_valid_calls_without_a_gfx950_fail_loudly(lib):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    assert _norm(lib) == -5 and _norm_backward(lib) == -5 and _dropout(lib) == -5
    for name in CALLS:
        assert _tokens(lib, name) == -5, name
    for name in ("forward", "backward", "both"):
        assert _preference(lib, name) == -5, name
    assert "device" in _error()


def test_binding_refuses_cpu_tensors():
    import torch
    from paper_2001_01347_amd import training as tr
    x, w, t, f = torch.zeros((2, 8)), torch.zeros(8), torch.zeros(2, dtype=torch.int64), torch.zeros(2)
    starts = torch.tensor([0, 1, 2])
    for call in (lambda: tr.ebsp_residual_norm_forward(x, x, w), lambda: tr.residual_norm(x, x, w), lambda: tr.ebsp_dropout(x, 0.5, (1, 2)),
                 lambda: tr.dropout(x, 0.5, (1, 2)), lambda: tr.ebsp_token_logp(x, t), lambda: tr.token_logp(x, t),
                 lambda: tr.ebsp_policy_forward(x, t, f, f), lambda: tr.policy_loss(x, t, f, f), lambda: tr.ebsp_preference_forward(x, t, starts),
                 lambda: tr.preference_loss(x, t, starts), lambda: tr.ebsp_residual_norm_backward(x, x, x, x, x, w)):
        with pytest.raises(ValueError):
            call()
