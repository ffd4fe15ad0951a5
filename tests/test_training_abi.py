"""Host-side checks of the training operators' C ABI that need no GPU: exported symbols, the header as C, workspace sizes, and the
refusal of bad arguments before anything touches a device."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "ebsp_training.h")
NULL = ctypes.c_void_p(0)
ONE = ctypes.c_void_p(256)           # never dereferenced: every call below fails validation first
BF16, F16, F32 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    from paper_2001_01347_amd import build, training, zipline
    if not os.path.exists(zipline.LIB_PATH):
        build.build()
    return training.load()


def _error():
    from paper_2001_01347_amd import zipline
    return zipline.ebsp_last_error()


def test_header_symbols_are_exported(lib):
    from paper_2001_01347_amd import training
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(ebsp_[a-z_]+)\s*\(", text)))
    for n in names:
        assert hasattr(lib, n), f"{n} declared in the header but not exported"
    assert sorted(training.EXPORTS) == names


def test_header_is_plain_c(tmp_path):
    src = tmp_path / "training.c"
    src.write_text(f'#include "{HEADER}"\nint main(void) {{ return 0; }}\n')
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Wextra", "-Wpedantic", "-Werror", "-I", os.path.dirname(HEADER), "-fsyntax-only", str(src)],
                   check=True)


def _forward(lib, x=ONE, ldx=64, wg=ONE, ldwg=64, wu=ONE, ldwu=64, M=4, K=64, F=32, dtype=BF16, act=0, h=ONE, ldh=32, g=NULL, u=NULL, ldg=32):
    return lib.ebsp_gated_ff_forward(x, ldx, wg, ldwg, wu, ldwu, M, K, F, dtype, act, h, ldh, g, u, ldg, NULL)


def test_gated_ff_forward_refuses(lib):
    for bad, rc in ((dict(M=-1), -2), (dict(K=-1), -2), (dict(F=-1), -2), (dict(M=1 << 31), -2), (dict(dtype=3), -6), (dict(dtype=-1), -6),
                    (dict(act=5), -6), (dict(act=-1), -6), (dict(x=NULL), -1), (dict(wg=NULL), -1), (dict(wu=NULL), -1), (dict(h=NULL), -1),
                    (dict(g=ONE), -1), (dict(u=ONE), -1), (dict(ldx=63), -6), (dict(ldwg=63), -6), (dict(ldwu=0), -6), (dict(ldh=31), -6),
                    (dict(g=ONE, u=ONE, ldg=31), -6), (dict(ldx=1 << 40), -6), (dict(x=ctypes.c_void_p(257)), -6),
                    (dict(h=ctypes.c_void_p(258), dtype=F32), -6)):
        assert _forward(lib, **bad) == rc, bad
        assert _error()
    assert _forward(lib, M=0, x=NULL, h=NULL) == 0 and _forward(lib, F=0, x=NULL, h=NULL) == 0       # nothing to do


def _backward(lib, dh=ONE, lddh=32, x=ONE, ldx=64, wg=ONE, ldwg=64, wu=ONE, ldwu=64, g=ONE, u=ONE, ldg=32, M=4, K=64, F=32, dtype=BF16, act=0,
              dx=ONE, lddx=64, dwg=ONE, dwu=ONE, lddw=64, workspace=ONE, nbytes=1 << 20):
    return lib.ebsp_gated_ff_backward(dh, lddh, x, ldx, wg, ldwg, wu, ldwu, g, u, ldg, M, K, F, dtype, act, dx, lddx, dwg, dwu, lddw,
                                      workspace, nbytes, NULL)


def test_gated_ff_backward_refuses(lib):
    for bad, rc in ((dict(M=-1), -2), (dict(F=1 << 31), -2), (dict(dtype=9), -6), (dict(act=7), -6), (dict(dh=NULL), -1), (dict(x=NULL), -1),
                    (dict(wg=NULL), -1), (dict(g=NULL), -1), (dict(u=NULL), -1), (dict(dwg=NULL), -1), (dict(dwu=NULL), -1),
                    (dict(workspace=NULL), -1), (dict(lddh=31), -6), (dict(ldg=31), -6), (dict(ldx=63), -6), (dict(ldwu=63), -6),
                    (dict(lddx=63), -6), (dict(lddw=63), -6), (dict(nbytes=511), -3), (dict(workspace=ctypes.c_void_p(264)), -3),
                    (dict(dx=ctypes.c_void_p(257)), -6)):
        assert _backward(lib, **bad) == rc, bad
        assert _error()
    assert _backward(lib, dx=NULL, dwg=NULL, dwu=NULL) == 0 and _backward(lib, K=0) == 0             # nothing to do


def test_gated_ff_workspace(lib):
    from paper_2001_01347_amd import training
    ws = lib.ebsp_gated_ff_workspace_bytes
    assert ws(4, 32, BF16) == 512 and ws(4, 33, BF16) == 768 and ws(1, 1, F32) == 256                # rows padded to 16 bytes, all to 256
    assert ws(0, 32, BF16) == 0 and ws(4, 32, 3) == 0 and ws(-1, 32, BF16) == 0 and ws(1 << 31, 1, BF16) == 0
    assert ws((1 << 31) - 1, 1 << 20, F32) > 1 << 53                                                 # no overflow on the way
    assert training.ebsp_gated_ff_workspace_bytes(4, 32, __import__("torch").bfloat16) == 512


def test_gated_ff_forward_workspace(lib):
    from paper_2001_01347_amd import training
    room = lib.ebsp_gated_ff_forward_workspace_bytes
    assert room(100, 4096, 3000, BF16) >= 2 * 2 * 100 * 3000 * 4                                     # two parts at least of gate and up
    for M, K, F in ((1, 4096, 12288), (8192, 4096, 12288), (64, 64, 64), (0, 4096, 300), (100, 0, 300), (100, 4096, 0), (-1, 8, 8), (1 << 31, 8, 8)):
        assert room(M, K, F, BF16) == 0, (M, K, F)
    assert room(100, 4096, 3000, 3) == 0
    for M in (17, 33, 65, 200, 1000, 5000):
        for K in (1, 1000, 2048, 4096, 9999):
            for F in (1, 64, 301, 5000):
                for dtype in (BF16, F16, F32):
                    assert room(M, K, F, dtype) % 256 == 0
    assert training.ebsp_gated_ff_forward_workspace_bytes(8, 8, 8, __import__("torch").bfloat16) == 0
    split = lib.ebsp_gated_ff_forward_split
    args = (ONE, 64, ONE, 64, ONE, 64, 4, 64, 32, BF16, 0, ONE, 32, NULL, NULL, 32)
    assert split(*args, ctypes.c_void_p(264), 1 << 20, NULL) == -3 and _error()
    assert split(*args[:12], 31, *args[13:], ONE, 1 << 20, NULL) == -6


def test_gated_ff_split_workspace(lib):
    from paper_2001_01347_amd import training
    least, split = lib.ebsp_gated_ff_workspace_bytes, lib.ebsp_gated_ff_split_workspace_bytes
    for M, K, F in ((1, 4096, 12288), (64, 1024, 2048), (8192, 64, 64), (8192, 4096, 12288), (8, 8, 8), (0, 8, 8), (1, 0, 512)):
        for dtype in (BF16, F16, F32):
            assert split(M, K, F, dtype) >= least(M, F, dtype) and split(M, K, F, dtype) % 256 == 0
    assert split(1, 4096, 12288, BF16) > least(1, 12288, BF16)                                       # one row of dx, summed in parts
    assert split(8192, 4096, 12288, BF16) == least(8192, 12288, BF16) and split(8, 8, 8, BF16) == least(8, 8, BF16)
    assert split(4, 8, 32, 3) == 0 and split(-1, 8, 32, BF16) == 0
    assert training.ebsp_gated_ff_split_workspace_bytes(8, 8, 8, __import__("torch").bfloat16) == 256


def test_a_valid_call_without_a_gfx950_fails_loudly(lib):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    assert _forward(lib) == -5 and "device" in _error()
    assert _backward(lib) == -5


def test_binding_refuses_cpu_tensors():
    import torch
    from paper_2001_01347_amd import training
    x, w = torch.zeros((2, 8), dtype=torch.bfloat16), torch.zeros((4, 8), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        training.ebsp_gated_ff_forward(x, w, w)
    with pytest.raises(ValueError):
        training.gated_ff(x, w, w)


def _distill(lib, name="forward", logits=ONE, ld=100, N=4, V=100, dtype=BF16, index=ONE, index_bytes=8, values=ONE, top_dtype=BF16, ldt=8, top=8,
             labels=NULL, T=1.0, loss=ONE, stats=ONE, status=NULL, dloss=ONE, grad=ONE, ldd=100, workspace=NULL, nbytes=0):
    common = (logits, ld, N, V, dtype, index, index_bytes, values, top_dtype, ldt, top, labels, T, 1.0, 0.0)
    if name == "forward":
        return lib.ebsp_distill_forward(*common, loss, stats, status, workspace, nbytes, NULL)
    if name == "backward":
        return lib.ebsp_distill_backward(*common, stats, dloss, grad, ldd, NULL)
    return lib.ebsp_distill_loss_grad(*common, dloss, loss, grad, ldd, status, workspace, nbytes, NULL)


def test_distill_refuses(lib):
    need = lib.ebsp_distill_workspace_bytes(2, 100000, BF16)
    assert need > 0 and need % 256 == 0
    wide = dict(N=2, V=100000, ld=100000, ldd=100000)
    for bad, rc in ((dict(N=-1), -2), (dict(V=0), -2), (dict(V=1 << 31), -2), (dict(top=-1), -2), (dict(top=1025, ldt=1025), -2), (dict(dtype=3), -6),
                    (dict(top_dtype=3), -6), (dict(index_bytes=2), -6), (dict(T=0.0), -6), (dict(T=-1.0), -6), (dict(T=float("nan")), -6),
                    (dict(T=float("inf")), -6), (dict(logits=NULL), -1), (dict(index=NULL), -1), (dict(values=NULL), -1), (dict(ld=99), -6),
                    (dict(ldt=7), -6), (dict(logits=ctypes.c_void_p(257)), -6), (dict(labels=ctypes.c_void_p(260)), -6),
                    (dict(index=ctypes.c_void_p(260)), -6)):
        for name in ("forward", "backward", "both"):
            assert _distill(lib, name, **bad) == rc, (name, bad)
            assert _error()
    for name, bad, rc in (("forward", dict(loss=NULL), -1), ("both", dict(loss=NULL), -1), ("backward", dict(stats=NULL), -1),
                          ("backward", dict(dloss=NULL), -1), ("backward", dict(grad=NULL), -1), ("both", dict(dloss=NULL), -1),
                          ("both", dict(grad=NULL), -1), ("both", dict(ldd=99), -6), ("backward", dict(ldd=99), -6),
                          ("backward", dict(logits=ONE, grad=ONE, ld=100, ldd=101), -6), ("forward", wide, -1),
                          ("forward", dict(workspace=ONE, nbytes=need - 1, **wide), -3), ("both", dict(workspace=ONE, nbytes=need - 1, **wide), -3),
                          ("both", dict(workspace=ctypes.c_void_p(264), nbytes=need, **wide), -3)):
        assert _distill(lib, name, **bad) == rc, (name, bad)
    for name in ("forward", "backward", "both"):
        assert _distill(lib, name, N=0, logits=NULL, loss=NULL, grad=NULL) == 0                      # nothing to do
        assert _distill(lib, name, N=(1 << 31) - 1, V=2, ld=2, ldd=2, top=0) == -2                   # more than a launch holds
    ws = lib.ebsp_distill_workspace_bytes
    assert ws(4096, 128000, BF16) == 0 and ws(0, 1000, BF16) == 0 and ws(1, 100, BF16) == 0 and ws(1, 0, BF16) == 0 and ws(1, 100, 3) == 0


def _merge(lib, pushes=ONE, stride=100, P=4, n=100, dtype=BF16, iters=ONE, weights=ONE, velocity=NULL, out=ONE, velocity_out=NULL, pull=NULL,
           pull_dtype=BF16):
    return lib.ebsp_merge_pushes(pushes, stride, P, n, dtype, iters, weights, velocity, 1.0, 0.0, 0, out, velocity_out, pull, pull_dtype, NULL)


def test_merge_refuses(lib):
    for bad, rc in ((dict(P=0), -2), (dict(P=4097), -2), (dict(n=-1), -2), (dict(n=1 << 34, stride=1 << 34), -2), (dict(dtype=3), -6),
                    (dict(pull=ONE, pull_dtype=3), -6), (dict(pushes=NULL), -1), (dict(iters=NULL), -1), (dict(weights=NULL), -1),
                    (dict(out=NULL), -1), (dict(velocity=ONE), -1), (dict(velocity_out=ONE), -1), (dict(stride=99), -6),
                    (dict(stride=1 << 40), -6), (dict(pushes=ctypes.c_void_p(257)), -6), (dict(iters=ctypes.c_void_p(258)), -6),
                    (dict(pull=ctypes.c_void_p(258), pull_dtype=F32), -6)):
        assert _merge(lib, **bad) == rc, bad
        assert _error()
    assert _merge(lib, n=0, pushes=NULL) == 0


def test_valid_calls_of_the_others_without_a_gfx950_fail_loudly(lib):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    for name in ("forward", "backward", "both"):
        assert _distill(lib, name) == -5
    assert _merge(lib) == -5


def test_binding_refuses_cpu_tensors_of_the_others():
    import torch
    from paper_2001_01347_amd import training
    logits, index, values = torch.zeros((2, 8)), torch.zeros((2, 3), dtype=torch.int64), torch.zeros((2, 3))
    with pytest.raises(ValueError):
        training.ebsp_distill_forward(logits, index, values)
    with pytest.raises(ValueError):
        training.distill_loss(logits, index, values)
    with pytest.raises(ValueError):
        training.ebsp_merge_pushes(torch.zeros(8), torch.zeros((2, 8)), torch.ones(2, dtype=torch.int32))
