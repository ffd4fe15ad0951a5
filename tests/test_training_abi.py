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
