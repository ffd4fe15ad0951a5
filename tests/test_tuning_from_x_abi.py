"""The backward pass of the residual norm from x: what it refuses before anything touches a device."""
import ctypes
import os

import pytest

NULL, ONE, TWO = (ctypes.c_void_p(n) for n in (0, 256, 512))                # (never dereferenced)
BF16, F16, F32 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    from paper_2001_01347_amd import build, training, zipline
    if not os.path.exists(zipline.LIB_PATH):
        build.build()
    return training.load()


def call(lib, x=ONE, ldx=64, branch=ONE, M=4, stream=BF16, dtype=BF16, gate=ONE, post=ONE, db=TWO, dpost=TWO, dgate=TWO, workspace=ONE, nbytes=1 << 20):
    return lib.ebsp_residual_norm_backward_from_x(ONE, 64, ONE, 64, x, ldx, branch, 64, M, 64, stream, dtype, ONE, post, gate, 0, 1.0, 0.0, 1, 2, NULL,
                                                  ONE, TWO, 64, db, 64, TWO, dpost, dgate, 64, workspace, nbytes, NULL)


def test_refusals(lib):
    import torch
    from paper_2001_01347_amd import zipline
    without = dict(branch=NULL, gate=NULL, post=NULL, db=NULL, dpost=NULL, dgate=NULL)
    for bad, rc in ((without, -6), (dict(stream=F32), -6), (dict(stream=F32, dtype=F32), -6), (dict(stream=F16), -6), (dict(x=NULL), -1), (dict(ldx=63), -6),
                    (dict(x=ctypes.c_void_p(257)), -6), (dict(M=-1), -2), (dict(workspace=NULL), -1), (dict(nbytes=64), -3)):
        assert call(lib, **bad) == rc, bad
        assert zipline.ebsp_last_error()
    if not torch.cuda.is_available():
        assert call(lib) == -5 and "device" in zipline.ebsp_last_error()
