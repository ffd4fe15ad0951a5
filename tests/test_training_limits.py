"""The limits of the training operators' sizes as the headers state them, on the host."""
import ctypes
import os

import pytest

NULL = ctypes.c_void_p(0)
ONE = ctypes.c_void_p(256)           # never dereferenced: the calls below fail validation, or find no device
BF16, F16, F32 = 0, 1, 2
LARGEST = (1 << 31) - 1


@pytest.fixture(scope="module")
def lib():
    from paper_2001_01347_amd import build, training, zipline
    if not os.path.exists(zipline.LIB_PATH):
        build.build()
    return training.load()


@pytest.mark.parametrize("dtype,size", [(BF16, 2), (F16, 2), (F32, 4)])
def test_a_workspace_size_does_not_wrap(lib, dtype, size):
    """What is asked for holds dg and du; sizes whose bytes pass 64 bits are refused."""
    for M in (1, 1000, 1 << 20, 1 << 25, 1 << 28, 1 << 30, LARGEST):
        for F in (1, 4096, 1 << 25, 1 << 28, 1 << 30, LARGEST):
            least = lib.ebsp_gated_ff_workspace_bytes(M, F, dtype)
            split = lib.ebsp_gated_ff_split_workspace_bytes(M, 64, F, dtype)
            if M * F < 1 << 56:
                assert least >= 2 * M * F * size and split >= least
            else:
                assert least == 0 and split == 0
                assert lib.ebsp_gated_ff_backward(ONE, F, ONE, 64, ONE, 64, ONE, 64, ONE, ONE, F, M, 64, F, dtype, 0, ONE, 64, ONE, ONE, 64, ONE,
                                                  1 << 40, NULL) == -2
                assert lib.ebsp_gated_ff_forward(ONE, 64, ONE, 64, ONE, 64, M, 64, F, dtype, 0, ONE, F, NULL, NULL, F, NULL) == -2


@pytest.mark.parametrize("dtype,most", [(BF16, (1 << 34) - 1), (F16, (1 << 34) - 1), (F32, (1 << 34) - 1024)])
def test_a_merge_of_the_most_weights(lib, dtype, most):
    """The largest n that the header names is taken (without a GPU: refused for that alone); one more is refused for its size."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present: the call would run")

    def merge(n):
        return lib.ebsp_merge_pushes(ONE, n, 2, n, dtype, ONE, ONE, NULL, 1.0, 0.0, 0, ONE, NULL, NULL, 0, NULL)
    assert merge(most) == -5 and merge(most + 1) == -2
    per = 256 * (4 if dtype == F32 else 8)                                   # weights of a workgroup; a launch counts its threads in 32 bits
    assert (most + per - 1) // per * 256 <= 0xFFFFFFFF


def test_a_temperature_without_an_inverse(lib):
    """Below some 4e-39 log2(e) / T is infinite, and would make a NaN of the largest logit's distance from itself."""
    def forward(T):
        return lib.ebsp_distill_forward(ONE, 100, 4, 100, BF16, ONE, 8, ONE, BF16, 8, 8, NULL, T, 1.0, 0.0, NULL, ONE, NULL, NULL, 0, NULL)
    # (a temperature that is taken is refused for the missing loss)
    assert forward(1e-39) == -6 and forward(4.2e-39) == -6 and forward(4.3e-39) == -1 and forward(1e-38) == -1
    assert forward(1.0) == -1 and forward(3.4e38) == -1 and forward(0.0) == -6
