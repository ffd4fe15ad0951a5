"""The training operators of libebsp_zipline.so (see include/ebsp_training.h): what a worker computes between two barriers.

``ebsp_*`` bind the C ABI 1:1 like ``zipline`` does: argument checks, ``torch.empty`` for outputs that are not given, the
current stream of the inputs' device, no synchronisation and no fallback.  ``gated_ff`` is the same operator as part of an
autograd graph.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from . import zipline
from .zipline import ZipLineError, _check_buffer, _check_workspace

DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2, "relu": 3, "sigmoid": 4}

EXPORTS = ("ebsp_gated_ff_forward", "ebsp_gated_ff_workspace_bytes", "ebsp_gated_ff_backward")

_lib = None


def load() -> ctypes.CDLL:
    """The HIP library with this module's entry points declared. Raises if it has not been built."""
    global _lib
    if _lib is None:
        lib = zipline.load()
        vp, i64, i32, sz, c_int = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t, ctypes.c_int
        lib.ebsp_gated_ff_forward.restype = c_int
        lib.ebsp_gated_ff_forward.argtypes = [vp, i64, vp, i64, vp, i64, i64, i64, i64, i32, i32, vp, i64, vp, vp, i64, vp]
        lib.ebsp_gated_ff_workspace_bytes.restype = sz
        lib.ebsp_gated_ff_workspace_bytes.argtypes = [i64, i64, i32]
        lib.ebsp_gated_ff_backward.restype = c_int
        lib.ebsp_gated_ff_backward.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, i64, i64, i64, i64, i32, i32, vp, i64, vp, vp,
                                               i64, vp, sz, vp]
        _lib = lib
    return _lib


def _call(name: str, dev: torch.device, *args) -> None:
    with torch.cuda.device(dev):
        rc = getattr(load(), name)(*args, torch.cuda.current_stream(dev).cuda_stream)
    if rc != zipline.EBSP_OK:
        raise ZipLineError(f"{name} failed ({rc}): {zipline.ebsp_last_error()}")


def _dtype(name: str, t: torch.Tensor) -> int:
    if not isinstance(t, torch.Tensor) or t.dtype not in DTYPES:
        raise ValueError(f"{name} must be a bfloat16, float16 or float32 tensor")
    return DTYPES[t.dtype]


def _rows(name: str, t: torch.Tensor, dev: torch.device, dtype: torch.dtype, shape) -> int:
    """Check a matrix operand; the distance between its rows, in elements."""
    if not isinstance(t, torch.Tensor) or t.device != dev or t.dtype != dtype or tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be a {dtype} tensor of shape {tuple(shape)} on {dev}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} must have unit stride along its rows")
    if t.shape[0] <= 1 or t.shape[1] == 0:
        return t.shape[1]
    if t.stride(0) < t.shape[1]:
        raise ValueError(f"the rows of {name} overlap (an expanded tensor: make it contiguous)")
    return t.stride(0)


def _matrix(name: str, t: torch.Tensor) -> Tuple[int, int]:
    if not isinstance(t, torch.Tensor) or t.dim() != 2 or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor with two dimensions")
    return int(t.shape[0]), int(t.shape[1])


def _output(name: str, t: Optional[torch.Tensor], dev, dtype, shape) -> torch.Tensor:
    if t is None:
        return torch.empty(shape, dtype=dtype, device=dev)
    _check_buffer(name, t, dev, dtype, shape)
    return t


def _activation(act: str) -> int:
    if act not in ACTIVATIONS:
        raise ValueError(f"act must be one of {', '.join(ACTIVATIONS)}")
    return ACTIVATIONS[act]


def _ff_operands(x, wg, wu):
    code = _dtype("x", x)
    M, K = _matrix("x", x)
    F, _ = _matrix("wg", wg)
    dev, dt = x.device, x.dtype
    return code, M, K, F, dev, dt, (x.data_ptr(), _rows("x", x, dev, dt, (M, K)), wg.data_ptr(), _rows("wg", wg, dev, dt, (F, K)),
                                    wu.data_ptr(), _rows("wu", wu, dev, dt, (F, K)))


def ebsp_gated_ff_forward(x: torch.Tensor, wg: torch.Tensor, wu: torch.Tensor, act: str = "silu", save: bool = False,
                          h: Optional[torch.Tensor] = None, g: Optional[torch.Tensor] = None, u: Optional[torch.Tensor] = None):
    """``act(x wg^T) * (x wu^T)`` for x [M, K] and weights [F, K]; see the header.

    Returns ``(h[M, F], g, u)``; with ``save`` g and u are the products [M, F] that ``ebsp_gated_ff_backward`` takes,
    otherwise None.  Rows of the operands may lie any distance apart.  Does not synchronise.
    """
    code, M, K, F, dev, dt, operands = _ff_operands(x, wg, wu)
    act = _activation(act)
    h = _output("h", h, dev, dt, (M, F))
    if save or g is not None or u is not None:
        g, u = _output("g", g, dev, dt, (M, F)), _output("u", u, dev, dt, (M, F))
    _call("ebsp_gated_ff_forward", dev, *operands, M, K, F, code, act, h.data_ptr(), F,
          None if g is None else g.data_ptr(), None if u is None else u.data_ptr(), F)
    return h, g, u


def ebsp_gated_ff_workspace_bytes(M: int, F: int, dtype: torch.dtype) -> int:
    return int(load().ebsp_gated_ff_workspace_bytes(M, F, DTYPES[dtype]))


def ebsp_gated_ff_backward(dh: torch.Tensor, x: torch.Tensor, wg: torch.Tensor, wu: torch.Tensor, g: torch.Tensor, u: torch.Tensor,
                           act: str = "silu", dx: Optional[torch.Tensor] = None, dwg: Optional[torch.Tensor] = None,
                           dwu: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                           want_dx: bool = True, want_dw: bool = True):
    """Gradients of ``ebsp_gated_ff_forward`` from ``dh`` and the products it saved; see the header.

    Returns ``(dx[M, K], dwg[F, K], dwu[F, K])``, None in the place of what is not wanted.  Does not synchronise.
    """
    code, M, K, F, dev, dt, operands = _ff_operands(x, wg, wu)
    act = _activation(act)
    lddh = _rows("dh", dh, dev, dt, (M, F))
    ldg = _rows("g", g, dev, dt, (M, F))
    if _rows("u", u, dev, dt, (M, F)) != ldg:
        raise ValueError("g and u must have the same row stride")
    dx = _output("dx", dx, dev, dt, (M, K)) if want_dx else None
    dwg = _output("dwg", dwg, dev, dt, (F, K)) if want_dw else None
    dwu = _output("dwu", dwu, dev, dt, (F, K)) if want_dw else None
    need = ebsp_gated_ff_workspace_bytes(M, F, dt)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    _check_workspace(workspace, dev, need)
    ptr = [None if t is None else t.data_ptr() for t in (dx, dwg, dwu)]
    _call("ebsp_gated_ff_backward", dev, dh.data_ptr(), lddh, *operands, g.data_ptr(), u.data_ptr(), ldg, M, K, F, code, act,
          ptr[0], K, ptr[1], ptr[2], K, workspace.data_ptr(), workspace.numel())
    return dx, dwg, dwu


class _GatedFF(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, wg, wu, act):
        save = any(ctx.needs_input_grad)
        h, g, u = ebsp_gated_ff_forward(x, wg, wu, act, save=save)
        if save:
            ctx.save_for_backward(x, wg, wu, g, u)
        ctx.act = act
        return h

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dh):
        x, wg, wu, g, u = ctx.saved_tensors
        need = ctx.needs_input_grad
        dx, dwg, dwu = ebsp_gated_ff_backward(_plain_rows(dh), x, wg, wu, g, u, ctx.act, want_dx=need[0], want_dw=need[1] or need[2])
        return dx, dwg if need[1] else None, dwu if need[2] else None, None


def _plain_rows(t: torch.Tensor) -> torch.Tensor:
    """t, or a copy where its rows are not stretches of memory of their own (transposed and expanded tensors)."""
    ok = t.shape[1] <= 1 or t.stride(1) == 1
    return t if ok and (t.shape[0] <= 1 or t.stride(0) >= t.shape[1]) else t.contiguous()


def gated_ff(x: torch.Tensor, wg: torch.Tensor, wu: torch.Tensor, act: str = "silu") -> torch.Tensor:
    """``act(x wg^T) * (x wu^T)`` for x [..., K], with gradients for all three tensors."""
    if not isinstance(x, torch.Tensor) or x.dim() < 1:
        raise ValueError("x must be a tensor of shape [..., K]")
    rows = _plain_rows(x.reshape(-1, x.shape[-1]) if x.shape[-1] > 0 else x.reshape(x.shape[:-1].numel(), 0))
    return _GatedFF.apply(rows, wg, wu, act).reshape(*x.shape[:-1], wg.shape[0])
