"""The training operators of libebsp_zipline.so (see include/ebsp_training.h): what a worker computes between two barriers
and what the server does at one.

``ebsp_*`` bind the C ABI 1:1 like ``zipline`` does: argument checks, ``torch.empty`` for outputs that are not given, the
current stream of the inputs' device, no synchronisation and no fallback.  ``gated_ff`` and ``distill_loss`` are the same
operators as part of an autograd graph.  (As with any torch operator, a HIP graph that captures a backward pass captures its forward
pass too, and no eager graph of the same leaves is alive meanwhile.)
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch
from torch.autograd.forward_ad import unpack_dual

from . import zipline
from .zipline import ZipLineError, _check_buffer, _check_workspace

DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2, "relu": 3, "sigmoid": 4}

EXPORTS = ("ebsp_gated_ff_forward", "ebsp_gated_ff_forward_workspace_bytes", "ebsp_gated_ff_forward_split", "ebsp_gated_ff_workspace_bytes",
           "ebsp_gated_ff_split_workspace_bytes", "ebsp_gated_ff_backward", "ebsp_distill_workspace_bytes",
           "ebsp_distill_forward", "ebsp_distill_backward", "ebsp_distill_loss_grad", "ebsp_merge_pushes")

STATUS_RANGE = 4          # a row's index or label lies beyond the vocabulary
TOP_MAX = 1024            # most teacher entries of a row

_lib = None


def load() -> ctypes.CDLL:
    """The HIP library with this module's entry points declared. Raises if it has not been built."""
    global _lib
    if _lib is None:
        lib = zipline.load()
        vp, i64, i32, sz, c_int = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t, ctypes.c_int
        lib.ebsp_gated_ff_forward.restype = c_int
        lib.ebsp_gated_ff_forward.argtypes = [vp, i64, vp, i64, vp, i64, i64, i64, i64, i32, i32, vp, i64, vp, vp, i64, vp]
        lib.ebsp_gated_ff_forward_workspace_bytes.restype = sz
        lib.ebsp_gated_ff_forward_workspace_bytes.argtypes = [i64, i64, i64, i32]
        lib.ebsp_gated_ff_forward_split.restype = c_int
        lib.ebsp_gated_ff_forward_split.argtypes = lib.ebsp_gated_ff_forward.argtypes[:-1] + [vp, sz, vp]
        lib.ebsp_gated_ff_workspace_bytes.restype = sz
        lib.ebsp_gated_ff_workspace_bytes.argtypes = [i64, i64, i32]
        lib.ebsp_gated_ff_split_workspace_bytes.restype = sz
        lib.ebsp_gated_ff_split_workspace_bytes.argtypes = [i64, i64, i64, i32]
        lib.ebsp_gated_ff_backward.restype = c_int
        lib.ebsp_gated_ff_backward.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, i64, i64, i64, i64, i32, i32, vp, i64, vp, vp,
                                               i64, vp, sz, vp]
        f32 = ctypes.c_float
        lib.ebsp_distill_workspace_bytes.restype = sz
        lib.ebsp_distill_workspace_bytes.argtypes = [i64, i64, i32]
        common = [vp, i64, i64, i64, i32, vp, i32, vp, i32, i64, i32, vp, f32, f32, f32]
        lib.ebsp_distill_forward.restype = c_int
        lib.ebsp_distill_forward.argtypes = common + [vp, vp, vp, vp, sz, vp]
        lib.ebsp_distill_backward.restype = c_int
        lib.ebsp_distill_backward.argtypes = common + [vp, vp, vp, i64, vp]
        lib.ebsp_distill_loss_grad.restype = c_int
        lib.ebsp_distill_loss_grad.argtypes = common + [vp, vp, vp, i64, vp, vp, sz, vp]
        lib.ebsp_merge_pushes.restype = c_int
        lib.ebsp_merge_pushes.argtypes = [vp, i64, i32, i64, i32, vp, vp, vp, f32, f32, i32, vp, vp, vp, i32, vp]
        _lib = lib
    return _lib


_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)         # the same, without an object around it


def _call(name: str, dev: torch.device, *args) -> None:
    fn = getattr(_lib or load(), name)
    if torch.cuda.current_device() == dev.index:
        rc = fn(*args, _current_stream(dev.index))
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, _current_stream(dev.index))
    if rc != zipline.EBSP_OK:
        raise ZipLineError(f"{name} failed ({rc}): {zipline.ebsp_last_error()}")


def _dtype(name: str, t: torch.Tensor) -> int:
    code = DTYPES.get(t.dtype) if isinstance(t, torch.Tensor) else None
    if code is None:
        raise ValueError(f"{name} must be a bfloat16, float16 or float32 tensor")
    return code


def _rows(name: str, t: torch.Tensor, dev: torch.device, dtype: torch.dtype, shape: Tuple[int, int]) -> int:
    """Check a matrix operand; the distance between its rows, in elements."""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.device != dev or t.shape != shape:
        raise ValueError(f"{name} must be a {dtype} tensor of shape {shape} on {dev}")
    rows, length = shape
    if t.is_contiguous():
        return length
    if length > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} must have unit stride along its rows")
    if rows <= 1 or length == 0:
        return length
    if t.stride(0) < length:
        raise ValueError(f"the rows of {name} overlap (an expanded tensor: make it contiguous)")
    return t.stride(0)


def _matrix(name: str, t: torch.Tensor) -> Tuple[int, int]:
    if not isinstance(t, torch.Tensor) or t.dim() != 2 or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor with two dimensions")
    return tuple(t.shape)


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
    ldx, ldwg, ldwu = _rows("x", x, dev, dt, (M, K)), _rows("wg", wg, dev, dt, (F, K)), _rows("wu", wu, dev, dt, (F, K))
    return code, M, K, F, dev, dt, (x.data_ptr(), ldx, wg.data_ptr(), ldwg, wu.data_ptr(), ldwu)


def ebsp_gated_ff_forward(x: torch.Tensor, wg: torch.Tensor, wu: torch.Tensor, act: str = "silu", save: bool = False,
                          h: Optional[torch.Tensor] = None, g: Optional[torch.Tensor] = None, u: Optional[torch.Tensor] = None,
                          workspace: Optional[torch.Tensor] = None):
    """``act(x wg^T) * (x wu^T)`` for x [M, K] and weights [F, K]; see the header.

    Returns ``(h[M, F], g, u)``; with ``save`` g and u are the products [M, F], float32, that ``ebsp_gated_ff_backward`` takes,
    otherwise None.  Rows of the operands may lie any distance apart.  A ``workspace`` smaller than
    ``ebsp_gated_ff_forward_workspace_bytes`` keeps sums whole.  Does not synchronise.
    """
    code, M, K, F, dev, dt, operands = _ff_operands(x, wg, wu)
    act = _activation(act)
    h = _output("h", h, dev, dt, (M, F))
    if save or g is not None or u is not None:
        g, u = _output("g", g, dev, torch.float32, (M, F)), _output("u", u, dev, torch.float32, (M, F))
    if workspace is None:
        need = M > 16 and (_lib or load()).ebsp_gated_ff_forward_workspace_bytes(M, K, F, code)     # (0 for fewer: spare the call)
        if need:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    else:
        _check_workspace(workspace, dev, 0)
    room = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel())
    _call("ebsp_gated_ff_forward_split", dev, *operands, M, K, F, code, act, h.data_ptr(), F,
          None if g is None else g.data_ptr(), None if u is None else u.data_ptr(), F, *room)
    return h, g, u


def ebsp_gated_ff_forward_workspace_bytes(M: int, K: int, F: int, dtype: torch.dtype) -> int:
    return int(load().ebsp_gated_ff_forward_workspace_bytes(M, K, F, DTYPES[dtype]))


def ebsp_gated_ff_workspace_bytes(M: int, F: int, dtype: torch.dtype) -> int:
    return int(load().ebsp_gated_ff_workspace_bytes(M, F, DTYPES[dtype]))


def ebsp_gated_ff_split_workspace_bytes(M: int, K: int, F: int, dtype: torch.dtype) -> int:
    return int(load().ebsp_gated_ff_split_workspace_bytes(M, K, F, DTYPES[dtype]))


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
    ldg = _rows("g", g, dev, torch.float32, (M, F))
    if _rows("u", u, dev, torch.float32, (M, F)) != ldg:
        raise ValueError("g and u must have the same row stride")
    dx = _output("dx", dx, dev, dt, (M, K)) if want_dx else None
    dwg = _output("dwg", dwg, dev, dt, (F, K)) if want_dw else None
    dwu = _output("dwu", dwu, dev, dt, (F, K)) if want_dw else None
    if workspace is None:
        need = ebsp_gated_ff_split_workspace_bytes(M, K, F, dt)
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    else:
        _check_workspace(workspace, dev, ebsp_gated_ff_workspace_bytes(M, F, dt))
    ptr = [None if t is None else t.data_ptr() for t in (dx, dwg, dwu)]
    _call("ebsp_gated_ff_backward", dev, dh.data_ptr(), lddh, *operands, g.data_ptr(), u.data_ptr(), ldg, M, K, F, code, act,
          ptr[0], K, ptr[1], ptr[2], K, workspace.data_ptr(), workspace.numel())
    return dx, dwg, dwu


def ebsp_distill_workspace_bytes(N: int, V: int, dtype: torch.dtype) -> int:
    return int(load().ebsp_distill_workspace_bytes(N, V, DTYPES[dtype]))


def _distill_operands(logits, top_index, top_logit, temperature, kl_weight, labels, ce_weight):
    code = _dtype("logits", logits)
    N, V = _matrix("logits", logits)
    dev = logits.device
    if V < 1:
        raise ValueError("the vocabulary must not be empty")
    ld = _rows("logits", logits, dev, logits.dtype, (N, V))
    if not isinstance(top_index, torch.Tensor) or top_index.dim() != 2 or top_index.dtype not in (torch.int32, torch.int64):
        raise ValueError("top_index must be an int32 or int64 tensor with two dimensions")
    top = int(top_index.shape[1])
    if top > TOP_MAX:
        raise ValueError(f"top_index must have at most {TOP_MAX} entries a row")
    top_code = _dtype("top_logit", top_logit)
    ldt = _rows("top_index", top_index, dev, top_index.dtype, (N, top))
    if _rows("top_logit", top_logit, dev, top_logit.dtype, (N, top)) != ldt:
        raise ValueError("top_index and top_logit must have the same row stride")
    if labels is not None:
        _check_buffer("labels", labels, dev, torch.int64, (N,))
    if not 0 < float(temperature) < float("inf"):
        raise ValueError("temperature must be a positive number")
    return N, V, dev, (logits.data_ptr(), ld, N, V, code, top_index.data_ptr(), top_index.element_size(), top_logit.data_ptr(), top_code, ldt,
                       top, None if labels is None else labels.data_ptr(), float(temperature), float(kl_weight), float(ce_weight))


def _distill_workspace(workspace, N, V, dtype, dev):
    need = ebsp_distill_workspace_bytes(N, V, dtype)
    if workspace is None and need:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    _check_workspace(workspace, dev, need)
    return (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel())


def ebsp_distill_forward(logits: torch.Tensor, top_index: torch.Tensor, top_logit: torch.Tensor, temperature: float = 1.0,
                         kl_weight: float = 1.0, labels: Optional[torch.Tensor] = None, ce_weight: float = 0.0,
                         loss: Optional[torch.Tensor] = None, stats: Optional[torch.Tensor] = None,
                         status: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """The distillation loss of every row of ``logits`` [N, V] from the teacher's entries [N, top]; see the header.

    Returns ``(loss[N], stats[N, 3], status[N])``; ``ebsp_distill_backward`` takes the stats.  Does not synchronise.
    """
    N, V, dev, args = _distill_operands(logits, top_index, top_logit, temperature, kl_weight, labels, ce_weight)
    loss = _output("loss", loss, dev, torch.float32, (N,))
    stats = _output("stats", stats, dev, torch.float32, (N, 3))
    status = _output("status", status, dev, torch.int32, (N,))
    ws = _distill_workspace(workspace, N, V, logits.dtype, dev)
    _call("ebsp_distill_forward", dev, *args, loss.data_ptr(), stats.data_ptr(), status.data_ptr(), *ws)
    return loss, stats, status


def _gradient_place(logits: torch.Tensor, dlogits: Optional[torch.Tensor], dev):
    """The gradient's tensor and row stride: a new one, a contiguous one, or the logits themselves."""
    if dlogits is logits:
        return logits, _rows("logits", logits, dev, logits.dtype, tuple(logits.shape))
    return _output("dlogits", dlogits, dev, logits.dtype, tuple(logits.shape)), int(logits.shape[1])


def ebsp_distill_backward(logits: torch.Tensor, top_index: torch.Tensor, top_logit: torch.Tensor, stats: torch.Tensor, dloss: torch.Tensor,
                          temperature: float = 1.0, kl_weight: float = 1.0, labels: Optional[torch.Tensor] = None, ce_weight: float = 0.0,
                          dlogits: Optional[torch.Tensor] = None):
    """The gradient of ``ebsp_distill_forward`` for the rows' ``dloss`` [N]; ``dlogits`` may be ``logits``; see the header.

    Returns ``dlogits[N, V]``.  Does not synchronise.
    """
    N, V, dev, args = _distill_operands(logits, top_index, top_logit, temperature, kl_weight, labels, ce_weight)
    _check_buffer("stats", stats, dev, torch.float32, (N, 3))
    _check_buffer("dloss", dloss, dev, torch.float32, (N,))
    dlogits, ldd = _gradient_place(logits, dlogits, dev)
    _call("ebsp_distill_backward", dev, *args, stats.data_ptr(), dloss.data_ptr(), dlogits.data_ptr(), ldd)
    return dlogits


def ebsp_distill_loss_grad(logits: torch.Tensor, top_index: torch.Tensor, top_logit: torch.Tensor, dloss: torch.Tensor,
                           temperature: float = 1.0, kl_weight: float = 1.0, labels: Optional[torch.Tensor] = None, ce_weight: float = 0.0,
                           loss: Optional[torch.Tensor] = None, dlogits: Optional[torch.Tensor] = None,
                           status: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Loss and gradient in one call, for a ``dloss`` [N] known beforehand; ``dlogits`` may be ``logits``; see the header.

    Returns ``(loss[N], dlogits[N, V], status[N])``.  Does not synchronise.
    """
    N, V, dev, args = _distill_operands(logits, top_index, top_logit, temperature, kl_weight, labels, ce_weight)
    _check_buffer("dloss", dloss, dev, torch.float32, (N,))
    loss = _output("loss", loss, dev, torch.float32, (N,))
    status = _output("status", status, dev, torch.int32, (N,))
    dlogits, ldd = _gradient_place(logits, dlogits, dev)
    ws = _distill_workspace(workspace, N, V, logits.dtype, dev)
    _call("ebsp_distill_loss_grad", dev, *args, dloss.data_ptr(), loss.data_ptr(), dlogits.data_ptr(), ldd, status.data_ptr(), *ws)
    return loss, dlogits, status


def ebsp_merge_pushes(weights: torch.Tensor, pushes: torch.Tensor, iters: torch.Tensor, lr: float = 1.0, momentum: float = 0.0,
                      nesterov: bool = False, velocity: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                      velocity_out: Optional[torch.Tensor] = None, pull=None):
    """The server's weights after a barrier: ``pushes`` [P, n] merged by ``iters`` [P] as a search returns them; see the header.

    ``weights`` and ``velocity`` are float32 [n]; ``out`` and ``velocity_out`` may be the same tensors.  ``pull`` is the type of
    the rounded copy that the workers fetch, or a tensor for it, or None.  Returns ``(out, velocity_out, pull)``, None in the
    place of what there is not.  Does not synchronise.
    """
    code = _dtype("pushes", pushes)
    P, n = _matrix("pushes", pushes)
    dev = pushes.device
    stride = _rows("pushes", pushes, dev, pushes.dtype, (P, n))
    _check_buffer("weights", weights, dev, torch.float32, (n,))
    _check_buffer("iters", iters, dev, torch.int32, (P,))
    out = _output("out", out, dev, torch.float32, (n,))
    if velocity is not None:
        _check_buffer("velocity", velocity, dev, torch.float32, (n,))
        velocity_out = _output("velocity_out", velocity_out, dev, torch.float32, (n,))
    elif velocity_out is not None or momentum != 0 or nesterov:
        raise ValueError("momentum needs a velocity")
    if isinstance(pull, torch.Tensor):
        _dtype("pull", pull)
        _check_buffer("pull", pull, dev, pull.dtype, (n,))
    elif pull is not None:
        if pull not in DTYPES:
            raise ValueError("pull must be bfloat16, float16, float32 or a tensor of one of them")
        pull = torch.empty((n,), dtype=pull, device=dev)
    ptr = [None if t is None else t.data_ptr() for t in (velocity, velocity_out, pull)]
    _call("ebsp_merge_pushes", dev, pushes.data_ptr(), stride, P, n, code, iters.data_ptr(), weights.data_ptr(), ptr[0], float(lr),
          float(momentum), 1 if nesterov else 0, out.data_ptr(), ptr[1], ptr[2], 0 if pull is None else DTYPES[pull.dtype])
    return out, velocity_out, pull


class _GatedFF(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, wg, wu, act, graph):
        save = graph and any(ctx.needs_input_grad)                           # (those are set with gradients off, too)
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
        return dx, dwg if need[1] else None, dwu if need[2] else None, None, None


def _plain_rows(t: torch.Tensor) -> torch.Tensor:
    """t, or a copy where its rows are not stretches of memory of their own (transposed and expanded tensors)."""
    ok = t.shape[1] <= 1 or t.stride(1) == 1
    return t if ok and (t.shape[0] <= 1 or t.stride(0) >= t.shape[1]) else t.contiguous()


def _has_tangent(*tensors) -> bool:
    return any(isinstance(t, torch.Tensor) and unpack_dual(t).tangent is not None for t in tensors)


def gated_ff(x: torch.Tensor, wg: torch.Tensor, wu: torch.Tensor, act: str = "silu") -> torch.Tensor:
    """``act(x wg^T) * (x wu^T)`` for x [..., K], with gradients for all three tensors.

    All three are of one type, in and outside autocast: nothing is cast.  For the backward pass the two products are kept in float32, 8
    bytes a token and unit.  Forward-mode tangents are refused (NotImplementedError)."""
    if not isinstance(x, torch.Tensor) or x.dim() < 1:
        raise ValueError("x must be a tensor of shape [..., K]")
    rows = _plain_rows(x.reshape(x.shape[:-1].numel(), x.shape[-1]))
    if torch.is_grad_enabled() or _has_tangent(rows, wg, wu):                # with gradients off too, a tangent has to be refused, not lost
        h = _GatedFF.apply(rows, wg, wu, act, torch.is_grad_enabled())
    else:
        h = ebsp_gated_ff_forward(rows, wg, wu, act)[0]                      # (five microseconds less than through autograd)
    return h.reshape(*x.shape[:-1], wg.shape[0])


class _Distill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, top_index, top_logit, temperature, kl_weight, labels, ce_weight):
        loss, stats, _ = ebsp_distill_forward(logits, top_index, top_logit, temperature, kl_weight, labels, ce_weight)
        ctx.save_for_backward(logits, top_index, top_logit, stats, labels)
        ctx.args = temperature, kl_weight, ce_weight
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss):
        logits, top_index, top_logit, stats, labels = ctx.saved_tensors
        temperature, kl_weight, ce_weight = ctx.args
        grad = ebsp_distill_backward(logits, top_index, top_logit, stats, dloss.contiguous(), temperature, kl_weight, labels, ce_weight)
        return grad, None, None, None, None, None, None


def _same_rows(shape: torch.Size, lead: torch.Size) -> bool:
    """Whether rows of these dimensions stand in the order of those of ``lead``: the same but for ones, or all as one dimension."""
    return [n for n in shape if n != 1] in ([n for n in lead if n != 1], [n for n in (lead.numel(),) if n != 1])


def distill_loss(logits: torch.Tensor, top_index: torch.Tensor, top_logit: torch.Tensor, temperature: float = 1.0, kl_weight: float = 1.0,
                 labels: Optional[torch.Tensor] = None, ce_weight: float = 0.0) -> torch.Tensor:
    """The distillation loss of every row [...], for logits [..., V] and teacher entries [..., top], with the logits' gradient.

    The teacher's tensors get none.  Indices and labels must lie in the vocabulary or be negative; those that do not are left
    out (``ebsp_distill_forward`` flags them)."""
    if not isinstance(logits, torch.Tensor) or logits.dim() < 1:
        raise ValueError("logits must be a tensor of shape [..., V]")
    lead = logits.shape[:-1]
    for name, t in (("top_index", top_index), ("top_logit", top_logit)):     # (a reshape alone would take rows in another order)
        if not isinstance(t, torch.Tensor) or t.dim() < 1 or not _same_rows(t.shape[:-1], lead):
            raise ValueError(f"{name} must be a tensor of shape [..., top], with the leading dimensions of logits or with those as one")
    if labels is not None and (not isinstance(labels, torch.Tensor) or not _same_rows(labels.shape, lead)):
        raise ValueError("labels must be a tensor of the leading dimensions of logits, or of those as one")
    rows = _plain_rows(logits.reshape(lead.numel(), logits.shape[-1]))
    entries = [t.reshape(lead.numel(), t.shape[-1]).contiguous() for t in (top_index, top_logit)]
    flat = None if labels is None else labels.reshape(lead.numel()).contiguous()
    return _Distill.apply(rows, *entries, temperature, kl_weight, flat, ce_weight).reshape(lead)
