"""The training operators of libebsp_zipline.so (see include/ebsp_training.h): what a worker computes between two barriers
and what the server does at one.

``ebsp_*`` bind the C ABI 1:1 like ``zipline`` does: argument checks, ``torch.empty`` for outputs that are not given, the
current stream of the inputs' device, no synchronisation and no fallback.  ``gated_ff``, ``residual_norm``, ``dropout``, ``distill_loss``,
``token_logp``, ``policy_loss`` and ``preference_loss`` are the same operators as part of an autograd graph.  (As with any torch operator, a HIP graph that captures a backward pass captures its forward
pass too, and no eager graph of the same leaves is alive meanwhile.)
"""
from __future__ import annotations

import ctypes
import functools
import operator
from typing import Optional, Tuple

import torch
from torch.autograd.forward_ad import unpack_dual

from . import zipline
from .zipline import ZipLineError, _check_buffer, _check_workspace

DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
PREFERENCES = {"sigmoid": 0, "hinge": 1, "square": 2}
ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2, "relu": 3, "sigmoid": 4}

EXPORTS = ("ebsp_gated_ff_forward", "ebsp_gated_ff_forward_workspace_bytes", "ebsp_gated_ff_forward_split", "ebsp_gated_ff_workspace_bytes",
           "ebsp_gated_ff_split_workspace_bytes", "ebsp_gated_ff_backward", "ebsp_distill_workspace_bytes",
           "ebsp_distill_forward", "ebsp_distill_backward", "ebsp_distill_loss_grad", "ebsp_merge_pushes",
           "ebsp_residual_norm_workspace_bytes", "ebsp_residual_norm_forward", "ebsp_residual_norm_backward",
           "ebsp_residual_norm_backward_from_x", "ebsp_dropout",
           "ebsp_token_logp_workspace_bytes", "ebsp_token_logp", "ebsp_token_logp_backward", "ebsp_policy_workspace_bytes",
           "ebsp_policy_forward", "ebsp_policy_backward", "ebsp_policy_loss_grad", "ebsp_preference_workspace_bytes",
           "ebsp_preference_forward", "ebsp_preference_backward", "ebsp_preference_loss_grad")

STATUS_RANGE = 4          # a row's index, label or token lies beyond the vocabulary, or the starts of a preference loss are not in order
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
        u64 = ctypes.c_uint64
        random = [f32, u64, u64, vp]
        lib.ebsp_residual_norm_workspace_bytes.restype = sz
        lib.ebsp_residual_norm_workspace_bytes.argtypes = [i64, i64]
        lib.ebsp_residual_norm_forward.restype = c_int
        lib.ebsp_residual_norm_forward.argtypes = [vp, i64, vp, i64, i64, i64, i32, i32, vp, vp, vp, i64, f32, f32] + random + [vp, i64, vp, i64, vp, vp]
        for backward in (lib.ebsp_residual_norm_backward, lib.ebsp_residual_norm_backward_from_x):
            backward.restype = c_int
            backward.argtypes = [vp, i64] * 4 + [i64, i64, i32, i32, vp, vp, vp, i64, f32] + random + [vp, vp, i64, vp, i64, vp, vp, vp, i64, vp, sz, vp]
        lib.ebsp_dropout.restype = c_int
        lib.ebsp_dropout.argtypes = [vp, i64, i64, i64, i32] + random + [vp, i64, vp]
        rows = [vp, i64, i64, i64, i32, vp]
        policy = rows + [f32, vp, vp, vp, f32, f32, f32]
        pairs = rows + [vp, i64]
        lib.ebsp_token_logp_workspace_bytes.restype = lib.ebsp_policy_workspace_bytes.restype = lib.ebsp_preference_workspace_bytes.restype = sz
        lib.ebsp_token_logp_workspace_bytes.argtypes = lib.ebsp_policy_workspace_bytes.argtypes = [i64, i64, i32]
        lib.ebsp_preference_workspace_bytes.argtypes = [i64, i64, i64, i32]
        for name, args in (("ebsp_token_logp", rows + [f32, vp, vp, vp, vp, sz, vp]), ("ebsp_token_logp_backward", rows + [f32, vp, vp, vp, i64, vp]),
                           ("ebsp_policy_forward", policy + [vp, vp, vp, vp, vp, sz, vp]), ("ebsp_policy_backward", policy + [vp, vp, vp, i64, vp]),
                           ("ebsp_policy_loss_grad", policy + [vp, vp, vp, vp, i64, vp, vp, sz, vp]),
                           ("ebsp_preference_forward", pairs + [vp, f32, i32, f32, i32, vp, vp, vp, vp, vp, sz, vp]),
                           ("ebsp_preference_backward", pairs + [vp, vp, vp, i64, vp]),
                           ("ebsp_preference_loss_grad", pairs + [vp, f32, i32, f32, i32, vp, vp, vp, vp, i64, vp, vp, sz, vp])):
            getattr(lib, name).restype = c_int
            getattr(lib, name).argtypes = args
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


def _operand(name: str, t: torch.Tensor) -> Tuple[int, int, int, int]:
    """Check a matrix operand that says what the others are: its type's number, its shape and the distance between its rows."""
    code = _dtype(name, t)
    if t.dim() != 2 or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor with two dimensions")
    M, K = t.shape
    return code, M, K, K if t.is_contiguous() else _rows(name, t, t.device, t.dtype, (M, K))


def _output(name: str, t: Optional[torch.Tensor], dev, dtype, shape) -> torch.Tensor:
    if t is None:
        return torch.empty(shape, dtype=dtype, device=dev)
    _check_buffer(name, t, dev, dtype, shape)
    return t


def _output_like(name: str, t: Optional[torch.Tensor], like: torch.Tensor, dtype) -> torch.Tensor:
    """An output of the shape of a checked operand (a third faster to allocate where it is of its type and layout, too)."""
    if t is None and like.dtype is dtype and like.is_contiguous():
        return torch.empty_like(like)
    return _output(name, t, like.device, dtype, like.shape)


@functools.lru_cache(maxsize=256)
def _bytes(name: str, *sizes: int) -> int:
    """What a size function of the library says: a function of sizes alone."""
    return int(getattr(load(), name)(*sizes))


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


def _random(p: float, rng, dev: torch.device):
    """The four arguments of a dropout: p, seed and offset, or where the two stand on the device."""
    p = float(p)
    if not 0 <= p <= 1:
        raise ValueError("p must be 0 to 1")
    if isinstance(rng, torch.Tensor):
        _check_buffer("rng", rng, dev, torch.int64, (2,))
        return p, 0, 0, rng.data_ptr()
    if rng is None:
        if p > 0:
            raise ValueError("dropout needs rng: a seed and an offset, or an int64 tensor of the two")
        return p, 0, 0, None
    seed, offset = (operator.index(v) for v in rng)                          # (a TypeError for what is no whole number)
    if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
        raise ValueError("seed and offset must be 0 to 2^64 - 1")
    return p, seed, offset, None


def _gate(gate: Optional[torch.Tensor], dev, dtype, M: int, K: int):
    """A gate's pointer and row stride: 0 for one of the channels."""
    if gate is None:
        return None, 0
    if isinstance(gate, torch.Tensor) and gate.dim() == 1:
        _check_buffer("gate", gate, dev, dtype, (K,))
        return gate.data_ptr(), 0
    return gate.data_ptr() if isinstance(gate, torch.Tensor) else None, max(_rows("gate", gate, dev, dtype, (M, K)), 1)


def _norm_operands(branch, M, K, stream, weight, post_weight, gate, scale, p, rng, dev):
    code = _dtype("weight", weight)
    dt = weight.dtype
    if stream != dt and stream != torch.float32:
        raise ValueError("x must be of the weight's type or float32")
    _check_buffer("weight", weight, dev, dt, (K,))
    ldb = K if branch is None else _rows("branch", branch, dev, dt, (M, K))
    if post_weight is not None:
        _check_buffer("post_weight", post_weight, dev, dt, (K,))
    if branch is None and (post_weight is not None or gate is not None or p > 0):
        raise ValueError("post_weight, gate and dropout need a branch")
    pg, ldgate = _gate(gate, dev, dt, M, K)
    return dt, (None if branch is None else branch.data_ptr(), ldb, M, K, DTYPES[stream], code, weight.data_ptr(),
                None if post_weight is None else post_weight.data_ptr(), pg, ldgate, float(scale)), _random(p, rng, dev)


def ebsp_residual_norm_forward(x: torch.Tensor, branch: Optional[torch.Tensor], weight: torch.Tensor, post_weight: Optional[torch.Tensor] = None,
                               gate: Optional[torch.Tensor] = None, scale: float = 1.0, p: float = 0.0, rng=None, eps: float = 1e-6,
                               y: Optional[torch.Tensor] = None, n: Optional[torch.Tensor] = None, stats: Optional[torch.Tensor] = None):
    """The stream ``x`` [M, K] with a block's output ``branch`` [M, K] joined to it, and its norm; see the header.

    ``x`` is of the others' type or float32.  ``gate`` is [K] or [M, K]; ``rng`` a seed and an offset, or an int64 tensor of the two.  Returns
    ``(y[M, K], n[M, K], stats[M, 2])``; without a branch y is x.  ``y`` may be ``x``.  Does not synchronise.
    """
    _, M, K, ldx = _operand("x", x)
    dev = x.device
    dt, operands, random = _norm_operands(branch, M, K, x.dtype, weight, post_weight, gate, scale, p, rng, dev)
    n = _output_like("n", n, x, dt)
    stats = _output("stats", stats, dev, torch.float32, (M, 2))
    if branch is None:
        y, py, ldy = x, None, K
    elif y is x:
        py, ldy = x.data_ptr(), ldx
    else:
        y = _output_like("y", y, x, x.dtype)
        py, ldy = y.data_ptr(), K
    _call("ebsp_residual_norm_forward", dev, x.data_ptr(), ldx, *operands, float(eps), *random, py, ldy, n.data_ptr(), K, stats.data_ptr())
    return y, n, stats


def ebsp_residual_norm_workspace_bytes(M: int, K: int) -> int:
    return int(load().ebsp_residual_norm_workspace_bytes(M, K))


def ebsp_residual_norm_backward(dy: Optional[torch.Tensor], dn: Optional[torch.Tensor], y: Optional[torch.Tensor], stats: torch.Tensor,
                                branch: Optional[torch.Tensor], weight: torch.Tensor, post_weight: Optional[torch.Tensor] = None,
                                gate: Optional[torch.Tensor] = None, scale: float = 1.0, p: float = 0.0, rng=None,
                                dx: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                                want: Tuple[bool, bool, bool, bool, bool] = (True,) * 5, x: Optional[torch.Tensor] = None):
    """Gradients of ``ebsp_residual_norm_forward`` from its ``y`` and ``stats``; ``dy`` or ``dn`` may be None: zero; see the header.

    Of a stream of 16 bits ``y`` was rounded behind its norm: give the forward pass' ``x``, not overwritten since, too, and where there is a branch the stream is formed again from it in 32
    bits, and ``y`` is not looked at.  Returns ``(dx[M, K], dbranch[M, K], dweight[K], dpost_weight[K], dgate)``, None in the place of what there is not or
    ``want`` leaves out.
    ``dx`` may be ``dy``.  Does not synchronise.
    """
    name, kept = "ebsp_residual_norm_backward", "y"
    if x is not None and branch is not None and _dtype("x", x) != DTYPES[torch.float32]:
        if isinstance(y, torch.Tensor) and y.data_ptr() == x.data_ptr() and y.numel():
            raise ValueError("x was overwritten by y: give y alone")
        name, kept, y = "ebsp_residual_norm_backward_from_x", "x", x
    _, M, K, ldy = _operand(kept, y)
    dev, stream = y.device, y.dtype
    dt, operands, random = _norm_operands(branch, M, K, stream, weight, post_weight, gate, scale, p, rng, dev)
    lddy = K if dy is None else _rows("dy", dy, dev, stream, (M, K))
    lddn = K if dn is None else _rows("dn", dn, dev, dt, (M, K))
    _check_buffer("stats", stats, dev, torch.float32, (M, 2))
    lddx = K
    if not want[0]:
        dx = None
    elif dx is not None and dx is dy:
        lddx = lddy
    else:
        dx = _output_like("dx", dx, y, stream)
    outs = [dx, None, None, None, None]
    for i, t in enumerate((branch, weight, post_weight, gate), 1):
        if t is not None and want[i]:
            outs[i] = _output_like("", None, t, dt)
    need = _bytes("ebsp_residual_norm_workspace_bytes", M, K) if outs[2] is not None or outs[3] is not None or outs[4] is not None else 0
    if workspace is None and need:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    _check_workspace(workspace, dev, need)
    ptr = [None if t is None else t.data_ptr() for t in (dy, dn, *outs, workspace)]
    _call(name, dev, ptr[0], lddy, ptr[1], lddn, y.data_ptr(), ldy, *operands, *random, stats.data_ptr(), ptr[2], lddx, ptr[3], K,
          ptr[4], ptr[5], ptr[6], K, ptr[7], 0 if workspace is None else workspace.numel())
    return tuple(outs)


def ebsp_dropout(x: torch.Tensor, p: float, rng, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """``x`` [M, K] over 1 - p where an element is kept, 0 elsewhere; on a gradient, with the same ``rng``, the backward pass; see the header.

    ``rng`` is a seed and an offset, or an int64 tensor of the two.  ``out`` may be ``x``.  Does not synchronise.
    """
    code, M, K, ldx = _operand("x", x)
    dev = x.device
    random = _random(p, rng, dev)
    ldout = ldx if out is x else K
    if out is not x:
        out = _output_like("out", out, x, x.dtype)
    _call("ebsp_dropout", dev, x.data_ptr(), ldx, M, K, code, *random, out.data_ptr(), ldout)
    return out


def _token_operands(logits, tokens, temperature):
    code, N, V, ld = _operand("logits", logits)
    dev = logits.device
    if V < 1:
        raise ValueError("the vocabulary must not be empty")
    _check_buffer("tokens", tokens, dev, torch.int64, (N,))
    if not 0 < float(temperature) < float("inf"):
        raise ValueError("temperature must be a positive number")
    return N, V, code, dev, (logits.data_ptr(), ld, N, V, code, tokens.data_ptr())


def _room(workspace, need: int, dev):
    if workspace is None:
        if not need:
            return None, 0
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    else:
        _check_workspace(workspace, dev, need)
    return workspace.data_ptr(), workspace.numel()


def ebsp_token_logp_workspace_bytes(N: int, V: int, dtype: torch.dtype) -> int:
    return int(load().ebsp_token_logp_workspace_bytes(N, V, DTYPES[dtype]))


def ebsp_token_logp(logits: torch.Tensor, tokens: torch.Tensor, temperature: float = 1.0, logp: Optional[torch.Tensor] = None,
                    stats: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """The log-probability of every row's token, for ``logits`` [N, V] and ``tokens`` [N] (negative: none); see the header.

    Returns ``(logp[N], stats[N, 3], status[N])``; ``ebsp_token_logp_backward`` takes the stats.  Does not synchronise.
    """
    N, V, code, dev, args = _token_operands(logits, tokens, temperature)
    logp = _output("logp", logp, dev, torch.float32, (N,))
    stats = _output("stats", stats, dev, torch.float32, (N, 3))
    status = _output("status", status, dev, torch.int32, (N,))
    room = _room(workspace, _bytes("ebsp_token_logp_workspace_bytes", N, V, code), dev)
    _call("ebsp_token_logp", dev, *args, float(temperature), logp.data_ptr(), stats.data_ptr(), status.data_ptr(), *room)
    return logp, stats, status


def ebsp_token_logp_backward(logits: torch.Tensor, tokens: torch.Tensor, stats: torch.Tensor, dlogp: torch.Tensor, temperature: float = 1.0,
                             dlogits: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient of ``ebsp_token_logp`` for the rows' ``dlogp`` [N]; ``dlogits`` may be ``logits``; see the header.  Does not synchronise."""
    N, V, code, dev, args = _token_operands(logits, tokens, temperature)
    _check_buffer("stats", stats, dev, torch.float32, (N, 3))
    _check_buffer("dlogp", dlogp, dev, torch.float32, (N,))
    dlogits, ldd = _gradient_place(logits, dlogits, dev)
    _call("ebsp_token_logp_backward", dev, *args, float(temperature), stats.data_ptr(), dlogp.data_ptr(), dlogits.data_ptr(), ldd)
    return dlogits


def _policy_operands(N, dev, old_logp, advantage, temperature, clip_low, clip_high, ref_logp, kl_weight):
    _check_buffer("old_logp", old_logp, dev, torch.float32, (N,))
    _check_buffer("advantage", advantage, dev, torch.float32, (N,))
    if ref_logp is not None:
        _check_buffer("ref_logp", ref_logp, dev, torch.float32, (N,))
    elif kl_weight != 0:
        raise ValueError("a KL term needs ref_logp")
    if not (clip_low >= 0 and clip_high >= 0):
        raise ValueError("clip_low and clip_high must not be negative")
    return (float(temperature), old_logp.data_ptr(), advantage.data_ptr(), None if ref_logp is None else ref_logp.data_ptr(), float(clip_low),
            float(clip_high), float(kl_weight))


def ebsp_policy_workspace_bytes(N: int, V: int, dtype: torch.dtype) -> int:
    return int(load().ebsp_policy_workspace_bytes(N, V, DTYPES[dtype]))


def ebsp_policy_forward(logits: torch.Tensor, tokens: torch.Tensor, old_logp: torch.Tensor, advantage: torch.Tensor, temperature: float = 1.0,
                        clip_low: float = 0.2, clip_high: float = 0.2, ref_logp: Optional[torch.Tensor] = None, kl_weight: float = 0.0,
                        loss: Optional[torch.Tensor] = None, logp: Optional[torch.Tensor] = None, stats: Optional[torch.Tensor] = None,
                        status: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """The clipped policy loss of every row's token with its KL term, for ``logits`` [N, V] and float32 [N] of the rest; see the header.

    Returns ``(loss[N], logp[N], stats[N, 3], status[N])``; ``ebsp_policy_backward`` takes the stats.  Does not synchronise.
    """
    N, V, code, dev, args = _token_operands(logits, tokens, temperature)
    policy = _policy_operands(N, dev, old_logp, advantage, temperature, clip_low, clip_high, ref_logp, kl_weight)
    loss, logp = _output("loss", loss, dev, torch.float32, (N,)), _output("logp", logp, dev, torch.float32, (N,))
    stats = _output("stats", stats, dev, torch.float32, (N, 3))
    status = _output("status", status, dev, torch.int32, (N,))
    room = _room(workspace, _bytes("ebsp_token_logp_workspace_bytes", N, V, code), dev)
    _call("ebsp_policy_forward", dev, *args, *policy, loss.data_ptr(), logp.data_ptr(), stats.data_ptr(), status.data_ptr(), *room)
    return loss, logp, stats, status


def ebsp_policy_backward(logits: torch.Tensor, tokens: torch.Tensor, old_logp: torch.Tensor, advantage: torch.Tensor, stats: torch.Tensor,
                         dloss: torch.Tensor, temperature: float = 1.0, clip_low: float = 0.2, clip_high: float = 0.2,
                         ref_logp: Optional[torch.Tensor] = None, kl_weight: float = 0.0, dlogits: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient of ``ebsp_policy_forward`` for the rows' ``dloss`` [N]; ``dlogits`` may be ``logits``; see the header.  Does not synchronise."""
    N, V, code, dev, args = _token_operands(logits, tokens, temperature)
    policy = _policy_operands(N, dev, old_logp, advantage, temperature, clip_low, clip_high, ref_logp, kl_weight)
    _check_buffer("stats", stats, dev, torch.float32, (N, 3))
    _check_buffer("dloss", dloss, dev, torch.float32, (N,))
    dlogits, ldd = _gradient_place(logits, dlogits, dev)
    _call("ebsp_policy_backward", dev, *args, *policy, stats.data_ptr(), dloss.data_ptr(), dlogits.data_ptr(), ldd)
    return dlogits


def ebsp_policy_loss_grad(logits: torch.Tensor, tokens: torch.Tensor, old_logp: torch.Tensor, advantage: torch.Tensor, dloss: torch.Tensor,
                          temperature: float = 1.0, clip_low: float = 0.2, clip_high: float = 0.2, ref_logp: Optional[torch.Tensor] = None,
                          kl_weight: float = 0.0, loss: Optional[torch.Tensor] = None, logp: Optional[torch.Tensor] = None,
                          dlogits: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Loss and gradient in one call, for a ``dloss`` [N] known beforehand; ``dlogits`` may be ``logits``; see the header.

    Returns ``(loss[N], dlogits[N, V], logp[N], status[N])``.  Does not synchronise.
    """
    N, V, code, dev, args = _token_operands(logits, tokens, temperature)
    policy = _policy_operands(N, dev, old_logp, advantage, temperature, clip_low, clip_high, ref_logp, kl_weight)
    _check_buffer("dloss", dloss, dev, torch.float32, (N,))
    loss, logp = _output("loss", loss, dev, torch.float32, (N,)), _output("logp", logp, dev, torch.float32, (N,))
    status = _output("status", status, dev, torch.int32, (N,))
    dlogits, ldd = _gradient_place(logits, dlogits, dev)
    room = _room(workspace, _bytes("ebsp_policy_workspace_bytes", N, V, code), dev)
    _call("ebsp_policy_loss_grad", dev, *args, *policy, dloss.data_ptr(), loss.data_ptr(), logp.data_ptr(), dlogits.data_ptr(), ldd, status.data_ptr(), *room)
    return loss, dlogits, logp, status


def _pairs(starts, dev) -> int:
    if not isinstance(starts, torch.Tensor) or starts.dim() != 1 or starts.shape[0] % 2 != 1:
        raise ValueError("starts must be a tensor with one dimension, of two answers a pair and the end of the last")
    _check_buffer("starts", starts, dev, torch.int64, tuple(starts.shape))
    return starts.shape[0] // 2


def _preference_arguments(ref, pairs, beta, kind, smoothing, mean, dev):
    if ref is not None:
        _check_buffer("ref", ref, dev, torch.float32, (2 * pairs,))
    if kind not in PREFERENCES:
        raise ValueError(f"kind must be one of {', '.join(PREFERENCES)}")
    if not 0 < float(beta) < float("inf"):
        raise ValueError("beta must be a positive number")
    if not 0 <= smoothing <= 1:
        raise ValueError("smoothing must be 0 to 1")
    if smoothing != 0 and kind != "sigmoid":
        raise ValueError("smoothing is of the sigmoid loss alone")
    return None if ref is None else ref.data_ptr(), float(beta), PREFERENCES[kind], float(smoothing), 1 if mean else 0


def ebsp_preference_workspace_bytes(N: int, pairs: int, V: int, dtype: torch.dtype) -> int:
    return int(load().ebsp_preference_workspace_bytes(N, pairs, V, DTYPES[dtype]))


def ebsp_preference_forward(logits: torch.Tensor, tokens: torch.Tensor, starts: torch.Tensor, ref: Optional[torch.Tensor] = None, beta: float = 0.1,
                            kind: str = "sigmoid", smoothing: float = 0.0, mean: bool = False, loss: Optional[torch.Tensor] = None,
                            sums: Optional[torch.Tensor] = None, saved: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                            workspace: Optional[torch.Tensor] = None):
    """The preference loss of pairs of answers, whose rows stand one behind the other in ``logits`` [N, V] from ``starts`` [2 pairs + 1] on; see the header.

    ``tokens`` [N] are negative where a row has none to score, ``ref`` [2 pairs] the answers' sums under a reference.  Returns ``(loss[pairs],
    sums[2 pairs], saved[N + pairs, 3], status[pairs])``; ``ebsp_preference_backward`` takes what is saved.  Does not synchronise.
    """
    N, V, code, dev, args = _token_operands(logits, tokens, 1.0)
    pairs = _pairs(starts, dev)
    more = _preference_arguments(ref, pairs, beta, kind, smoothing, mean, dev)
    loss, sums = _output("loss", loss, dev, torch.float32, (pairs,)), _output("sums", sums, dev, torch.float32, (2 * pairs,))
    saved = _output("saved", saved, dev, torch.float32, (N + pairs, 3))
    status = _output("status", status, dev, torch.int32, (pairs,))
    room = _room(workspace, _bytes("ebsp_token_logp_workspace_bytes", N, V, code), dev)
    _call("ebsp_preference_forward", dev, *args, starts.data_ptr(), pairs, *more, loss.data_ptr(), sums.data_ptr(), saved.data_ptr(), status.data_ptr(), *room)
    return loss, sums, saved, status


def ebsp_preference_backward(logits: torch.Tensor, tokens: torch.Tensor, starts: torch.Tensor, saved: torch.Tensor, dloss: torch.Tensor,
                             dlogits: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient of ``ebsp_preference_forward`` for the pairs' ``dloss``; ``dlogits`` may be ``logits``; see the header.  Does not synchronise."""
    N, V, code, dev, args = _token_operands(logits, tokens, 1.0)
    pairs = _pairs(starts, dev)
    _check_buffer("saved", saved, dev, torch.float32, (N + pairs, 3))
    _check_buffer("dloss", dloss, dev, torch.float32, (pairs,))
    dlogits, ldd = _gradient_place(logits, dlogits, dev)
    _call("ebsp_preference_backward", dev, *args, starts.data_ptr(), pairs, saved.data_ptr(), dloss.data_ptr(), dlogits.data_ptr(), ldd)
    return dlogits


def ebsp_preference_loss_grad(logits: torch.Tensor, tokens: torch.Tensor, starts: torch.Tensor, dloss: torch.Tensor,
                              ref: Optional[torch.Tensor] = None, beta: float = 0.1, kind: str = "sigmoid", smoothing: float = 0.0, mean: bool = False,
                              loss: Optional[torch.Tensor] = None, sums: Optional[torch.Tensor] = None, dlogits: Optional[torch.Tensor] = None,
                              status: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Loss and gradient in one call, for a ``dloss`` [pairs] known beforehand; ``dlogits`` may be ``logits``; see the header.

    Returns ``(loss[pairs], dlogits[N, V], sums[2 pairs], status[pairs])``.  Does not synchronise.
    """
    N, V, code, dev, args = _token_operands(logits, tokens, 1.0)
    pairs = _pairs(starts, dev)
    more = _preference_arguments(ref, pairs, beta, kind, smoothing, mean, dev)
    _check_buffer("dloss", dloss, dev, torch.float32, (pairs,))
    loss, sums = _output("loss", loss, dev, torch.float32, (pairs,)), _output("sums", sums, dev, torch.float32, (2 * pairs,))
    status = _output("status", status, dev, torch.int32, (pairs,))
    dlogits, ldd = _gradient_place(logits, dlogits, dev)
    room = _room(workspace, _bytes("ebsp_preference_workspace_bytes", N, pairs, V, code), dev)
    _call("ebsp_preference_loss_grad", dev, *args, starts.data_ptr(), pairs, *more, dloss.data_ptr(), loss.data_ptr(), sums.data_ptr(), dlogits.data_ptr(),
          ldd, status.data_ptr(), *room)
    return loss, dlogits, sums, status


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


def _flat(name: str, t: torch.Tensor, last: str) -> torch.Tensor:
    """t [..., last] as rows."""
    if not isinstance(t, torch.Tensor) or t.dim() < 1:
        raise ValueError(f"{name} must be a tensor of shape [..., {last}]")
    return _plain_rows(t.reshape(t.shape[:-1].numel(), t.shape[-1]))


def _flat_rows(name: str, t: Optional[torch.Tensor], lead: torch.Size) -> Optional[torch.Tensor]:
    """A value for every row, as one dimension."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not _same_rows(t.shape, lead):
        raise ValueError(f"{name} must be a tensor of the leading dimensions of logits, or of those as one")
    return t.reshape(lead.numel()).contiguous()


def _place(rng):
    """A seed and an offset as they are now, where they are numbers: a program moves its offset on between the passes."""
    return rng if rng is None or isinstance(rng, torch.Tensor) else tuple(rng)


def _kept_place(rng):
    """The same for what stands on the device."""
    return rng.clone() if isinstance(rng, torch.Tensor) else rng


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, p, rng):
        ctx.p, ctx.rng = p, _kept_place(rng) if ctx.needs_input_grad[0] else None
        return ebsp_dropout(x, p, rng)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        return ebsp_dropout(_plain_rows(dy), ctx.p, ctx.rng), None, None


def dropout(x: torch.Tensor, p: float, rng) -> torch.Tensor:
    """Dropout of x [..., K] with its gradient; which elements are kept is computed from ``rng`` in either pass and stored in none.

    ``rng`` is a seed and an offset, or an int64 tensor of the two on x's device (the backward pass uses what either held in the forward pass).  Calls of one
    seed and offset keep the same elements of the same rows: give every call an offset of its own.  Forward-mode tangents are
    refused (NotImplementedError)."""
    return _Dropout.apply(_flat("x", x, "K"), float(p), _place(rng)).reshape(x.shape)


class _ResidualNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, branch, weight, post_weight, gate, scale, p, rng, eps):
        y, n, stats = ebsp_residual_norm_forward(x, branch, weight, post_weight, gate, scale, p, rng, eps)
        if any(ctx.needs_input_grad):
            # the stream, y as it is or formed again from x: of 16 bits y was rounded behind its norm
            ctx.from_x = branch is not None and x.dtype is not torch.float32
            ctx.save_for_backward(x if ctx.from_x else y, stats, branch, weight, post_weight, gate)
            ctx.rng = _kept_place(rng)
        ctx.args = scale, p
        ctx.set_materialize_grads(False)
        return n if branch is None else (y, n)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, *grads):
        kept, stats, branch, weight, post_weight, gate = ctx.saved_tensors
        y, x = (None, kept) if ctx.from_x else (kept, None)
        scale, p = ctx.args
        dy, dn = [None if g is None else _plain_rows(g) for g in ((None, *grads) if branch is None else grads)]
        if dy is None and dn is None:
            return (None,) * 9
        out = ebsp_residual_norm_backward(dy, dn, y, stats, branch, weight, post_weight, gate, scale, p, ctx.rng, want=ctx.needs_input_grad[:5], x=x)
        return (*out, None, None, None, None)


def residual_norm(x: torch.Tensor, branch: Optional[torch.Tensor], weight: torch.Tensor, post_weight: Optional[torch.Tensor] = None,
                  gate: Optional[torch.Tensor] = None, scale: float = 1.0, p: float = 0.0, rng=None, eps: float = 1e-6):
    """A block's output joined to the residual stream, and the norm before the next block, with gradients for all tensors.

    x [..., K] is of the type of the others or float32 and is never cast, under autocast neither; ``branch`` is of its shape, or None in front of the
    first block; ``post_weight`` norms it first; ``gate`` is [K] or broadcasts to x; ``p`` and ``rng`` drop out of it as ``dropout`` does.  Returns the new
    stream and its norm, ``(y, n)``; without a branch ``(x, n)``.  Forward-mode tangents are refused (NotImplementedError)."""
    rows = _flat("x", x, "K")
    if branch is not None:
        if not isinstance(branch, torch.Tensor) or branch.shape != x.shape:
            raise ValueError("branch must be a tensor of the shape of x")
        branch = _flat("branch", branch, "K")
    if gate is not None:
        if not isinstance(gate, torch.Tensor):
            raise ValueError("gate must be a tensor")
        if gate.shape == x.shape[-1:]:
            gate = gate.contiguous()
        else:
            try:
                gate = _flat("gate", gate.expand(x.shape), "K")
            except RuntimeError:
                raise ValueError("gate must broadcast to x") from None
    vectors = [w.contiguous() if isinstance(w, torch.Tensor) else w for w in (weight, post_weight)]
    out = _ResidualNorm.apply(rows, branch, *vectors, gate, float(scale), float(p), _place(rng), eps)
    if branch is None:
        return x, out.reshape(x.shape)
    return out[0].reshape(x.shape), out[1].reshape(x.shape)


class _TokenLogp(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, temperature):
        logp, stats, _ = ebsp_token_logp(logits, tokens, temperature)
        ctx.save_for_backward(logits, tokens, stats)
        ctx.temperature = temperature
        return logp

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dlogp):
        logits, tokens, stats = ctx.saved_tensors
        return ebsp_token_logp_backward(logits, tokens, stats, dlogp.contiguous(), ctx.temperature), None, None


def token_logp(logits: torch.Tensor, tokens: torch.Tensor, temperature: float = 1.0) -> torch.Tensor:
    """The log-probability [...] of every row's token, for logits [..., V] and tokens [...], with the logits' gradient.

    Rows with a negative token have none: 0, without a gradient.  So do those whose token lies beyond the vocabulary
    (``ebsp_token_logp`` flags them)."""
    rows = _flat("logits", logits, "V")
    lead = logits.shape[:-1]
    if tokens is None:
        raise ValueError("tokens must be a tensor of the leading dimensions of logits, or of those as one")
    return _TokenLogp.apply(rows, _flat_rows("tokens", tokens, lead), float(temperature)).reshape(lead)


class _Policy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, old_logp, advantage, ref_logp, *args):
        temperature, clip_low, clip_high, kl_weight = args
        loss, _, stats, _ = ebsp_policy_forward(logits, tokens, old_logp, advantage, temperature, clip_low, clip_high, ref_logp, kl_weight)
        ctx.save_for_backward(logits, tokens, old_logp, advantage, ref_logp, stats)
        ctx.args = args
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss):
        logits, tokens, old_logp, advantage, ref_logp, stats = ctx.saved_tensors
        temperature, clip_low, clip_high, kl_weight = ctx.args
        grad = ebsp_policy_backward(logits, tokens, old_logp, advantage, stats, dloss.contiguous(), temperature, clip_low, clip_high, ref_logp, kl_weight)
        return (grad,) + (None,) * 8


def policy_loss(logits: torch.Tensor, tokens: torch.Tensor, old_logp: torch.Tensor, advantage: torch.Tensor, temperature: float = 1.0,
                clip_low: float = 0.2, clip_high: float = 0.2, ref_logp: Optional[torch.Tensor] = None, kl_weight: float = 0.0) -> torch.Tensor:
    """The clipped policy loss [...] of every row's token with its KL term, for logits [..., V], with the logits' gradient.

    ``tokens`` (negative: none), ``old_logp``, ``advantage`` and ``ref_logp`` are [...], the last three float32 without gradients."""
    rows = _flat("logits", logits, "V")
    lead = logits.shape[:-1]
    named = [("tokens", tokens), ("old_logp", old_logp), ("advantage", advantage)]
    for name, t in named:
        if t is None:
            raise ValueError(f"{name} must be a tensor of the leading dimensions of logits, or of those as one")
    flat = [_flat_rows(name, t, lead) for name, t in (*named, ("ref_logp", ref_logp))]
    return _Policy.apply(rows, *flat, float(temperature), float(clip_low), float(clip_high), float(kl_weight)).reshape(lead)


class _Preference(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, starts, ref, *args):
        loss, _, saved, _ = ebsp_preference_forward(logits, tokens, starts, ref, *args)
        ctx.save_for_backward(logits, tokens, starts, saved)
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss):
        logits, tokens, starts, saved = ctx.saved_tensors
        return (ebsp_preference_backward(logits, tokens, starts, saved, dloss.contiguous()),) + (None,) * 7


def preference_loss(logits: torch.Tensor, tokens: torch.Tensor, starts: torch.Tensor, ref: Optional[torch.Tensor] = None, beta: float = 0.1,
                    kind: str = "sigmoid", smoothing: float = 0.0, mean: bool = False) -> torch.Tensor:
    """The preference loss [pairs] of pairs of answers, for the rows [N, V] of all answers one behind the other, with the logits' gradient.

    ``starts`` [2 pairs + 1] says where each answer begins (the preferred one of a pair first) and where the last ends; ``tokens`` [N] are negative
    where a row has none to score; ``ref`` [2 pairs] are the answers' sums under a reference, float32.  Tokens out of range are
    left out (``ebsp_preference_forward`` flags their pairs); where a start is out of range or below the one before there is no gradient (it flags all)."""
    if not isinstance(logits, torch.Tensor) or logits.dim() != 2:
        raise ValueError("logits must be a tensor of shape [N, V]")
    return _Preference.apply(_plain_rows(logits), tokens, starts, ref, beta, kind, smoothing, mean)
