"""ctypes binding of the C ABI in ``include/dropit_layers.h`` -- marshalling and checks only.

The operators that stand beside the dropped cache in a training step: the gated projection of a feed-forward block
and its backward pass, the AdamW step over many tensors, the global gradient norm.  Functions have the names of the C entry points without the ``dropit_`` prefix; the
formulas stand in the header.
"""
from __future__ import annotations

import ctypes
import math
import struct
from operator import attrgetter
from typing import List, Optional, Sequence, Tuple, Union

import numpy as np
import torch

from .binding import BF16, F32, _check, _dtype_code, _on, _require_device, _stream_ptr, lib

ADAMW_BLOCK = 256      # DROPIT_ADAMW_BLOCK: elements that share an offset of the 8-bit states

_CODES = {torch.float32: F32, torch.bfloat16: BF16}


ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2, "relu": 3, "sigmoid": 4}      # dropit_act


def _act_code(act: str) -> int:
    if act not in ACTIVATIONS:
        raise ValueError("act must be one of %s, got %r" % (", ".join(ACTIVATIONS), act))
    return ACTIVATIONS[act]


def _gated_sizes(weight: torch.Tensor) -> Tuple[int, int]:
    shape = weight.shape
    if len(shape) != 2 or shape[0] % 2 or shape[0] == 0 or shape[1] == 0:
        raise ValueError("weight must be [2 * hidden, c_in], gate rows first, got %s" % (tuple(shape),))
    return shape[0] // 2, shape[1]


def _like(t: Optional[torch.Tensor], shape, dtype: torch.dtype, device: torch.device, what: str) -> torch.Tensor:
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if t.dtype != dtype or t.numel() != math.prod(shape) or t.device != device:
        raise ValueError("%s must hold %s elements of %s on %s" % (what, tuple(shape), dtype, device))
    return t


def _check_tensors(first: torch.Tensor, *others: Optional[torch.Tensor]) -> None:
    where = first.get_device()
    for t in (first,) + others:
        if t is not None:
            if not t.is_cuda:
                raise ValueError("dropit operates on device tensors only (no CPU path)")
            if not t.is_contiguous():
                raise ValueError("dropit tensors must be contiguous")
            if t.get_device() != where:
                raise ValueError("the tensors of a call must be on one device")


def _area(workspace: Optional[torch.Tensor], need: int, device: torch.device) -> Tuple[Optional[int], int]:
    if workspace is None:
        if need == 0:
            return None, 0
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def gated_forward(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, act: str = "silu",
                  save: bool = False, h: Optional[torch.Tensor] = None, pre: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None, stream=None):
    """dropit_gated_forward: h = act(x Wg^T + bg) * (x Wu^T + bu) with ``weight`` = [Wg; Wu] of shape [2 * hidden, c_in]
    and ``bias`` [2 * hidden]; ``x`` [..., c_in] gives h [..., hidden].  ``save`` returns (h, pre) with the
    pre-activations [..., 2 * hidden] that ``gated_backward`` takes.  ``act``: silu, gelu, gelu_tanh, relu or sigmoid."""
    _check_tensors(x, weight, bias, h, pre, workspace)
    code, hidden, c_in, act_code = _dtype_code(x.dtype), *_gated_sizes(weight), _act_code(act)
    if weight.dtype != x.dtype or (bias is not None and (bias.dtype != x.dtype or bias.numel() != 2 * hidden)):
        raise ValueError("weight and bias must have x's dtype, bias 2 * hidden = %d elements" % (2 * hidden))
    if x.dim() < 1 or x.shape[-1] != c_in:
        raise ValueError("x must be [..., %d], got %s" % (c_in, tuple(x.shape)))
    lead, tokens = tuple(x.shape[:-1]), x.numel() // c_in
    h = _like(h, lead + (hidden,), x.dtype, x.device, "h")
    if save or pre is not None:
        pre = _like(pre, lead + (2 * hidden,), x.dtype, x.device, "pre")
    need = int(lib().dropit_gated_forward_workspace_bytes(tokens, c_in, hidden, code))
    area, size = _area(workspace, need, x.device)
    with _on(x.device):
        _check(lib().dropit_gated_forward(x.data_ptr(), tokens, c_in, code, weight.data_ptr(),
                                          bias.data_ptr() if bias is not None else None, hidden, act_code, h.data_ptr(),
                                          pre.data_ptr() if pre is not None else None, area, size,
                                          _stream_ptr(stream, x.device)))
    return (h, pre) if pre is not None else h


def gated_backward(dh: torch.Tensor, pre: torch.Tensor, weight: torch.Tensor, act: str = "silu", need_dx: bool = True,
                   need_dbias: bool = False, dpre: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None,
                   dbias: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None
                   ) -> Tuple[torch.Tensor, Optional[torch.Tensor], Optional[torch.Tensor]]:
    """dropit_gated_backward: (dpre [..., 2 * hidden], dx [..., c_in] or None, dbias [2 * hidden] float32 or None) from
    dh [..., hidden] and what ``gated_forward`` saved.  The weight gradient is ``weight_grad`` of the cached x with
    dY = dpre and c_out = 2 * hidden."""
    _check_tensors(dh, pre, weight, dpre, dx, dbias, workspace)
    code, hidden, c_in, act_code = _dtype_code(dh.dtype), *_gated_sizes(weight), _act_code(act)
    if weight.dtype != dh.dtype or pre.dtype != dh.dtype:
        raise ValueError("pre and weight must have dh's dtype")
    if dh.dim() < 1 or dh.shape[-1] != hidden or tuple(pre.shape) != tuple(dh.shape[:-1]) + (2 * hidden,):
        raise ValueError("dh must be [..., %d] and pre [..., %d], got %s and %s" % (hidden, 2 * hidden, tuple(dh.shape), tuple(pre.shape)))
    lead, tokens = tuple(dh.shape[:-1]), dh.numel() // hidden
    dpre = _like(dpre, lead + (2 * hidden,), dh.dtype, dh.device, "dpre")
    need_dx, need_dbias = need_dx or dx is not None, need_dbias or dbias is not None
    if need_dx:
        dx = _like(dx, lead + (c_in,), dh.dtype, dh.device, "dx")
    if need_dbias:
        dbias = _like(dbias, (2 * hidden,), torch.float32, dh.device, "dbias")
    need = int(lib().dropit_gated_backward_workspace_bytes(tokens, c_in, hidden, code, int(need_dx), int(need_dbias)))
    area, size = _area(workspace, need, dh.device)
    with _on(dh.device):
        _check(lib().dropit_gated_backward(dh.data_ptr(), pre.data_ptr(), tokens, c_in, code, weight.data_ptr(), hidden, act_code,
                                           dpre.data_ptr(), dx.data_ptr() if need_dx else None,
                                           dbias.data_ptr() if need_dbias else None, area, size,
                                           _stream_ptr(stream, dh.device)))
    return dpre, dx if need_dx else None, dbias if need_dbias else None


class _AdamwHyper(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps", "weight_decay")] + [
        ("step", ctypes.c_int64), ("step_device", ctypes.c_void_p), ("grad_scale", ctypes.c_void_p)]


# What a call over hundreds of tensors asks of each goes through map() over the tensor's own methods, some 40 ns a tensor and
# question; a step of 152 tensors asks twenty, and the kernels of a small encoder take 140 us.
_dtype_of = attrgetter("dtype")


def _same_device(*lists: Sequence[torch.Tensor]) -> int:
    found = set()
    for tensors in lists:
        found.update(map(torch.Tensor.get_device, tensors))
        if not all(map(torch.Tensor.is_contiguous, tensors)):
            raise ValueError("dropit tensors must be contiguous")
    if len(found) != 1 or -1 in found:
        raise ValueError("dropit operates on device tensors only (no CPU path), and on one device per call")
    return found.pop()


def _one_dtype(tensors: Sequence[torch.Tensor], allowed, what: str) -> torch.dtype:
    found = set(map(_dtype_of, tensors))
    if len(found) != 1 or not found <= set(allowed):
        raise TypeError("%s must all be %s, got %s" % (what, " or ".join(map(str, allowed)), sorted(map(str, found))))
    return found.pop()


def _pointers(tensors: Sequence[torch.Tensor]) -> List[int]:
    return list(map(torch.Tensor.data_ptr, tensors))


def _numels(tensors: Sequence[torch.Tensor]) -> List[int]:
    return list(map(torch.Tensor.numel, tensors))


def _int64(values: List[int]) -> np.ndarray:
    return np.frombuffer(struct.pack("%dq" % len(values), *values), dtype=np.int64)      # (np.array asks each value what it is)


def _scalar(t: Optional[torch.Tensor], dtype: torch.dtype, device: int, what: str) -> Optional[int]:
    if t is None:
        return None
    if t.dtype != dtype or t.numel() < 1 or t.get_device() != device:
        raise ValueError("%s must be a %s tensor of one element on the tensors' device" % (what, dtype))
    return t.data_ptr()


def adamw(params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], m: Sequence[torch.Tensor],
          v: Sequence[torch.Tensor], *, lr: float, betas: Tuple[float, float] = (0.9, 0.999), eps: float = 1e-8,
          weight_decay: float = 0.01, step: Union[int, torch.Tensor] = 1,
          m_offset: Optional[Sequence[torch.Tensor]] = None, v_offset: Optional[Sequence[torch.Tensor]] = None,
          residual: Optional[Sequence[torch.Tensor]] = None, grad_scale: Optional[torch.Tensor] = None,
          stream=None) -> None:
    """dropit_adamw: one AdamW step over the tensors of the lists, in place.  ``m`` / ``v`` are fp32, or uint8 codes
    with int16 ``m_offset`` / ``v_offset`` of ceil(numel / 256) entries each (8-bit states).  ``residual`` (int16, as
    many elements as the parameter) makes bf16 parameters exact fp32 masters.  ``step`` counts from 1; as an int32
    device tensor it is read when the kernels run, which a captured graph needs.  ``grad_scale`` is a device scalar
    that multiplies every gradient (``grad_norm(...)[1:]`` clips)."""
    count = len(params)
    bits8 = m_offset is not None or v_offset is not None
    if bits8 and (m_offset is None or v_offset is None):
        raise ValueError("8-bit states need m_offset and v_offset")
    lists = [params, grads, m, v] + ([m_offset, v_offset] if bits8 else []) + ([residual] if residual is not None else [])
    if any(len(x) != count for x in lists):
        raise ValueError("the lists of a step must have one entry per parameter")
    if isinstance(step, torch.Tensor):
        step_host = 0
    else:
        step_host = int(step)
        if step_host < 1:
            raise ValueError("step counts from 1, got %d" % step_host)
    if count == 0:
        return
    device = _same_device(*lists)
    p_dtype = _one_dtype(params, (torch.float32, torch.bfloat16), "parameters")
    g_dtype = _one_dtype(grads, (torch.float32, torch.bfloat16), "gradients")
    state_dtype = (torch.uint8,) if bits8 else (torch.float32,)
    _one_dtype(m, state_dtype, "states m")
    _one_dtype(v, state_dtype, "states v")
    numels = _numels(params)
    for name, x in (("gradients", grads), ("m", m), ("v", v)) + ((("residual", residual),) if residual is not None else ()):
        if _numels(x) != numels:
            raise ValueError("%s must have as many elements as their parameters" % name)
    table = np.zeros((count, 8), dtype=np.int64)
    if bits8:
        blocks = (_int64(numels) + (ADAMW_BLOCK - 1)) // ADAMW_BLOCK
        for at, x in ((4, m_offset), (5, v_offset)):
            _one_dtype(x, (torch.int16,), "offsets of 8-bit states")
            if bool((_int64(_numels(x)) < blocks).any()):
                raise ValueError("an offset for every %d elements of a parameter" % ADAMW_BLOCK)
            table[:, at] = _int64(_pointers(x))
    if residual is not None:
        if p_dtype != torch.bfloat16:
            raise TypeError("residuals belong to bfloat16 parameters")
        _one_dtype(residual, (torch.int16,), "residuals")
        table[:, 6] = _int64(_pointers(residual))
    pointers = _pointers(params)
    if len(set(pointers)) != count and len({q for q, n in zip(pointers, numels) if n}) != sum(1 for n in numels if n):
        raise ValueError("a parameter appears twice in one step")
    for at, x in ((0, pointers), (1, _pointers(grads)), (2, _pointers(m)), (3, _pointers(v)), (7, numels)):
        table[:, at] = _int64(x)
    hyper = _AdamwHyper(float(lr), float(betas[0]), float(betas[1]), float(eps), float(weight_decay), step_host,
                        _scalar(step, torch.int32, device, "step") if isinstance(step, torch.Tensor) else None,
                        _scalar(grad_scale, torch.float32, device, "grad_scale"))
    where = params[0].device
    with _on(where):
        _check(lib().dropit_adamw(table.ctypes.data, count, _CODES[p_dtype], _CODES[g_dtype], 8 if bits8 else 32,
                                  ctypes.byref(hyper), _stream_ptr(stream, where)))


def adamw_unpack(codes: torch.Tensor, offset: torch.Tensor, signed: bool, values: Optional[torch.Tensor] = None,
                 stream=None) -> torch.Tensor:
    """dropit_adamw_unpack: the values that 8-bit states stand for, as bfloat16 (exact), in the codes' shape;
    ``signed`` for m, not for v."""
    _require_device(codes, offset, values)
    n = codes.numel()
    if codes.dtype != torch.uint8 or offset.dtype != torch.int16 or offset.numel() < (n + ADAMW_BLOCK - 1) // ADAMW_BLOCK:
        raise ValueError("codes must be uint8 with an int16 offset for every %d of them" % ADAMW_BLOCK)
    if offset.device != codes.device or (values is not None and values.device != codes.device):
        raise ValueError("codes, offsets and values must be on one device")
    if values is None:
        values = torch.empty(codes.shape, dtype=torch.bfloat16, device=codes.device)
    elif values.dtype != torch.bfloat16 or values.numel() != n:
        raise ValueError("values must hold %d bfloat16 elements" % n)
    with _on(codes.device):
        _check(lib().dropit_adamw_unpack(codes.data_ptr(), offset.data_ptr(), n, 1 if signed else 0, values.data_ptr(),
                                         _stream_ptr(stream, codes.device)))
    return values


def grad_norm(grads: Sequence[torch.Tensor], max_norm: float = math.inf, out: Optional[torch.Tensor] = None,
              workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """dropit_grad_norm: float32 [2] on the device, the 2-norm over all elements of ``grads`` (float32 or bfloat16, mixed
    as they come) and min(1, max_norm / (norm + 1e-6)), the factor that clips them."""
    count = len(grads)
    if not float(max_norm) > 0.0:
        raise ValueError("max_norm must be positive, got %r" % (max_norm,))
    if count == 0:
        raise ValueError("grad_norm needs a tensor (it tells the device)")
    device = _same_device(grads)
    types = set(map(_dtype_of, grads))
    if not types <= set(_CODES):
        raise TypeError("dropit supports float32 and bfloat16 tensors, got %s" % sorted(map(str, types)))
    if len(types) == 1:
        dtypes = np.full(count, _CODES[types.pop()], dtype=np.int32)
    else:
        dtypes = np.array([_CODES[t.dtype] for t in grads], dtype=np.int32)
    where = grads[0].device
    if out is None:
        out = torch.empty(2, dtype=torch.float32, device=where)
    elif out.dtype != torch.float32 or out.numel() < 2 or out.get_device() != device or not out.is_contiguous():
        raise ValueError("out must hold two contiguous float32 elements on the gradients' device")
    pointers, numels = _int64(_pointers(grads)), _int64(_numels(grads))
    at_pointers, at_numels = pointers.ctypes.data, numels.ctypes.data
    need = int(lib().dropit_grad_norm_workspace_bytes(at_numels, count))
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=where) if need else None
    else:
        _require_device(workspace)
    with _on(where):
        _check(lib().dropit_grad_norm(at_pointers, at_numels, dtypes.ctypes.data, count, float(max_norm),
                                      out.data_ptr(), workspace.data_ptr() if workspace is not None else None,
                                      workspace.numel() if workspace is not None else 0, _stream_ptr(stream, where)))
    return out
