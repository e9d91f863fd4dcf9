"""ctypes binding of the C ABI in ``include/dropit_layers.h`` -- marshalling and checks only.

The operators that stand beside the dropped cache in a training step: the AdamW step over many tensors, the
global gradient norm.  Functions have the names of the C entry points without the ``dropit_`` prefix; the
formulas stand in the header.
"""
from __future__ import annotations

import ctypes
import math
from typing import List, Optional, Sequence, Tuple, Union

import numpy as np
import torch

from .binding import BF16, F32, _check, _on, _require_device, _stream_ptr, lib

ADAMW_BLOCK = 256      # DROPIT_ADAMW_BLOCK: elements that share an offset of the 8-bit states

_CODES = {torch.float32: F32, torch.bfloat16: BF16}


class _AdamwHyper(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps", "weight_decay")] + [
        ("step", ctypes.c_int64), ("step_device", ctypes.c_void_p), ("grad_scale", ctypes.c_void_p)]


# What a call over hundreds of tensors asks of each goes through map() over the tensor's own methods: 40 ns a tensor and
# question, a third of what a Python loop takes.
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
    found = {t.dtype for t in tensors}
    if len(found) != 1 or not found <= set(allowed):
        raise TypeError("%s must all be %s, got %s" % (what, " or ".join(map(str, allowed)), sorted(map(str, found))))
    return found.pop()


def _pointers(tensors: Sequence[torch.Tensor]) -> List[int]:
    return list(map(torch.Tensor.data_ptr, tensors))


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
    numels = list(map(torch.Tensor.numel, params))
    for name, x in (("gradients", grads), ("m", m), ("v", v)) + ((("residual", residual),) if residual is not None else ()):
        if list(map(torch.Tensor.numel, x)) != numels:
            raise ValueError("%s must have as many elements as their parameters" % name)
    table = np.zeros((8, count), dtype=np.int64)
    if bits8:
        _one_dtype(list(m) + list(v), (torch.uint8,), "8-bit states")
        _one_dtype(list(m_offset) + list(v_offset), (torch.int16,), "offsets of 8-bit states")
        blocks = [(n + ADAMW_BLOCK - 1) // ADAMW_BLOCK for n in numels]
        for x in (m_offset, v_offset):
            if any(have < need for have, need in zip(map(torch.Tensor.numel, x), blocks)):
                raise ValueError("an offset for every %d elements of a parameter" % ADAMW_BLOCK)
        table[4], table[5] = _pointers(m_offset), _pointers(v_offset)
    else:
        _one_dtype(list(m) + list(v), (torch.float32,), "states")
    if residual is not None:
        if p_dtype != torch.bfloat16:
            raise TypeError("residuals belong to bfloat16 parameters")
        _one_dtype(residual, (torch.int16,), "residuals")
        table[6] = _pointers(residual)
    pointers = _pointers(params)
    if len(set(pointers)) != count and len({q for q, n in zip(pointers, numels) if n}) != sum(1 for n in numels if n):
        raise ValueError("a parameter appears twice in one step")
    table[0], table[1], table[2], table[3], table[7] = pointers, _pointers(grads), _pointers(m), _pointers(v), numels
    table = np.ascontiguousarray(table.T)
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
    codes = [_CODES.get(t.dtype, -1) for t in grads]
    if -1 in codes:
        raise TypeError("dropit supports float32 and bfloat16 tensors, got %s" % {str(t.dtype) for t in grads})
    where = grads[0].device
    if out is None:
        out = torch.empty(2, dtype=torch.float32, device=where)
    elif out.dtype != torch.float32 or out.numel() < 2 or out.get_device() != device or not out.is_contiguous():
        raise ValueError("out must hold two contiguous float32 elements on the gradients' device")
    pointers = np.array(_pointers(grads), dtype=np.int64)
    numels = np.array(list(map(torch.Tensor.numel, grads)), dtype=np.int64)
    dtypes = np.array(codes, dtype=np.int32)
    need = int(lib().dropit_grad_norm_workspace_bytes(numels.ctypes.data, count))
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=where) if need else None
    else:
        _require_device(workspace)
    with _on(where):
        _check(lib().dropit_grad_norm(pointers.ctypes.data, numels.ctypes.data, dtypes.ctypes.data, count, float(max_norm),
                                      out.data_ptr(), workspace.data_ptr() if workspace is not None else None,
                                      workspace.numel() if workspace is not None else 0, _stream_ptr(stream, where)))
    return out
