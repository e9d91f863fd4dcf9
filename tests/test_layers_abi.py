"""include/dropit_layers.h: the library exports what it declares and refuses bad arguments before it touches a GPU."""
import ctypes
import math
import os
import re

import numpy as np
import pytest
import torch

import paper_2202_13808_amd as dropit
from paper_2202_13808_amd import binding, layers

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x100000            # never dereferenced: validation fails first


def test_library_exports_every_declared_symbol():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "dropit_layers.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(dropit_[a-z_0-9]+)\s*\(", text))
    assert {"dropit_gated_forward", "dropit_gated_forward_workspace_bytes", "dropit_gated_backward",
            "dropit_gated_backward_workspace_bytes"} <= names
    assert {"dropit_adamw", "dropit_adamw_unpack", "dropit_grad_norm", "dropit_grad_norm_workspace_bytes"} <= names
    for name in names:
        assert hasattr(dropit.lib(), name), name


def _hyper(**kw):
    h = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, step=1, step_device=None, grad_scale=None)
    h.update(kw)
    return layers._AdamwHyper(*[h[f[0]] for f in layers._AdamwHyper._fields_])


def _step(count=1, p_dtype=binding.F32, g_dtype=binding.F32, bits=32, hyper=None, **fields):
    row = dict(p=FAKE, g=FAKE, m=FAKE, v=FAKE, mo=0, vo=0, low=0, n=10)
    row.update(fields)
    table = np.array([list(row.values())] * max(count, 1), dtype=np.int64)
    h = hyper or _hyper()
    return dropit.lib().dropit_adamw(table.ctypes.data, count, p_dtype, g_dtype, bits, ctypes.byref(h), None)


def test_adamw_refuses_bad_arguments_without_a_gpu():
    bad = [dict(count=-1), dict(p_dtype=7), dict(g_dtype=7), dict(bits=16), dict(n=-1), dict(n=(1 << 34) + 1), dict(bits=8),
           dict(mo=FAKE), dict(vo=FAKE), dict(low=FAKE)]
    bad += [{k: 0} for k in "pgmv"] + [{k: FAKE + 1} for k in "pgmv"]
    bad += [dict(hyper=_hyper(**h)) for h in (dict(lr=math.nan), dict(lr=math.inf), dict(beta1=1.0), dict(beta1=-0.1),
                                              dict(beta2=1.0), dict(beta2=math.nan), dict(eps=-1.0), dict(eps=math.inf),
                                              dict(weight_decay=math.nan), dict(step=0), dict(step=-5),
                                              dict(step_device=FAKE + 2), dict(grad_scale=FAKE + 1))]
    for kw in bad:
        assert _step(**kw) == binding.EINVAL, kw
    assert dropit.lib().dropit_adamw(None, 1, 0, 0, 32, ctypes.byref(_hyper()), None) == binding.EINVAL
    assert dropit.lib().dropit_adamw(None, 0, 0, 0, 32, None, None) == binding.EINVAL
    # nothing to do: no launch, no error
    assert dropit.lib().dropit_adamw(None, 0, 0, 0, 32, ctypes.byref(_hyper()), None) == binding.OK
    table = np.zeros((2, 8), dtype=np.int64)
    assert dropit.lib().dropit_adamw(table.ctypes.data, 2, 0, 0, 8, ctypes.byref(_hyper()), None) == binding.OK


def test_residuals_belong_to_all_tensors_of_a_call_or_none():
    rows = np.array([[FAKE, FAKE, FAKE, FAKE, 0, 0, FAKE, 10], [FAKE, FAKE, FAKE, FAKE, 0, 0, 0, 10]], dtype=np.int64)
    h = _hyper()
    assert dropit.lib().dropit_adamw(rows.ctypes.data, 2, binding.BF16, binding.F32, 32, ctypes.byref(h), None) == binding.EINVAL


def test_unpack_and_norm_refuse_bad_arguments_without_a_gpu():
    L = dropit.lib()
    assert L.dropit_adamw_unpack(FAKE, FAKE, -1, 1, FAKE, None) == binding.EINVAL
    assert L.dropit_adamw_unpack(FAKE, FAKE, 5, 2, FAKE, None) == binding.EINVAL
    for bad in ((None, FAKE, FAKE), (FAKE, None, FAKE), (FAKE, FAKE, None), (FAKE, FAKE + 1, FAKE), (FAKE, FAKE, FAKE + 1)):
        assert L.dropit_adamw_unpack(bad[0], bad[1], 5, 1, bad[2], None) == binding.EINVAL
    assert L.dropit_adamw_unpack(None, None, 0, 0, None, None) == binding.OK

    def norm(ptr=FAKE, n=100000, dt=0, count=1, max_norm=1.0, out=FAKE, ws=FAKE, nbytes=1 << 20):
        p, s, d = np.array([ptr], np.int64), np.array([n], np.int64), np.array([dt], np.int32)
        return L.dropit_grad_norm(p.ctypes.data, s.ctypes.data, d.ctypes.data, count, max_norm, out, ws, nbytes, None)

    for kw in (dict(ptr=0), dict(ptr=FAKE + 2), dict(n=-1), dict(n=(1 << 34) + 1), dict(dt=3), dict(count=-1), dict(max_norm=0.0),
               dict(max_norm=-1.0), dict(max_norm=math.nan), dict(out=None), dict(out=FAKE + 2), dict(ws=None), dict(ws=FAKE + 8)):
        assert norm(**kw) == binding.EINVAL, kw
    assert norm(nbytes=8) == binding.EWORKSPACE
    n = np.array([100000, 5], np.int64)
    assert L.dropit_grad_norm_workspace_bytes(n.ctypes.data, 2) == 8 * 8
    assert L.dropit_grad_norm_workspace_bytes(n.ctypes.data, -1) == 0 and L.dropit_grad_norm_workspace_bytes(None, 1) == 0


def test_python_entry_points_refuse_host_tensors_and_mismatches():
    x = torch.zeros(8)
    with pytest.raises(ValueError):
        dropit.adamw([x], [x], [x.clone()], [x.clone()], lr=1e-3, step=1)
    with pytest.raises(ValueError):
        dropit.adamw([x], [x], [x], [], lr=1e-3, step=1)
    with pytest.raises(ValueError):
        dropit.adamw([x], [x], [x], [x], lr=1e-3, step=0)
    with pytest.raises(ValueError):
        dropit.adamw([x], [x], [x], [x], lr=1e-3, m_offset=[x])
    with pytest.raises(ValueError):
        dropit.grad_norm([])
    with pytest.raises(ValueError):
        dropit.grad_norm([x])
    with pytest.raises(ValueError):
        dropit.grad_norm([x], max_norm=0.0)
    with pytest.raises(ValueError):
        dropit.adamw_unpack(torch.zeros(3, dtype=torch.uint8), torch.zeros(1, dtype=torch.int16), True)
    dropit.adamw([], [], [], [], lr=1e-3, step=1)


def test_gated_projection_refuses_bad_arguments_without_a_gpu():
    L, big = dropit.lib(), 1 << 40

    def forward(x=FAKE, t=10, c=16, dt=binding.BF16, w=FAKE, b=None, n=8, act=0, h=FAKE, pre=None, ws=FAKE, nbytes=big):
        return L.dropit_gated_forward(x, t, c, dt, w, b, n, act, h, pre, ws, nbytes, None)

    for kw in (dict(x=None), dict(w=None), dict(h=None), dict(x=FAKE + 8), dict(w=FAKE + 2), dict(h=FAKE + 4), dict(b=FAKE + 2),
               dict(pre=FAKE + 8), dict(t=-1), dict(c=0), dict(n=0), dict(c=(1 << 28) + 1), dict(n=(1 << 27) + 1),
               dict(t=1 << 31), dict(t=(1 << 31) - 1, n=1 << 20), dict(dt=2), dict(act=-1), dict(act=5)):
        assert forward(**kw) == binding.EINVAL, kw
    assert forward(t=0, x=None, w=None, h=None) == binding.OK
    need = L.dropit_gated_forward_workspace_bytes(1, 4097, 64, binding.F32)          # (odd rows, few tiles: in slices)
    assert need > 0
    assert forward(t=1, c=4097, n=64, dt=binding.F32, nbytes=need - 1) == binding.EWORKSPACE
    assert forward(t=1, c=4097, n=64, dt=binding.F32, ws=None) == binding.EINVAL
    assert forward(t=1, c=4097, n=64, dt=binding.F32, ws=FAKE + 16) == binding.EINVAL

    def backward(dh=FAKE, pre=FAKE, t=10, c=16, dt=binding.BF16, w=FAKE, n=8, act=0, dpre=FAKE, dx=FAKE, db=FAKE, ws=FAKE, nbytes=big):
        return L.dropit_gated_backward(dh, pre, t, c, dt, w, n, act, dpre, dx, db, ws, nbytes, None)

    for kw in (dict(dh=None), dict(pre=None), dict(w=None), dict(dpre=None), dict(dh=FAKE + 2), dict(pre=FAKE + 8),
               dict(dpre=FAKE + 8), dict(dx=FAKE + 8), dict(db=FAKE + 4), dict(w=FAKE + 4), dict(t=-1), dict(c=0), dict(n=0),
               dict(dt=9), dict(act=7), dict(ws=None), dict(ws=FAKE + 64)):
        assert backward(**kw) == binding.EINVAL, kw
    assert backward(nbytes=16) == binding.EWORKSPACE
    assert L.dropit_gated_backward_workspace_bytes(10, 16, 8, binding.BF16, 0, 0) == 0
    assert L.dropit_gated_backward_workspace_bytes(10, 16, 8, binding.BF16, 0, 1) == 3 * 16 * 4       # blocks of four tokens
    assert L.dropit_gated_backward_workspace_bytes(10, 0, 8, binding.BF16, 1, 1) == 0


def test_gated_projection_in_python_refuses_host_tensors_and_mismatches():
    x, w = torch.zeros(4, 8), torch.zeros(6, 8)
    with pytest.raises(ValueError):
        dropit.gated_forward(x, w)
    with pytest.raises(ValueError):
        dropit.gated_backward(torch.zeros(4, 3), torch.zeros(4, 6), w)
    with pytest.raises(ValueError):
        layers._act_code("tanh")
    for bad in (torch.zeros(5, 8), torch.zeros(6), torch.zeros(0, 8), torch.zeros(6, 0)):
        with pytest.raises(ValueError):
            layers._gated_sizes(bad)
