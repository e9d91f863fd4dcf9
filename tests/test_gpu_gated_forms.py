"""nn.gated_linear in the forms of inference that the kernels take no part in, and what it refuses."""
import pytest
import torch
import torch.autograd.forward_ad as fwad

import paper_2202_13808_amd as dropit
from paper_2202_13808_amd import nn as dnn

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _layer(act="gelu_tanh", dtype=torch.float32, **kw):
    torch.manual_seed(5)
    return dnn.GatedLinear(24, 20, act=act, device=DEV, dtype=dtype, **kw)


def _tangent(layer, x, v, act):
    """The derivative along v of the formula, in 64 bits."""
    w, b = layer.weight.detach().cpu().double(), layer.bias.detach().cpu().double()
    fn = {"gelu_tanh": lambda t: torch.nn.functional.gelu(t, approximate="tanh"), "silu": torch.nn.functional.silu}[act]
    z, dz = x.cpu().double() @ w.t() + b, v.cpu().double() @ w.t()
    with torch.enable_grad():
        gate = z[:, :20].clone().requires_grad_(True)
        a = fn(gate)
        (slope,) = torch.autograd.grad(a.sum(), gate)
    return slope * dz[:, :20] * z[:, 20:] + a.detach() * dz[:, 20:]


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("how", ["no_grad", "frozen"])
def test_forward_mode_keeps_its_tangent(how, act):
    print("gated forward mode", how, act, flush=True)
    layer = _layer(act, gamma=0.5)
    x, v = torch.randn(3, 24, device=DEV), torch.randn(3, 24, device=DEV)
    if how == "frozen":
        layer.requires_grad_(False)
    with torch.set_grad_enabled(how == "frozen"), fwad.dual_level():
        out = fwad.unpack_dual(layer(fwad.make_dual(x, v)))
        assert out.tangent is not None
        # 24 terms and some twenty operations in fp32, of sizes around ten
        assert float((out.tangent.cpu().double() - _tangent(layer, x, v, act)).abs().max()) <= 64 * 2.0 ** -24 * 10
        weight = fwad.make_dual(layer.weight.detach(), torch.randn_like(layer.weight))
        assert fwad.unpack_dual(dnn.gated_linear(x, weight, layer.bias.detach(), act=act)).tangent is not None
        bias = fwad.make_dual(layer.bias.detach(), torch.randn_like(layer.bias))
        assert fwad.unpack_dual(dnn.gated_linear(x, layer.weight.detach(), bias, act=act)).tangent is not None
        # nothing is differentiated here: the kernel's bits
        got = dnn.gated_linear(x, layer.weight.detach(), layer.bias.detach(), act=act)
    assert torch.equal(got, dropit.gated_forward(x, layer.weight.detach(), layer.bias.detach(), act=act))


def test_forward_mode_through_the_dropping_layer_is_refused():
    print("gated forward mode in training", flush=True)
    layer = _layer(gamma=0.5)
    with fwad.dual_level(), pytest.raises(Exception, match="forward"):
        layer(fwad.make_dual(torch.randn(3, 24, device=DEV), torch.randn(3, 24, device=DEV)))


def test_function_transforms_of_inference():
    print("gated transforms", flush=True)
    layer = _layer("silu").eval().requires_grad_(False)
    x, v = torch.randn(4, 24, device=DEV), torch.randn(4, 24, device=DEV)
    h = layer(x)
    out, tangent = torch.func.jvp(layer, (x,), (v,))
    assert float((out - h).abs().max()) <= 64 * 2.0 ** -24 * 10
    assert float((tangent.cpu().double() - _tangent(layer, x, v, "silu")).abs().max()) <= 64 * 2.0 ** -24 * 10
    rows = torch.func.vmap(layer)(x)
    assert rows.shape == h.shape and float((rows - h).abs().max()) <= 64 * 2.0 ** -24 * 10


def test_a_traced_layer_computes():
    print("gated trace", flush=True)
    layer = _layer("silu").eval()
    x, other = torch.randn(4, 24, device=DEV), torch.randn(4, 24, device=DEV)
    with torch.no_grad():
        traced = torch.jit.trace(layer, (x,))
        for t in (x, other):
            assert float((traced(t) - layer(t)).abs().max()) <= 64 * 2.0 ** -24 * 10


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64])
def test_types_without_a_kernel_run_plainly_where_nothing_is_dropped(dtype):
    print("gated other types", dtype, flush=True)
    wide = _layer("silu").eval()
    layer = _layer("silu", dtype=dtype, gamma=0.0)
    x = torch.randn(5, 24, device=DEV)
    half = torch.finfo(dtype).eps / 2
    with torch.no_grad():
        h = wide(x)
        layer.load_state_dict(wide.state_dict())
        # the inputs, the weights and three results rounded to the type, fp32's own roundings: sizes around ten
        assert float((layer(x.to(dtype)).float() - h).abs().max()) <= (24 + 6) * (half + 2.0 ** -24) * 10
        with torch.autocast("cuda", dtype=torch.float16):
            assert wide(x).dtype == torch.float16
    layer(x.to(dtype)).sum().backward()                # gamma = 0: the plain layer's gradients
    assert layer.weight.grad.dtype == dtype and bool(layer.weight.grad.isfinite().all())
    layer.gamma = 0.5
    with pytest.raises(TypeError, match="float32 and bfloat16"):
        layer(x.to(dtype))
    with torch.autocast("cuda", dtype=torch.float16), pytest.raises(TypeError, match="float32 and bfloat16"):
        _layer("silu", gamma=0.5)(x)


def test_a_layer_that_trains_without_dropping_is_followed_too():
    print("gated forward mode, nothing dropped", flush=True)
    layer = _layer("silu", gamma=0.0)
    x, v = torch.randn(3, 24, device=DEV), torch.randn(3, 24, device=DEV)
    want = _tangent(layer, x, v, "silu")
    with fwad.dual_level():
        out = fwad.unpack_dual(layer(fwad.make_dual(x, v)))
        assert float((out.tangent.detach().cpu().double() - want).abs().max()) <= 64 * 2.0 ** -24 * 10
    grad = torch.func.grad(lambda t: layer(t).sum())(x)
    xr = x.clone().requires_grad_(True)
    layer(xr).sum().backward()                         # the kernels'
    assert float((grad - xr.grad).abs().max()) <= 64 * 2.0 ** -24 * 10
    frozen = _layer("silu", gamma=0.5).requires_grad_(False)
    with fwad.dual_level():
        out = fwad.unpack_dual(frozen(fwad.make_dual(xr, v)))
        assert float((out.tangent.detach().cpu().double() - want).abs().max()) <= 64 * 2.0 ** -24 * 10
