"""The activations of the gated projection far out, relative to their own size: a value or a slope that is lost there is small,
and an allowance that does not shrink with it would not see the loss.

Tolerances.  ``unit`` is a relative error: in fp32, roundings of 2^-24 of the operations and of the arguments of the exponential
(an argument y that is rounded by 2^-24 of itself moves e^y by y 2^-24 of itself); in bf16 the hardware's exponential and
reciprocal, 2^-20 with the same growth.  It is taken of the sum of the terms' sizes, where terms cancel.  What leaves in bf16 is
off by half a step more, 2^-8 of itself.  Below 2^-120 fp32 runs out of bits (e^-z overflows, or the results are denormal)."""
import math

import pytest
import torch

import paper_2202_13808_amd as dropit

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
FLOOR = 2.0 ** -120


def gates(dtype):
    z = torch.cat([torch.linspace(-30, 30, 1201), torch.linspace(-1, 1, 41) / 64,
                   torch.tensor([0.0, -0.0, 40.0, -40.0, 87.0, -87.0, 90.0, -90.0, 300.0, -300.0, 1e10, -1e10, 3e18, -3e18, 1e20, -1e20, 3e38, -3e38])])
    return z.to(DT[dtype])


def sigmoid_bounds(z, dtype, forward):
    s, t = torch.sigmoid(z), torch.sigmoid(-z)
    unit = 16 * 2.0 ** -24 if dtype == "f32" else 2.0 ** -20 * (1 + z.abs())
    return (s, unit * s), (s * t, unit * s * t)


def gelu_tanh_bounds(z, dtype, forward):
    k, c = math.sqrt(2 / math.pi), 0.044715
    y = 2 * k * (z + c * z ** 3)
    s, t = torch.sigmoid(y), torch.sigmoid(-y)
    unit = (32 + 8 * y.abs()) * 2.0 ** -24 if dtype == "f32" else 2.0 ** -20 * (1 + y.abs())
    inner = torch.where(t > 0, 2 * k * z * (1 + 3 * c * z * z), torch.zeros_like(z))
    # t = 1 - s is off by a rounding of 1, and is zero where it is smaller than that
    lost = torch.where(t < 2.0 ** -25, t, torch.full_like(z, 2.0 ** -23 if dtype == "f32" else 2.0 ** -20))
    s_off = unit * s * t + (8 * 2.0 ** -24 if dtype == "f32" else 2.0 ** -20) * s        # (the argument moves s by s t)
    return (z * s, z.abs() * s_off), (s + s * t * inner, s_off + (unit * s * t + lost * s) * inner.abs())


def gelu_bounds(z, dtype, forward):
    ndtr = lambda x: 0.5 * torch.special.erfc(-x * math.sqrt(0.5))  # noqa: E731  (torch.special.ndtr is 0 from -9 on)
    phi, bell = ndtr(z), torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    near_z = z.clamp(-100, 100)
    # the argument of both exponentials is z^2 / 2; bf16's forward pass takes Phi(-|z|) from a polynomial that is off by 1e-4 of it
    # at most
    unit = (32 + 2 * near_z ** 2) * 2.0 ** -24 if dtype == "f32" else 2.0 ** -20 * (1 + near_z ** 2)
    tail = 1e-4 if dtype == "bf16" and forward else unit
    phi_off = tail * ndtr(-z.abs()) + (4 * 2.0 ** -24) * phi
    return (z * phi, z.abs() * phi_off), (phi + near_z * bell, phi_off + unit * (near_z * bell).abs())


def silu_bounds(z, dtype, forward):
    s, t = torch.sigmoid(z), torch.sigmoid(-z)
    unit = 16 * 2.0 ** -24 if dtype == "f32" else 2.0 ** -20 * (1 + z.clamp(-100, 100).abs())
    lost = torch.where(t < 2.0 ** -25, t, torch.full_like(z, 2.0 ** -23 if dtype == "f32" else 2.0 ** -20))       # t = 1 - s
    return (z * s, (unit * z * s).abs()), (s * (1 + z * t), unit * s * (1 + z.abs() * t) + lost * s * z.abs())


def relu_bounds(z, dtype, forward):
    nothing = torch.zeros_like(z)
    return (z.clamp(min=0), nothing), ((z > 0).double(), nothing)


# (act, its tolerance), (slope, its tolerance), in 64 bits
BOUNDS = {"sigmoid": sigmoid_bounds, "gelu_tanh": gelu_tanh_bounds, "gelu": gelu_bounds, "silu": silu_bounds, "relu": relu_bounds}


def near(got, want, tol, dtype, z, what):
    diff = (got.cpu().double() - want).abs()
    bad = ~(diff <= tol + HALF[dtype] * want.abs() + FLOOR * (1 + want.abs()))
    assert not bool(bad.any()), (what, [(float(a), float(b), float(c)) for a, b, c in zip(z[bad][:4], got.cpu()[bad][:4], want[bad][:4])])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", list(BOUNDS))
def test_activations_far_out(act, dtype):
    print("gated tails", act, dtype, flush=True)
    z = gates(dtype)
    n = z.numel()
    (value, value_tol), (slope, slope_tol) = BOUNDS[act](z.double(), dtype, False)
    pre = torch.cat([z, torch.ones(n, dtype=DT[dtype])]).unsqueeze(0).to(DEV)
    w = torch.zeros(2 * n, 8, dtype=DT[dtype], device=DEV)
    w[:, 0] = pre[0]
    dpre, _, dbias = dropit.gated_backward(torch.ones(1, n, dtype=DT[dtype], device=DEV), pre, w, act=act, need_dx=False, need_dbias=True)
    # (one token: the sums of its gradients are those gradients, not rounded)
    near(dbias[:n], slope, slope_tol, "f32", z, "slope in the sum")
    near(dbias[n:], value, value_tol, "f32", z, "value in the sum")
    near(dpre[0, :n], slope, slope_tol, dtype, z, "slope")
    near(dpre[0, n:], value, value_tol, dtype, z, "value in the gradient")
    value_tol = BOUNDS[act](z.double(), dtype, True)[0][1]
    for tokens in (1, 70, 1500):                       # the products for few, for some and for many tokens
        x = torch.zeros(tokens, 8, dtype=DT[dtype], device=DEV)
        x[:, 0] = 1.0
        h = dropit.gated_forward(x, w, act=act)
        assert torch.equal(h, h[:1].expand_as(h))
        near(h[0], value, value_tol, dtype, z, "value")
