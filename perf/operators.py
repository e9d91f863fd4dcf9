"""Operators of a training step beside the dropped cache, as cases to time: the gated projection of a
feed-forward block (forward, with and without what its backward pass needs, and the backward pass), the
AdamW step over many tensors with states in 32 or in 8 bits, and the global gradient norm that a clipped
step takes its factor from.

``run`` computes a case in elementary torch operations where ``own`` is false and through the package's
entry points where it is true.  ``exact`` computes it in 64 bits, apart from both.
"""
import math

import torch

own = False

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 256                                     # elements that share an offset of the 8-bit states
WEYL_I, WEYL_T = 0x6A09E667, 0x9E3779B9         # the dither of element i at step t: (i * WEYL_I + t * WEYL_T) mod 2^32
HYPER = {"lr": 1e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 0.05}


# ---- the cases ------------------------------------------------------------------------------------
# kind "forward": x [tokens, c] -> h [tokens, hidden] (save: and the pre-activations [tokens, 2 * hidden]),
# "backward": dh -> gradients of the pre-activations, of x and of the bias;  weight [2 * hidden, c], gate rows first
def _gated(name, kind, dtype, tokens, c, hidden, act, bias=False, save=False):
    return {"name": name, "kind": kind, "dtype": dtype, "tokens": tokens, "c": c, "hidden": hidden, "act": act,
            "bias": bias, "save": save}


# kind "adamw": one step over the tensors of `model`;  "norm": their global gradient norm and clipping factor.
# model "encoder": the parameters of an encoder of `depth` blocks of width `dim`;  "square": `depth` matrices
# [dim, dim + odd];  bits: of the states;  residual: 16 more bits beside each bf16 parameter
def _tensors(name, kind, model, depth, dim, odd, p, g, bits=32, residual=False, clip=False, step=100):
    return {"name": name, "kind": kind, "model": model, "depth": depth, "dim": dim, "odd": odd, "p": p, "g": g,
            "bits": bits, "residual": residual, "clip": clip, "step": step}


def listed():
    return [
        # one token of one sequence through the layer of a small encoder: latency
        _gated("gated_token", "forward", "bf16", 1, 384, 1024, "silu"),
        # 16 sequences decoded together through a large layer: the weights are streamed once
        _gated("gated_decode16", "forward", "bf16", 16, 4096, 10240, "silu"),
        # a long prompt through the same layer: the largest product
        _gated("gated_prompt", "forward", "bf16", 8192, 4096, 10240, "silu"),
        # training forward of ViT-B/16 at 64 images of 197 tokens, gated with the same parameter count as its MLP
        _gated("gated_vitb_train", "forward", "bf16", 64 * 197, 768, 2048, "gelu", bias=True, save=True),
        # odd sizes in torch's default type: a ragged batch, no dimension a multiple of anything
        _gated("gated_ragged_f32", "forward", "f32", 1003, 387, 515, "gelu_tanh", bias=True, save=True),
        # the backward pass of the ViT-B layer
        _gated("gated_vitb_backward", "backward", "bf16", 64 * 197, 768, 2048, "gelu", bias=True),
        # the backward pass of a DeiT-S layer at a fine-tuning batch of 8 images, in torch's default type
        _gated("gated_batch8_backward_f32", "backward", "f32", 8 * 197, 384, 1024, "silu"),
        # the step of the DeiT-S-shaped encoder (12 blocks of 384) in torch's default type, clipped
        _tensors("adamw_deits", "adamw", "encoder", 12, 384, 0, "f32", "f32", clip=True),
        # ViT-B in bf16 with exact masters (16 more bits a parameter) and 8-bit states
        _tensors("adamw_vitb_8bit", "adamw", "encoder", 12, 768, 0, "bf16", "bf16", bits=8, residual=True, clip=True),
        # large matrices of odd width in bf16 with 8-bit states: the largest step
        _tensors("adamw_large_8bit", "adamw", "square", 16, 4096, 13, "bf16", "bf16", bits=8),
        # gradients of one block of a tiny encoder, and of ViT-B
        _tensors("norm_tiny", "norm", "encoder", 1, 64, 0, "f32", "f32"),
        _tensors("norm_vitb", "norm", "encoder", 12, 768, 0, "bf16", "bf16"),
    ]


def _log_int(rng, lo, hi, round_to=1):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return min(hi, max(lo, v // round_to * round_to))


def draw(rng):
    if rng.random() < 0.55:
        while True:
            even = rng.random() < 0.6
            tokens = _log_int(rng, 1, 16384)
            c = _log_int(rng, 64, 4096, 64 if even else 1)
            hidden = _log_int(rng, 64, 10240, 64 if even else 1)
            dtype = "f32" if rng.random() < 0.25 else "bf16"
            if 4 * tokens * c * hidden <= (2e11 if dtype == "f32" else 4 * 8192 * 4096 * 10240):
                break
        kind = rng.choice(["forward", "backward"])
        return _gated("", kind, dtype, tokens, c, hidden, rng.choice(["silu", "gelu", "gelu_tanh", "relu", "sigmoid"]),
                      bias=rng.random() < 0.5, save=kind == "forward" and rng.random() < 0.5) | {"name": "drawn"}
    kind = "adamw" if rng.random() < 0.7 else "norm"
    if rng.random() < 0.5:
        model, depth, dim, odd = "encoder", rng.randint(1, 24), _log_int(rng, 16, 768, 16), 0
    else:
        model, depth, dim, odd = "square", rng.randint(1, 32), _log_int(rng, 3, 2800), rng.randint(0, 31)
    p = rng.choice(["f32", "bf16"])
    residual = p == "bf16" and rng.random() < 0.5
    return _tensors("drawn", kind, model, depth, dim, odd, p, "bf16" if p == "bf16" and rng.random() < 0.7 else "f32",
                    bits=rng.choice([8, 32]), residual=residual, clip=rng.random() < 0.5, step=_log_int(rng, 1, 100000))


def _shapes(case):
    d = case["dim"]
    if case["model"] == "square":
        return [(d, d + case["odd"])] * case["depth"]
    block = [(d,), (d,), (3 * d, d), (3 * d,), (d, d), (d,), (d,), (d,), (4 * d, d), (4 * d,), (d, 4 * d), (d,)]
    return [(d, d), (d,)] + block * case["depth"] + [(d,), (d,), (1000, d), (1000,)]


# ---- inputs ---------------------------------------------------------------------------------------
def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed) * 7919 + 13)
    if case["kind"] in ("forward", "backward"):
        dt, t, c, h = DT[case["dtype"]], case["tokens"], case["c"], case["hidden"]
        s = {"case": dict(case), "w": (_randn(gen, 2 * h, c) / math.sqrt(c)).to(dt)}
        s["b"] = (0.1 * _randn(gen, 2 * h)).to(dt) if case["bias"] else None
        if case["kind"] == "forward":
            s["x"] = _randn(gen, t, c).to(dt)                     # behind a layer norm
        else:
            s["pre"] = _randn(gen, t, 2 * h).to(dt)
            s["dh"] = (0.02 * _randn(gen, t, h)).to(dt)
        return s
    # the tensors lie one behind the other in flat buffers, each from a multiple of BLOCK elements on
    shapes = _shapes(case)
    sizes = [math.prod(x) for x in shapes]
    starts, at = [], 0
    for n in sizes:
        starts.append(at)
        at += -(-n // BLOCK) * BLOCK
    # where an element lies in its tensor, and whether it belongs to one
    counts = torch.tensor([-(-n // BLOCK) * BLOCK for n in sizes], device=DEV)
    first = torch.repeat_interleave(torch.tensor(starts, device=DEV), counts, output_size=at)
    index = (torch.arange(at, device=DEV) - first).to(torch.int32)
    inside = index < torch.repeat_interleave(torch.tensor(sizes, device=DEV, dtype=torch.int32), counts, output_size=at)
    del first
    # gradients of different tensors have different sizes; within one they are far from uniform too
    scale = torch.repeat_interleave(1e-3 * torch.exp(_randn(gen, len(sizes))), counts, output_size=at)
    g = torch.where(inside, _randn(gen, at) * scale, 0.0)
    s = {"case": dict(case), "sizes": sizes, "starts": starts, "g": g.to(DT[case["g"]])}
    cut = lambda flat: [flat[a:a + n].view(x) for a, n, x in zip(starts, sizes, shapes)]  # noqa: E731
    s["g_list"] = cut(s["g"])
    if case["kind"] == "norm":
        return s
    master = torch.where(inside, 0.02 * _randn(gen, at), 0.0)
    s["low"] = None
    if case["residual"]:
        s["p"], s["low"] = _split(master)
        s["low_list"] = cut(s["low"])
    else:
        s["p"] = master.to(DT[case["p"]])
    s["p_list"] = cut(s["p"])
    m = torch.where(inside, 0.3 * g + 0.3 * scale * _randn(gen, at), 0.0)
    v = torch.where(inside, (0.9 * scale * (1 + 0.3 * _randn(gen, at))).square(), 0.0)
    s["scale"] = torch.full((1,), 0.37, device=DEV) if case["clip"] else None
    if case["bits"] == 8:
        s["index"] = index
        s["m"], s["mo"] = _encode(m, index, 0, True)
        s["v"], s["vo"] = _encode(v, index, 0, False)
        blocks = lambda flat: [flat[a // BLOCK:a // BLOCK + -(-n // BLOCK)] for a, n in zip(starts, sizes)]  # noqa: E731
        s["mo_list"], s["vo_list"] = blocks(s["mo"]), blocks(s["vo"])
        s["m_list"], s["v_list"] = cut(s["m"]), cut(s["v"])
    else:
        s["m"], s["v"] = m, v
        s["m_list"], s["v_list"] = cut(m), cut(v)
    return s


# ---- plain forms ----------------------------------------------------------------------------------
def _act(z, act):
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "relu":
        return torch.clamp(z, min=0.0)
    return 1.0 / (1.0 + torch.exp(-z))


def _slope(z, act):
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "gelu_tanh":
        k = math.sqrt(2.0 / math.pi)
        t = torch.tanh(k * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * k * (1.0 + 3 * 0.044715 * z * z)
    if act == "relu":
        return (z > 0).to(z.dtype)
    s = 1.0 / (1.0 + torch.exp(-z))
    return s * (1.0 - s)


def _split(master):
    """fp32 -> (bf16, the 16 bits that, added below it, give the fp32 pattern back)."""
    bits = master.view(torch.int32)
    high = (bits + 0x8000) >> 16
    return high.to(torch.int16).view(torch.bfloat16), (bits - (high << 16)).to(torch.int16)


def _join(p, low):
    return ((p.view(torch.int16).to(torch.int32) << 16) + low.to(torch.int32)).view(torch.float32)


def _encode(x, index, step, signed):
    """fp32 -> 8-bit codes and an offset for each block: the pattern's exponent and three bits of its mantissa, less the
    offset that brings the block's largest to the top code, rounded up where the dither says so."""
    top = 127 if signed else 255
    bits = x.abs().view(torch.int32)
    dither = ((index.to(torch.int64) * WEYL_I + step * WEYL_T) & 0xFFFFFFFF) >> 12
    dither = (dither if signed else dither ^ 0xFFFFF).to(torch.int32)
    largest = bits.view(-1, BLOCK).amax(1)
    offset = (torch.clamp((largest + 0xFFFFF) >> 20, max=0x7F7) - top).clamp(min=0)
    code = torch.clamp((bits + dither) >> 20, max=0x7F7).view(-1, BLOCK) - offset[:, None]
    code = code.clamp(min=0).view(-1)
    if signed:
        code = code + 128 * (x < 0).to(torch.int32)
    else:
        code = torch.where((code == 0) & (bits > 0), 1, code)
    return code.to(torch.uint8), offset.to(torch.int16)


def _decode(code, offset, signed):
    c = code.to(torch.int32)
    size = c & 127 if signed else c
    bits = (size.view(-1, BLOCK) + offset.to(torch.int32)[:, None]).clamp(max=0x7FF).view(-1) << 20
    x = torch.where(size == 0, 0, bits).view(torch.float32)
    return torch.where(c >= 128, -x, x) if signed else x


def _plain_adamw(s):
    case, h = s["case"], HYPER
    bc1, bc2 = 1.0 - h["beta1"] ** case["step"], 1.0 - h["beta2"] ** case["step"]
    g = s["g"].float()
    if s["scale"] is not None:
        g = g * s["scale"]
    if case["bits"] == 8:
        m, v = _decode(s["m"], s["mo"], True), _decode(s["v"], s["vo"], False)
    else:
        m, v = s["m"], s["v"]
    m = m * h["beta1"] + g * (1.0 - h["beta1"])
    v = v * h["beta2"] + (g * g) * (1.0 - h["beta2"])
    step = m / (torch.sqrt(v) * (1.0 / math.sqrt(bc2)) + h["eps"])
    p = s["p"].float() if s["low"] is None else _join(s["p"], s["low"])
    p = p * (1.0 - h["lr"] * h["weight_decay"]) - step * (h["lr"] / bc1)
    out = {}
    if s["low"] is not None:
        high, low = _split(p)
        s["p"].copy_(high)
        out["low"] = s["low"].copy_(low)
    else:
        s["p"].copy_(p.to(s["p"].dtype))
    out["p"] = s["p"]
    if case["bits"] == 8:
        for name, x, signed in (("m", m, True), ("v", v, False)):
            code, offset = _encode(x, s["index"], case["step"], signed)
            s[name].copy_(code)
            s[name + "o"].copy_(offset)
            out[name] = _decode(code, offset, signed).to(torch.bfloat16)      # (exact: three bits of mantissa)
    else:
        out["m"], out["v"] = s["m"].copy_(m), s["v"].copy_(v)
    return out


def _plain(s):
    case = s["case"]
    if case["kind"] == "forward":
        pre = s["x"].float() @ s["w"].float().t()
        if s["b"] is not None:
            pre = pre + s["b"].float()
        gate, up = pre.chunk(2, 1)
        h = (_act(gate, case["act"]) * up).to(s["x"].dtype)
        return {"h": h, "pre": pre.to(s["x"].dtype)} if case["save"] else {"h": h}
    if case["kind"] == "backward":
        gate, up = s["pre"].float().chunk(2, 1)
        dh = s["dh"].float()
        dpre = torch.cat([dh * up * _slope(gate, case["act"]), dh * _act(gate, case["act"])], 1)
        out = {"dpre": dpre.to(s["dh"].dtype), "dx": (dpre @ s["w"].float()).to(s["dh"].dtype)}
        if case["bias"]:
            out["dbias"] = dpre.sum(0)
        return out
    if case["kind"] == "norm":
        norm = torch.sqrt(s["g"].float().square().sum())
        return {"norm": torch.stack([norm, torch.clamp(1.0 / (norm + 1e-6), max=1.0)])}
    return _plain_adamw(s)


def run(s):
    if not own:
        return _plain(s)
    import paper_2202_13808_amd as dropit
    case = s["case"]
    if case["kind"] == "forward":
        if case["save"]:
            h, pre = dropit.gated_forward(s["x"], s["w"], s["b"], act=case["act"], save=True)
            return {"h": h, "pre": pre}
        return {"h": dropit.gated_forward(s["x"], s["w"], s["b"], act=case["act"])}
    if case["kind"] == "backward":
        dpre, dx, dbias = dropit.gated_backward(s["dh"], s["pre"], s["w"], act=case["act"], need_dbias=case["bias"])
        return {"dpre": dpre, "dx": dx, "dbias": dbias} if case["bias"] else {"dpre": dpre, "dx": dx}
    if case["kind"] == "norm":
        return {"norm": dropit.grad_norm(s["g_list"], max_norm=1.0)}
    more = {"m_offset": s["mo_list"], "v_offset": s["vo_list"]} if case["bits"] == 8 else {}
    dropit.adamw(s["p_list"], s["g_list"], s["m_list"], s["v_list"], lr=HYPER["lr"], betas=(HYPER["beta1"], HYPER["beta2"]),
                 eps=HYPER["eps"], weight_decay=HYPER["weight_decay"], step=case["step"], grad_scale=s["scale"],
                 residual=s["low_list"] if case["residual"] else None, **more)
    out = {"low": s["low"]} if case["residual"] else {}
    out["p"] = s["p"]
    if case["bits"] == 8:
        out["m"], out["v"] = dropit.adamw_unpack(s["m"], s["mo"], signed=True), dropit.adamw_unpack(s["v"], s["vo"], signed=False)
    else:
        out["m"], out["v"] = s["m"], s["v"]
    return out


# ---- what a pass cannot do without ----------------------------------------------------------------
def work(case):
    if case["kind"] in ("forward", "backward"):
        size, t, c, h = (2 if case["dtype"] == "bf16" else 4), case["tokens"], case["c"], case["hidden"]
        moved = t * c + 2 * h * c + (t * h * (3 if case["save"] else 1) if case["kind"] == "forward" else 5 * t * h)
        return {"bytes": size * moved + (size * 2 * h if case["bias"] else 0), "flops": 4 * t * c * h}
    n = sum(math.prod(x) for x in _shapes(case))
    g = 2 if case["g"] == "bf16" else 4
    if case["kind"] == "norm":
        return {"bytes": n * g, "flops": 2 * n}
    p = 2 * (2 if case["p"] == "bf16" else 4) + (4 if case["residual"] else 0)
    return {"bytes": n * (p + g + (4 + 4 if case["bits"] == 8 else 16)), "flops": 20 * n}


# ---- the definitions in 64 bits -------------------------------------------------------------------
def _gate64(z, act):
    if act == "silu":
        return z * torch.special.expit(z)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "gelu_tanh":
        return z * torch.special.expit(math.sqrt(8.0 / math.pi) * (z + 0.044715 * z ** 3))
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    return torch.special.expit(z)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        norm = torch.linalg.vector_norm(s["g"].double())
        return {"norm": torch.stack([norm, 1.0 / torch.clamp(norm + 1e-6, min=1.0)])}
    if case["kind"] in ("forward", "backward"):
        w, hidden = s["w"].double(), case["hidden"]
        if case["kind"] == "forward":
            pre = torch.mm(s["x"].double(), w.t().contiguous())
            if s["b"] is not None:
                pre += s["b"].double()
            h = _gate64(pre[:, :hidden], case["act"]) * pre[:, hidden:]
            return {"h": h, "pre": pre} if case["save"] else {"h": h}
        pre = s["pre"].double().requires_grad_(True)
        h = _gate64(pre[:, :hidden], case["act"]) * pre[:, hidden:]
        (dpre,) = torch.autograd.grad(h, pre, s["dh"].double())
        out = {"dpre": dpre, "dx": torch.mm(dpre, w)}
        if case["bias"]:
            out["dbias"] = dpre.sum(0)
        return out
    h, t = HYPER, case["step"]
    g = s["g"].double() * (s["scale"].double() if s["scale"] is not None else 1.0)
    wide = case["bits"] == 32
    m = (s["m"] if wide else _decode(s["m"], s["mo"], True)).double()
    v = (s["v"] if wide else _decode(s["v"], s["vo"], False)).double()
    p = (s["p"].float() if s["low"] is None else _join(s["p"], s["low"])).double()
    m = torch.lerp(g, m, h["beta1"])
    v = torch.lerp(g ** 2, v, h["beta2"])
    bc1, bc2 = -math.expm1(t * math.log(h["beta1"])), -math.expm1(t * math.log(h["beta2"]))
    p = (1.0 - h["lr"] * h["weight_decay"]) * p - h["lr"] * (m / bc1) / (torch.sqrt(v / bc2) + h["eps"])
    out = {"low": None} if case["residual"] else {}
    out["p"] = p
    if wide:
        out["m"], out["v"] = m, v
    else:
        for name, x, signed in (("m", m, True), ("v", v, False)):
            out[name] = _decode(*_encode(x.float(), s["index"], t, signed), signed).double()
    return out
