"""dropit_gated_forward / dropit_gated_backward on the GPU against the formulas in 64 bits.

Tolerances, per element.  A product of K terms: K + 4 roundings of 2^-24 of the sum of the terms' magnitudes.  The
activations have slopes of at most 1.13 and, in bf16, errors of at most 2^-18 (1 + |z|)^2 (the exponential's argument is
rounded to 2^-24 of itself and the hardware adds 2^-22; its products with z and its square follow), in fp32 32 x 2^-24
(1 + |z|).  What leaves in bf16 is off by half a step more, 2^-8 of itself, in fp32 by 2^-24."""
import math

import pytest
import torch

import paper_2202_13808_amd as dropit

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
ACTS = ["silu", "gelu", "gelu_tanh", "relu", "sigmoid"]


def act64(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    return torch.sigmoid(z)


def act_error(z, dtype):
    return 2.0 ** -18 * (1 + z.abs()) ** 2 if dtype == "bf16" else 32 * 2.0 ** -24 * (1 + z.abs())


def guarded(shape, dtype):
    """A tensor of that shape in the middle of a larger one of sevens."""
    n = math.prod(shape)
    around = torch.full((n + 64,), 7.0, dtype=dtype, device=DEV)
    return around[32:32 + n].view(shape), around


def intact(around):
    return bool((around[:32] == 7).all()) and bool((around[-32:] == 7).all())


def inputs(tokens, c, hidden, dtype, bias, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(tokens, c, generator=g).to(DT[dtype])
    w = (torch.randn(2 * hidden, c, generator=g) / math.sqrt(c)).to(DT[dtype])
    b = (0.3 * torch.randn(2 * hidden, generator=g)).to(DT[dtype]) if bias else None
    dh = (0.02 * torch.randn(tokens, hidden, generator=g)).to(DT[dtype])
    return x, w, b, dh


def check_forward(x, w, b, act, dtype, h, pre):
    hidden = w.shape[0] // 2
    x, w = x.double(), w.double()
    ref = x @ w.t()
    size = x.abs() @ w.abs().t()
    if b is not None:
        ref, size = ref + b.double(), size + b.double().abs()
    off = (x.shape[1] + 4) * 2.0 ** -24 * size
    if pre is not None:
        assert bool(((pre.cpu().double() - ref).abs() <= off + HALF[dtype] * ref.abs()).all())
    g, u = ref[:, :hidden], ref[:, hidden:]
    a = act64(g, act)
    want = a * u
    tol = (1.13 * off[:, :hidden] + act_error(g, dtype)) * u.abs() + a.abs() * off[:, hidden:] + HALF[dtype] * want.abs() + 1e-30
    d = (h.cpu().double() - want).abs()
    assert bool((d <= 1.01 * tol).all()), float((d / tol).max())


def check_backward(dh, pre, w, act, dtype, dpre, dx, dbias):
    hidden = w.shape[0] // 2
    z = pre.double().requires_grad_(True)
    h = act64(z[:, :hidden], act) * z[:, hidden:]
    (ref,) = torch.autograd.grad(h, z, dh.double())
    g, u = pre.double()[:, :hidden], pre.double()[:, hidden:]
    d = dh.double().abs()
    off = torch.cat([d * u.abs() * act_error(g, dtype), d * act_error(g, dtype)], 1) + 4 * 2.0 ** -24 * ref.abs()
    diff = (dpre.cpu().double() - ref).abs()
    tol = off + HALF[dtype] * ref.abs() + 1e-30
    assert bool((diff <= 1.01 * tol).all()), float((diff / tol).max())
    if dx is not None:
        have = dpre.cpu().double()
        want = have @ w.double()
        tol = (2 * hidden + 4) * 2.0 ** -24 * (have.abs() @ w.double().abs()) + HALF[dtype] * want.abs() + 1e-30
        diff = (dx.cpu().double() - want).abs()
        assert bool((diff <= 1.01 * tol).all()), float((diff / tol).max())
    if dbias is not None:
        # 16 rows a thread, four groups, 16 chains of row blocks: fewer than 64 + tokens / 1024 roundings of the sum of sizes
        tol = off.sum(0) + (64 + dh.shape[0] / 1024) * 2.0 ** -24 * ref.abs().sum(0) + 1e-30
        diff = (dbias.cpu().double() - ref.sum(0)).abs()
        assert bool((diff <= 1.01 * tol).all()), float((diff / tol).max())


def run_case(tokens, c, hidden, dtype, act, bias, seed=3, shape=None):
    print("gated", tokens, c, hidden, dtype, act, bias, flush=True)
    x, w, b, dh = inputs(tokens, c, hidden, dtype, bias, seed)
    xd, wd, bd, dhd = (t.to(DEV) if t is not None else None for t in (x, w, b, dh))
    h, h_around = guarded((tokens, hidden), DT[dtype])
    pre, pre_around = guarded((tokens, 2 * hidden), DT[dtype])
    dropit.gated_forward(xd, wd, bd, act=act, h=h, pre=pre)
    only_h = dropit.gated_forward(xd, wd, bd, act=act)
    torch.cuda.synchronize()
    assert intact(h_around) and intact(pre_around)
    assert torch.equal(only_h, h)                      # saving changes nothing
    check_forward(x, w, b, act, dtype, h, pre)
    dpre, dpre_around = guarded((tokens, 2 * hidden), DT[dtype])
    dx, dx_around = guarded((tokens, c), DT[dtype])
    dbias, dbias_around = guarded((2 * hidden,), torch.float32)
    dropit.gated_backward(dhd, pre, wd, act=act, dpre=dpre, dx=dx, dbias=dbias)
    torch.cuda.synchronize()
    assert intact(dpre_around) and intact(dx_around) and intact(dbias_around)
    check_backward(dh, pre.cpu(), w, act, dtype, dpre, dx, dbias)
    again = dropit.gated_backward(dhd, pre, wd, act=act, need_dbias=True)
    for a, b in zip(again, (dpre, dx, dbias)):
        assert torch.equal(a, b)                       # the same bits run to run
    some = dropit.gated_backward(dhd, pre, wd, act=act, need_dx=False)
    assert torch.equal(some[0], dpre) and some[1] is None and some[2] is None


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,c,hidden", [(1, 1, 1), (1, 8, 4), (3, 7, 5), (1, 384, 1024), (2, 64, 64), (15, 40, 24), (16, 128, 64),
                                             (17, 136, 72), (33, 100, 515), (64, 512, 96), (65, 387, 66), (257, 96, 40),
                                             (300, 256, 260), (1003, 48, 129), (130, 2056, 8), (700, 264, 332)])
def test_sizes(tokens, c, hidden, dtype):
    run_case(tokens, c, hidden, dtype, "silu", bias=hidden % 2 == 0)


@pytest.mark.parametrize("tokens,c,hidden", [
    (4001, 515, 1027), (2500, 1030, 770),              # rows that are no whole 16-byte units, copied into such
    (100, 2048, 131), (70, 4096, 40),                  # few tiles: the sum in slices, odd width and even
    (16384, 64, 512), (32768, 512, 32),                # 256 and 192 tokens to a tile, several tiles a workgroup
    (12608, 128, 2048), (9400, 72, 2041), (4660, 64, 4100)])           # the last tiles not full
def test_larger_products(tokens, c, hidden):
    run_case(tokens, c, hidden, "bf16", "gelu", bias=True, seed=6)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ACTS)
def test_activations(act, dtype):
    run_case(90, 72, 48, dtype, act, bias=True, seed=4)
    run_case(520, 64, 264, dtype, act, bias=True, seed=5)


@pytest.mark.parametrize("act", ACTS)
def test_far_and_special_gates(act):
    # pre-activations from one-hot tokens: 0, far out on both sides, next to overflow
    print("gated far", act, flush=True)
    values = [0.0, -0.0, 1e-30, 5.0, -5.0, 20.0, -20.0, 90.0, -90.0, 1e4, -1e4, 3e18]
    n = len(values)
    for dtype in ("f32", "bf16"):
        w = torch.zeros(2 * n, 8, dtype=DT[dtype])
        w[:n, 0] = torch.tensor(values, dtype=DT[dtype])
        w[n:, 0] = 1.0
        x = torch.zeros(2, 8, dtype=DT[dtype])
        x[0, 0] = 1.0
        h, pre = dropit.gated_forward(x.to(DEV), w.to(DEV), act=act, save=True)
        check_forward(x, w, None, act, dtype, h, pre)
        dh = torch.ones(2, n, dtype=DT[dtype])
        dpre, dx, _ = dropit.gated_backward(dh.to(DEV), pre, w.to(DEV), act=act)
        z = pre.cpu().double().requires_grad_(True)
        (ref,) = torch.autograd.grad(act64(z[:, :n], act) * z[:, n:], z, dh.double())
        ok = ref.isfinite()
        assert bool(dpre.cpu().isfinite()[ok].all())
        diff = (dpre.cpu().double() - ref).abs()[ok]
        tol = (act_error(z.detach()[:, :n].clamp(-100, 100), dtype).repeat(1, 2) + 2 * HALF[dtype] * ref.abs())[ok] + 1e-30
        assert bool((diff <= tol).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,c,hidden", [(5, 40, 24), (20, 72, 40), (300, 264, 136)])
def test_values_that_are_not_finite_touch_their_own_rows_and_columns(tokens, c, hidden, dtype):
    print("gated nonfinite", tokens, c, hidden, dtype, flush=True)
    x, w, b, dh = inputs(tokens, c, hidden, dtype, True, 8)
    x[2, 3] = float("nan")
    x[4, c - 1] = float("inf")
    w[7] = float("inf")
    h, pre = dropit.gated_forward(x.to(DEV), w.to(DEV), b.to(DEV), save=True)
    fine = torch.ones(tokens, hidden, dtype=torch.bool)
    fine[2], fine[4], fine[:, 7] = False, False, False
    assert bool(h.cpu().isfinite()[fine].all()) and not bool(h.cpu().isfinite()[2].any()) and not bool(h.cpu().isfinite()[:, 7].all())
    x, w, b, dh = inputs(tokens, c, hidden, dtype, True, 8)
    pre = torch.randn(tokens, 2 * hidden, dtype=torch.float32).to(DT[dtype])
    dh[3, 5] = float("nan")
    w[:, 6] = float("inf")
    dpre, dx, dbias = dropit.gated_backward(dh.to(DEV), pre.to(DEV), w.to(DEV), need_dbias=True)
    ok = torch.ones(tokens, 2 * hidden, dtype=torch.bool)
    ok[3, 5] = ok[3, hidden + 5] = False
    assert bool((dpre.cpu().isfinite() == ok).all())
    cols = torch.ones(c, dtype=torch.bool)
    cols[6] = False
    rows = torch.ones(tokens, dtype=torch.bool)
    rows[3] = False
    assert bool(dx.cpu().isfinite()[rows][:, cols].all()) and bool(dx.cpu()[3].isnan().all()) and not bool(dx.cpu()[:, 6].isfinite().any())
    bad = ~dbias.cpu().isfinite()
    assert bad.nonzero().flatten().tolist() == [5, hidden + 5]


def test_gradients_against_differences():
    print("gated differences", flush=True)
    tokens, c, hidden = 6, 12, 9
    for act in ACTS:
        x, w, b, dh = inputs(tokens, c, hidden, "f32", True, 12)
        dh = dh * 50
        _, pre = dropit.gated_forward(x.to(DEV), w.to(DEV), b.to(DEV), act=act, save=True)
        _, dx, dbias = dropit.gated_backward(dh.to(DEV), pre, w.to(DEV), act=act, need_dbias=True)

        def loss(x, b):
            p = x @ w.double().t() + b
            return float((act64(p[:, :hidden], act) * p[:, hidden:] * dh.double()).sum())

        step = 1e-4                                    # differences of 64-bit values: off by step^2 and 1e-16 / step
        for i, j in ((0, 0), (5, 11), (2, 7)):
            e = torch.zeros(tokens, c, dtype=torch.double)
            e[i, j] = step
            slope = (loss(x.double() + e, b.double()) - loss(x.double() - e, b.double())) / (2 * step)
            assert abs(slope - float(dx[i, j])) <= 2e-5 * (1 + abs(slope))
        for j in (0, hidden, 2 * hidden - 1):
            e = torch.zeros(2 * hidden, dtype=torch.double)
            e[j] = step
            slope = (loss(x.double(), b.double() + e) - loss(x.double(), b.double() - e)) / (2 * step)
            assert abs(slope - float(dbias[j])) <= 2e-5 * (1 + abs(slope))


def test_leading_dimensions_empty_batches_and_streams():
    print("gated shapes", flush=True)
    x, w, b, dh = (t.to(DEV) for t in inputs(24, 64, 32, "bf16", True, 9))
    h, pre = dropit.gated_forward(x, w, b, save=True)
    h3, pre3 = dropit.gated_forward(x.view(2, 3, 4, 64), w, b, save=True)
    assert h3.shape == (2, 3, 4, 32) and torch.equal(h3.view(24, 32), h) and torch.equal(pre3.view(24, 64), pre)
    assert torch.equal(dropit.gated_forward(x[0], w, b), dropit.gated_forward(x[:1], w, b)[0])
    empty = dropit.gated_forward(x[:0], w, b, save=True)
    assert empty[0].shape == (0, 32) and empty[1].shape == (0, 64)
    dpre, dx, dbias = dropit.gated_backward(dh[:0], pre[:0], w, need_dbias=True)
    assert dpre.shape == (0, 64) and dx.shape == (0, 64) and dbias.tolist() == [0.0] * 64
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = dropit.gated_forward(x, w, b)
    s.synchronize()
    assert torch.equal(other, h)
    late = torch.empty_like(h)
    dropit.gated_forward(x, w, b, h=late, stream=s)
    s.synchronize()
    assert torch.equal(late, h)


def test_what_a_call_allocates_belongs_to_its_stream():
    print("gated allocation", flush=True)
    x, w, b, dh = (t.to(DEV) for t in inputs(600, 264, 520, "bf16", True, 12))
    h, pre = dropit.gated_forward(x, w, b, save=True)
    back = dropit.gated_backward(dh, pre, w, need_dbias=True)
    norm = dropit.grad_norm([x, w])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    # memory that the current stream will still write: freed here, it may serve this stream, not another
    doomed = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in (600 * 520 * 2, 600 * 1040 * 2, 600 * 264 * 2, 2 << 20, 4096, 512)]
    torch.cuda._sleep(20_000_000)
    for d in doomed:
        d.fill_(255)
    del doomed, d
    got = dropit.gated_forward(x, w, b, save=True, stream=side)
    got_back = dropit.gated_backward(dh, pre, w, need_dbias=True, stream=side)
    got_norm = dropit.grad_norm([x, w], stream=side)
    torch.cuda.synchronize()
    for mine, other in zip((h, pre) + back + (norm,), got + got_back + (got_norm,)):
        assert torch.equal(mine, other)


@pytest.mark.parametrize("tokens,c,hidden,dtype", [(3, 512, 64, "bf16"), (40, 512, 48, "f32"), (600, 264, 520, "bf16")])
def test_graph_replays_follow_their_inputs(tokens, c, hidden, dtype):
    print("gated graph", tokens, c, hidden, dtype, flush=True)
    x, w, b, dh = (t.to(DEV) for t in inputs(tokens, c, hidden, dtype, True, 10))

    def both():
        h, pre = dropit.gated_forward(x, w, b, act="gelu", save=True)
        return (h, pre) + dropit.gated_backward(dh, pre, w, act="gelu", need_dbias=True)

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for seed in (21, 22, 23):
        fresh = inputs(tokens, c, hidden, dtype, True, seed)
        for t, f in zip((x, w, b, dh), fresh):
            t.copy_(f)
        graph.replay()
        torch.cuda.synchronize()
        for a, e in zip(got, both()):
            assert torch.equal(a, e)


def test_outputs_beyond_two_to_the_31_elements():
    # 70016 tokens of 2 x 16384 pre-activations: offsets pass 2^31 elements (and 2^32 bytes)
    print("gated large", flush=True)
    tokens, c, hidden = 70016, 8, 16384
    g = torch.Generator(device=DEV).manual_seed(5)
    x = torch.randn(tokens, c, generator=g, device=DEV).bfloat16()
    w = (torch.randn(2 * hidden, c, generator=g, device=DEV) / 3).bfloat16()
    h, pre = dropit.gated_forward(x, w, save=True)
    dh = (h * 0.01).contiguous()
    dpre, dx, _ = dropit.gated_backward(dh, pre, w)
    for rows in (slice(0, 3), slice(65530, 65540), slice(tokens - 3, tokens)):
        check_forward(x[rows].cpu(), w.cpu(), None, "silu", "bf16", h[rows], pre[rows])
        check_backward(dh[rows].cpu(), pre[rows].cpu(), w.cpu(), "silu", "bf16", dpre[rows], dx[rows], None)
