"""optim.AdamW on the GPU: refusals that change nothing, states that were loaded, steps captured into a graph."""
import copy

import pytest
import torch
import torch.nn.functional as F

import paper_2202_13808_amd as dropit
from paper_2202_13808_amd import block_bench
from paper_2202_13808_amd import nn as dnn

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def test_a_group_over_several_devices_is_refused_before_anything_changes():
    print("optim devices", flush=True)
    p, q = torch.nn.Parameter(torch.zeros(300, device=DEV)), torch.nn.Parameter(torch.zeros(300))
    p.grad, q.grad = torch.ones_like(p), torch.ones_like(q)
    opt = dropit.optim.AdamW([p, q])
    for _ in range(2):
        with pytest.raises(RuntimeError, match="one device"):
            opt.step()
    assert all(not opt.state[t] or opt.state[t]["step"] == 0 for t in (p, q)) and not bool(p.any())
    split = dropit.optim.AdamW([{"params": [p]}, {"params": [q]}])
    with pytest.raises(RuntimeError, match="no CPU path"):
        split.step()
    assert not split.state[p] or split.state[p]["step"] == 0
    assert not bool(p.any())
    q.grad = None
    split.step()                                       # the device's group alone
    assert split.state[p]["step"] == 1 and bool((p != 0).all())


@pytest.mark.parametrize("copied", [copy.deepcopy], ids=["deepcopy"])
def test_a_copy_of_the_optimizer_steps_as_it_does(copied):
    print("optim copy", flush=True)
    g = torch.Generator(device=DEV).manual_seed(3)
    p = torch.nn.Parameter(torch.randn(3000, generator=g, device=DEV))
    opt = dropit.optim.AdamW([p], max_norm=0.5, state_bits=8)
    p.grad = torch.randn(3000, generator=g, device=DEV)
    opt.step()
    other = copied(opt)
    (q,) = other.param_groups[0]["params"]
    p.grad = torch.randn(3000, generator=g, device=DEV)
    q.grad = p.grad.clone()
    opt.step()
    other.step()
    assert torch.equal(p, q) and torch.equal(opt.last_grad_norm, other.last_grad_norm) and float(other.last_grad_norm) > 0.5


@pytest.mark.parametrize("bits", [32, 8])
def test_a_loaded_capturable_group_counts_for_all_its_parameters(bits):
    print("optim loaded counts", bits, flush=True)
    g = torch.Generator(device=DEV).manual_seed(4)
    params = [torch.nn.Parameter(torch.randn(n, generator=g, device=DEV)) for n in (300, 5000)]
    grads = [[torch.randn(p.shape, generator=g, device=DEV) for p in params] for _ in range(4)]

    def run(opt, params, some):
        for gs in some:
            for p, x in zip(params, gs):
                p.grad = x
            opt.step()

    opt = dropit.optim.AdamW(params, state_bits=bits, capturable=True)
    run(opt, params, grads[:2])
    sd = opt.state_dict()
    sd["state"] = {i: {k: v.cpu() for k, v in s.items()} for i, s in sd["state"].items()}       # each tensor by itself
    others = [torch.nn.Parameter(p.detach().clone()) for p in params]
    again = dropit.optim.AdamW(others, state_bits=bits, capturable=True)
    again.load_state_dict(sd)
    run(opt, params, grads[2:])
    run(again, others, grads[2:])
    assert [int(again.state[q]["step"]) for q in others] == [4, 4]
    for p, q in zip(params, others):
        assert torch.equal(p, q)


def _master(opt, p):
    """What a step moves: an update of lr = 1e-3 is less than half a step of a bfloat16 of 0.5, so it may show in the residual only."""
    residual = opt.state[p].get("residual")
    return p.detach().clone() if residual is None else torch.stack([p.detach().float(), residual.float()])


def _same(a_params, a, b_params, b):
    for p, q in zip(a_params, b_params):
        assert torch.equal(p, q)
        for k in a.state[p]:
            assert torch.equal(a.state[p][k], b.state[q][k]), k
    assert torch.equal(a.last_grad_norm, b.last_grad_norm)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [32, 8])
def test_a_captured_step_makes_the_bits_of_an_eager_one(bits, dtype):
    print("optim captured bits", bits, dtype, flush=True)
    g = torch.Generator(device=DEV).manual_seed(6)
    sizes = [(300,), (64, 65), (7, 5000), (1,)]
    eager = [torch.nn.Parameter(torch.randn(s, generator=g, device=DEV).to(dtype)) for s in sizes]
    captured = [torch.nn.Parameter(p.detach().clone()) for p in eager]
    make = lambda params: dropit.optim.AdamW(params, lr=1e-3, state_bits=bits, max_norm=1.0, capturable=True)  # noqa: E731
    eo, co = make(eager), make(captured)

    def feed(scale):
        for p, q in zip(eager, captured):
            x = (scale * torch.randn(p.shape, generator=g, device=DEV)).to(dtype)
            for t in (p, q):
                t.grad = x.clone() if t.grad is None else t.grad.copy_(x)

    feed(1.0)
    eo.step()
    co.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        co.step()
    for t, scale in enumerate((1.0, 1e-6, 30.0, 1.0)):             # clipped and not
        feed(scale)
        before = [_master(co, p) for p in captured]
        graph.replay()
        eo.step()
        torch.cuda.synchronize()
        _same(eager, eo, captured, co)
        if scale == 1.0:
            assert all(bool((_master(co, p) != b).any()) for p, b in zip(captured, before))
        assert int(co.state[captured[0]]["step"]) == t + 2


@pytest.mark.parametrize("bits", [32, 8])
def test_training_steps_captured_into_a_graph_make_the_bits_of_eager_ones(bits):
    print("train captured bits", bits, flush=True)
    x = torch.randn(4, 20, 64, device=DEV, dtype=torch.bfloat16)
    target = torch.randint(0, 10, (4,), device=DEV)

    def make():
        torch.manual_seed(11)
        net = block_bench.encoder(2, 64, 2, 256, 10, gated=True).to(DEV, torch.bfloat16)
        dnn.apply_dropit(net, 0.8)
        return net, dropit.optim.AdamW(net.parameters(), lr=1e-3, state_bits=bits, max_norm=1.0, capturable=True)

    def train(net, opt):
        opt.zero_grad(set_to_none=False)
        F.cross_entropy(net(x).float(), target).backward()
        opt.step()

    (eager, eo), (captured, co) = make(), make()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            train(eager, eo)
            train(captured, co)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        train(captured, co)
    for _ in range(4):
        x.copy_(torch.randn(4, 20, 64, device=DEV, dtype=torch.bfloat16))
        before = [_master(co, q) for q in captured.parameters()]
        graph.replay()
        torch.cuda.synchronize()
        train(eager, eo)
        torch.cuda.synchronize()
        for (name, p), q, b in zip(eager.named_parameters(), captured.parameters(), before):
            assert torch.equal(p.grad, q.grad), name
            assert bool((_master(co, q) != b).any()), name
        _same(list(eager.parameters()), eo, list(captured.parameters()), co)
