"""optim.AdamW on the GPU: refusals that change nothing, states that were loaded, steps captured into a graph."""
import copy

import pytest
import torch

import paper_2202_13808_amd as dropit

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
