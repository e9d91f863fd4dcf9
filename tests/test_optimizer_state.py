"""optim.AdamW without a GPU: what copies of the optimizer and loaded states hold."""
import copy
import pickle

import pytest
import torch

import paper_2202_13808_amd as dropit


@pytest.mark.parametrize("copied", [copy.deepcopy, lambda o: pickle.loads(pickle.dumps(o))], ids=["deepcopy", "pickle"])
@pytest.mark.parametrize("max_norm", [None, 0.25])
def test_copies_clip_as_the_optimizer_does(copied, max_norm):
    p = torch.nn.Parameter(torch.zeros(4))
    opt = dropit.optim.AdamW([p], max_norm=max_norm)
    opt.last_grad_norm = torch.tensor(3.0)
    other = copied(opt)
    assert other.max_norm == max_norm and float(other.last_grad_norm) == 3.0
    assert other.param_groups[0]["state_bits"] == 32
    other.step()                                       # no gradients: nothing to do
    other.param_groups[0]["params"][0].grad = torch.ones(4)
    with pytest.raises(RuntimeError, match="no CPU path"):
        other.step()


def test_loading_a_state_keeps_the_own_clipping():
    p, q = (torch.nn.Parameter(torch.zeros(4)) for _ in range(2))
    a, b = dropit.optim.AdamW([p], max_norm=0.5), dropit.optim.AdamW([q], max_norm=2.0)
    a.load_state_dict(b.state_dict())
    assert a.max_norm == 0.5 and a.last_grad_norm is None
