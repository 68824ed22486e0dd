"""Options of optim.AdamW's parameter groups, without a GPU: a group's own options are checked like the optimiser's."""
import pytest
import torch

from paper_2104_06700_b200 import optim

WRONG = [dict(state_bits=16), dict(state_bits=4), dict(lr=-1.0), dict(lr=float("nan")), dict(eps=-1e-8), dict(weight_decay=-0.1),
         dict(betas=(0.9, 1.0)), dict(betas=(-0.1, 0.9)), dict(betas=(0.9,))]


def parameter():
    return torch.nn.Parameter(torch.zeros(8))


@pytest.mark.parametrize("wrong", WRONG)
def test_options_of_a_group_are_refused(wrong):
    with pytest.raises(ValueError):
        optim.AdamW([{"params": [parameter()], **wrong}])
    opt = optim.AdamW([parameter()])
    late = parameter()
    with pytest.raises(ValueError):
        opt.add_param_group({"params": [late], **wrong})
    assert len(opt.param_groups) == 1
    opt.add_param_group({"params": [late]})              # it was not taken
    assert len(opt.param_groups) == 2


def test_groups_with_options_of_their_own():
    opt = optim.AdamW([{"params": [parameter()], "state_bits": 8, "lr": 0.0, "weight_decay": 0.0}, {"params": [parameter()]}],
                      betas=(0.0, 0.9), seed=3)
    assert [g["state_bits"] for g in opt.param_groups] == [8, 32] and [g["lr"] for g in opt.param_groups] == [0.0, 1e-3]
    with pytest.raises(ValueError):
        optim.AdamW([parameter()], betas=(0.9,))
