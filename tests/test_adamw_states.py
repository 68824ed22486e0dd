"""State dictionaries of optim.AdamW and their hooks, without a GPU."""
import copy

import pytest
import torch

from paper_2104_06700_b200 import optim


def optimiser(value):
    """An optimiser of an fp32 and a bf16 parameter with states as a GPU's steps leave them."""
    p, q = torch.nn.Parameter(torch.zeros(5)), torch.nn.Parameter(torch.zeros(3, dtype=torch.bfloat16))
    opt = optim.AdamW([p, q], lr=1e-3 * (1 + value), master_weights=True, max_norm=1.0)
    for t, master in ((p, None), (q, torch.full((3,), value + 2.0 ** -20))):
        opt.state[t] = {"step": torch.tensor(int(value)), "exp_avg": torch.full(t.shape, value + 2.0 ** -20),
                        "exp_avg_sq": torch.full(t.shape, value).to(torch.float8_e4m3fn)}
        if master is not None:
            opt.state[t]["master"] = master
    return opt, p, q


def holds(opt, p, q, value):
    for t in (p, q):
        s = opt.state[t]
        assert s["step"].dtype == torch.int64 and int(s["step"]) == int(value)
        assert torch.equal(s["exp_avg"], torch.full(t.shape, value + 2.0 ** -20)) and s["exp_avg"].dtype == torch.float32
        assert s["exp_avg_sq"].dtype == torch.float8_e4m3fn and bool((s["exp_avg_sq"].float() == value).all())
    assert torch.equal(opt.state[q]["master"], torch.full((3,), value + 2.0 ** -20))
    assert opt.param_groups[0]["lr"] == 1e-3 * (1 + value)


def test_states_keep_their_types_and_are_copies():
    saved = optimiser(2.0)[0].state_dict()
    opt, p, q = optimiser(1.0)
    opt.load_state_dict(saved)
    holds(opt, p, q, 2.0)
    assert opt.state[p]["exp_avg"] is not saved["state"][0]["exp_avg"]
    opt.state[p]["exp_avg"].zero_()
    assert bool(saved["state"][0]["exp_avg"].all())


@pytest.mark.parametrize("prepend", [False, True])
def test_a_hook_may_return_another_dictionary(prepend):
    saved, other = optimiser(2.0)[0].state_dict(), optimiser(3.0)[0].state_dict()
    opt, p, q = optimiser(1.0)
    opt.register_load_state_dict_pre_hook(lambda _, given: other if given["state"][0]["step"] == 2 else None, prepend=prepend)
    opt.load_state_dict(saved)
    holds(opt, p, q, 3.0)
    opt.load_state_dict(optimiser(1.0)[0].state_dict())      # the hook leaves this one
    holds(opt, p, q, 1.0)


def test_hooks_behind_it_see_and_may_change_the_states():
    opt, p, q = optimiser(1.0)
    seen = []

    def behind(o):
        seen.append((o.state[q]["master"].dtype, o.state[p]["exp_avg_sq"].dtype))
        o.state[p]["step"] = o.state[p]["step"] * 0

    opt.register_load_state_dict_post_hook(behind, prepend=True)
    opt.load_state_dict(optimiser(2.0)[0].state_dict())
    assert seen == [(torch.float32, torch.float8_e4m3fn)] and int(opt.state[p]["step"]) == 0
    opt.load_state_dict(copy.deepcopy(optimiser(2.0)[0].state_dict()))
    assert len(seen) == 2


def test_a_dictionary_that_does_not_fit_changes_nothing():
    opt, p, q = optimiser(1.0)
    saved = optim.AdamW([torch.nn.Parameter(torch.zeros(5))]).state_dict()
    with pytest.raises(ValueError):
        opt.load_state_dict(saved)
    holds(opt, p, q, 1.0)
    opt.load_state_dict(optimiser(2.0)[0].state_dict())
    holds(opt, p, q, 2.0)
