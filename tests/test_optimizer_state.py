"""Copies of the optimizer and its saved states (host memory: no GPU, no step)."""

import copy
import pickle

import pytest
import torch


@pytest.fixture(scope="module")
def mpc():
    import paper_2401_07788_gb300 as m

    return m


def made(mpc, bits=8):
    torch.manual_seed(0)
    ps = [torch.nn.Parameter(torch.randn(300)), torch.nn.Parameter(torch.randn(7, 5))]
    opt = mpc.AdamW(ps, lr=2e-3, state_bits=bits, max_norm=0.5, copies={ps[1]: torch.zeros(7, 5, dtype=torch.bfloat16)})
    for p in ps:
        s = opt._state(p)
        s["step"] = 3
        s["exp_avg"].add_(7)
    return ps, opt


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("how", [copy.deepcopy, lambda x: pickle.loads(pickle.dumps(x))], ids=["deepcopy", "pickle"])
def test_a_copied_optimizer_is_whole(mpc, bits, how):
    """Options, states and bf16 copies come along, tied to the copied parameters; its lists are its own."""
    ps, opt = made(mpc, bits)
    model, twin = how((ps, opt))
    assert (twin.state_bits, twin.max_norm, twin.last_norm, twin._plans) == (bits, 0.5, None, {})
    assert [p for g in twin.param_groups for p in g["params"]][0] is model[0]
    assert list(twin.copies) == [model[1]] or [id(p) for p in twin.copies] == [id(model[1])]
    assert twin.copies[model[1]].dtype == torch.bfloat16
    for p, q in zip(ps, model):
        a, b = opt.state[p], twin.state[q]
        assert a.keys() == b.keys() and a["step"] == b["step"]
        assert torch.equal(a["exp_avg"], b["exp_avg"]) and a["exp_avg"] is not b["exp_avg"]
        assert a["exp_avg"].dtype == b["exp_avg"].dtype


@pytest.mark.parametrize("saved,here", [(32, 8), (8, 32)])
def test_states_of_other_bits_are_refused(mpc, saved, here):
    """States saved with one state_bits are not loaded into an optimizer of the other, which stays as it was."""
    _, old = made(mpc, saved)
    ps, opt = made(mpc, here)
    before = copy.deepcopy(opt.state_dict())
    with pytest.raises(ValueError, match="state_bits"):
        opt.load_state_dict(old.state_dict())
    after = opt.state_dict()
    assert after["param_groups"] == before["param_groups"]
    for i, s in before["state"].items():
        for k, x in s.items():
            assert torch.equal(x, after["state"][i][k]) if isinstance(x, torch.Tensor) else x == after["state"][i][k]


@pytest.mark.parametrize("bits", [32, 8])
def test_states_are_loaded_as_they_were_saved(mpc, bits):
    ps, old = made(mpc, bits)
    qs, opt = made(mpc, bits)
    for q in qs:
        opt.state[q]["exp_avg"].zero_()
        opt.state[q]["step"] = 0
    opt.load_state_dict(old.state_dict())
    for p, q in zip(ps, qs):
        a, b = old.state[p], opt.state[q]
        assert b["step"] == 3 and a["exp_avg"].dtype == b["exp_avg"].dtype and torch.equal(a["exp_avg"], b["exp_avg"])
        assert a["exp_avg"].data_ptr() != b["exp_avg"].data_ptr()
