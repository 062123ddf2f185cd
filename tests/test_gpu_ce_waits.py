"""Device-side waits of the matrix products that run out in some warps and not in others."""

import pytest
import torch

from test_gpu_linear_ce import inputs, mpc  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("limit", [1, 2, 20])
def test_waits_of_one_and_a_few_tries(mpc, dtype, limit):  # noqa: F811
    """Whichever wait gives up first, the kernels return with nothing in flight: the status says so, and the
    calls after that are as before."""
    h, w, y = inputs(600, 296, 3000, dtype, seed=70)
    before = mpc.mpc_linear_ce_train(h, w, y)
    lse = mpc.mpc_linear_ce_forward(h, w, y)[1]
    assert mpc.mpc_get_status() == 0
    mpc.mpc_set_knob(mpc.MPC_KNOB_SPIN_LIMIT, limit)
    try:
        mpc.mpc_linear_ce_train(h, w, y)
        mpc.mpc_linear_ce_backward(h, w, y, lse)
        assert mpc.mpc_get_status() in (0, 5)
    finally:
        mpc.mpc_set_knob(mpc.MPC_KNOB_SPIN_LIMIT, 1 << 20)
    assert mpc.mpc_get_status() == 0
    for a, b in zip(before, mpc.mpc_linear_ce_train(h, w, y)):
        assert torch.equal(a, b)
    assert mpc.mpc_get_status() == 0
