"""Quantisation of few long rows: the slices of a row are doubled to fill the GPU as far as a cluster holds
them, on the GPU against the CPU oracle bit for bit."""

import numpy as np
import pytest
import torch

import oracle
from gpu_cases import assert_bits_equal, rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mpc():
    import __graft_entry__ as g

    g.build()
    import paper_2401_07788_gb300 as m

    torch.cuda.set_device(0)
    return m


@pytest.mark.parametrize("rows", [1, 3, 50])
@pytest.mark.parametrize("L", [17000, 24576, 24577, 40000, 49152, 57000])
def test_few_rows_of_three_to_seven_slices(mpc, rows, L):
    x = rows_of("normal", rows, L, rows + L)
    for bits in (3, 8):
        codes, scale, minv = mpc.mpc_quant_compress(torch.from_numpy(x).cuda(), bits)
        assert mpc.mpc_get_status() == 0
        oc, osc, omn = oracle.quant_compress(x, bits)
        assert_bits_equal(codes.cpu().numpy().view(np.uint32), oc, "codes")
        assert_bits_equal(scale.cpu().numpy(), osc, "scale")
        assert_bits_equal(minv.cpu().numpy(), omn, "min")
