"""The norm gradient's workspace holds a row of sums for each row of the input, 304 at most, whatever their length (no GPU)."""

import pytest


@pytest.fixture(scope="module")
def mpc():
    import __graft_entry__ as g

    g.build()
    import paper_2401_07788_gb300 as m

    return m


@pytest.mark.parametrize("D", [64, 8192, 8193, 17000, 1 << 24])
@pytest.mark.parametrize("rows", [1, 2, 7, 303, 304, 305, 100000])
def test_grows_with_the_rows(mpc, rows, D):
    parts = min(rows, 304)
    dots = rows if D > 8192 else 0  # fp32 rows that are read twice
    assert mpc.mpc_rms_norm_workspace_bytes(rows, D) == 4 * (parts * D + dots)
