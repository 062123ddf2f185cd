"""The linear layer's workspace of a gradient call whose dz is dy itself (no activation, no dropout, a bf16 dy that the
matrix units read in place) has no room for another one (no GPU)."""

import pytest
import torch

P = 1 << 20  # an address that no call reaches


@pytest.fixture(scope="module")
def mpc():
    import __graft_entry__ as g

    g.build()
    import paper_2401_07788_gb300 as m

    m.lib()
    return m


def up(n):
    return (n + 255) // 256 * 256


@pytest.mark.parametrize("M,K,N", [(300, 64, 512), (16384, 4096, 16384), (70, 72, 80)])
def test_query(mpc, M, K, N):
    query = lambda plain, dtype=torch.bfloat16, **ld: mpc.mpc_linear_workspace_bytes(  # noqa: E731
        M, K, N, dtype, backward=True, plain=plain, **ld)
    dz = up(M * N * 2)
    assert query(False) - query(True) == dz
    assert query(True, lddy=0) == query(False, lddy=0) == query(False)  # a dy off 16 bytes is copied
    assert query(True, torch.float32) == query(False, torch.float32)  # and an fp32 one split
    assert query(True, ldx=K + 8, ldw=K + 16, lddy=N + 8) == query(True)


@pytest.mark.parametrize("act,p,code", [(0, 0.0, 0), (0, 1e-7, 0), (0, 0.5, 3), (1, 0.0, 3)])
def test_what_a_call_needs(mpc, act, p, code):
    """The C call asks for the room that it uses: without activation and dropped entries a workspace of the smaller size
    passes the check of its size (and stops at the next one, of its alignment)."""
    M, K, N = 300, 64, 512
    size = mpc.mpc_linear_workspace_bytes(M, K, N, torch.bfloat16, backward=True, plain=True)

    def call(ws, size):
        return mpc.lib().mpc_linear_backward(P, N, P, K, P, K, P, N, M, K, N, 1, act, p, 0, None, P, K, P, K, None, ws, size, None)

    assert call(P + 8, size) == (1 if code == 0 else code)
    assert call(P, size - 1) == 3
