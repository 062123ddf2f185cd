"""Kernels whose CTAs store into each other's shared memory, launched on several streams at once, so that
the CTAs of a cluster start among those of other kernels: results as one at a time."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mpc():
    import __graft_entry__ as g

    g.build()
    import paper_2401_07788_gb300 as m

    torch.cuda.set_device(0)
    return m


def bits(out):
    return [x.view(torch.int32) for x in out]


@pytest.mark.parametrize("rows", [3, 200, 1500])
def test_clusters_beside_other_kernels(mpc, rows):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    jobs = []
    for L in (8193, 30001, 65535, 65536):  # one to eight CTAs a row; rows on and off 16 bytes
        x = torch.randn(rows, L, device="cuda", generator=gen)
        for b in (2, 4, 8, 5):
            jobs.append(lambda x=x, b=b: mpc.mpc_quant_compress(x, b))
        for k in (L // 100, L // 2, L):
            jobs.append(lambda x=x, k=k: mpc.mpc_topk_compress(x, k))
        jobs.append(lambda x=x, L=L: mpc.mpc_ef_topk_compress(x, torch.full_like(x, 0.25), L // 10))
    want = [bits(job()) for job in jobs]
    torch.cuda.synchronize()
    assert mpc.mpc_get_status() == 0
    streams = [torch.cuda.Stream() for _ in range(6)]
    for turn in range(3):
        got = {}
        for i, job in enumerate(jobs):
            j = (i * 7 + turn) % len(jobs)
            with torch.cuda.stream(streams[i % len(streams)]):
                got[j] = bits(jobs[j]())
        torch.cuda.synchronize()
        assert len(got) == len(jobs) and mpc.mpc_get_status() == 0
        for j, out in got.items():
            for a, b in zip(out, want[j]):
                assert torch.equal(a, b), j
