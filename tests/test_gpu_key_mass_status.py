"""Key weights that are queued behind a kernel which gave up a wait: they write nothing, whatever their workspace held."""
import pytest
import torch

import paper_2603_15619_b200 as moda

from test_wait_reporting import kernels, source


def test_the_directory_of_pieces_is_written_before_anything_can_return():
    bodies = dict(kernels(source("moda_keymass.cuh")))
    sums, join = bodies["key_mass_kernel"], bodies["key_mass_join_kernel"]
    assert sums.index("kPieceNone") < sums.index("return")
    assert join.index("grid_dependency_wait()") < join.index("if (g_moda_status != 0) return;") < join.index("dir[")


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_nothing_is_written_behind_a_wait_that_ran_out(d):
    B, T_q, T, H, Hk = 1, 1100, 3100, 8, 2
    g = torch.Generator(device="cuda").manual_seed(1)
    n = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)
    Q, K, LSE = n(B, T_q, H, d), n(B, T, Hk, d), torch.full((B, H, T_q), 8.0, device="cuda")
    # what an earlier call of another shape may have left: every entry of the directory names a tile (that there is) that starts here
    work = torch.ones((moda.moda_key_mass_workspace_bytes(B, T_q, T, H, Hk, d) // 4,), dtype=torch.int32, device="cuda")
    mass = torch.zeros((B, Hk, T), device="cuda")
    want = moda.moda_attn_key_mass(Q, K, LSE, d ** -0.5, workspace=work.clone())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):                                             # queued without the host's look at the status
        moda.moda_attn_key_mass(Q, K, LSE, d ** -0.5, mass=mass, workspace=work)
    mass.fill_(7.0)
    assert moda.moda_last_status() == 0
    try:
        moda.moda_selftest_wait_timeout()                                     # returns by itself, after 1 ms
        graph.replay()
        torch.cuda.synchronize()
        assert moda.moda_last_status() != 0 and bool((mass == 7.0).all())
    finally:
        moda.moda_last_status(clear=True)
    work.fill_(1)
    graph.replay()
    torch.cuda.synchronize()
    assert moda.moda_last_status() == 0 and torch.equal(mass, want)
