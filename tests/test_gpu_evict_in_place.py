"""A cut whose new lengths take the place of the old ones: every head of a sequence is cut by the old length, whenever its turn comes."""
import ctypes

import pytest
import torch

import paper_2603_15619_b200 as moda
from paper_2603_15619_b200 import binding

from test_wait_reporting import kernels, source


def test_the_lengths_are_written_behind_the_selection():
    # a selection CTA may start after another of its sequence has ended: none of them writes what all of them read
    text = source("moda_evict.cuh")
    bodies = dict(kernels(text))
    assert "lens_out" not in bodies["evict_select_kernel"]
    gather = bodies["evict_gather_kernel"]
    assert gather.count("p.lens_out[") == 1 and gather.index("grid_dependency_wait()") < gather.index("p.lens_out[")


def test_lengths_that_overlap_in_part_are_refused():
    lib = binding.load()
    P, FAR, at = ctypes.c_void_p(4096), ctypes.c_void_p(1 << 40), 1 << 20
    for B, off in [(2, 4), (2, -4), (7, 24), (7, -24)]:
        assert lib.moda_kv_evict(P, P, P, ctypes.c_void_p(at), B, 100, 128, 2, 64, 50, 10, 64, FAR, FAR, None, FAR, ctypes.c_void_p(at + off), None) == -3


CASES = [
    # B, T, H_kv, d, n_keep, n_recent: several times the CTAs that fit at once, with heads of one sequence in different turns; clusters; two CTAs an SM
    (64, 700, 7, 64, 300, 20), (64, 2100, 16, 64, 400, 0), (30, 5000, 16, 64, 1000, 100), (40, 9000, 9, 64, 500, 7), (7, 36000, 4, 64, 900, 30), (300, 40, 3, 128, 11, 2),
]


@pytest.mark.gpu
@pytest.mark.parametrize("B,T,Hk,d,n_keep,n_recent", CASES)
def test_in_place_is_as_out_of_place(B, T, Hk, d, n_keep, n_recent):
    g = torch.Generator(device="cuda").manual_seed(B)
    K, V = (torch.randn((B, T, Hk, d), generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    mass = torch.randn((B, Hk, T), generator=g, device="cuda").mul_(2).exp_()
    lens = torch.tensor([T - (b * 37) % T for b in range(B)], dtype=torch.int32, device="cuda")
    want = moda.moda_kv_evict(K, V, mass, T, n_keep, n_recent, seq_lens=lens)
    kept = lens.clamp(max=n_keep)
    assert torch.equal(want[4], kept)
    # the positions by a stable sort: what the out-of-place call is held against elsewhere, here for every head
    at = torch.arange(T, device="cuda").expand(B, Hk, T)
    n, recent = lens.long()[:, None, None], kept.clamp(max=n_recent).long()[:, None, None]
    rank = mass.masked_fill(at >= n - recent, torch.inf).masked_fill(at >= n, -torch.inf)
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :n_keep]
    order = torch.sort(order.masked_fill(torch.arange(n_keep, device="cuda") >= kept[:, None, None], T), dim=-1).values
    assert torch.equal(want[3].long(), torch.where(order < T, order, -1)[..., :n_keep])
    for _ in range(10):
        now = lens.clone()
        got = moda.moda_kv_evict(K, V, mass, T, n_keep, n_recent, seq_lens=now, lens_out=now)
        assert got[4] is now and torch.equal(now, kept) and torch.equal(got[3], want[3])
        for b in (0, B // 2, B - 1):
            k = int(kept[b])
            assert torch.equal(got[0][b, :k], want[0][b, :k]) and torch.equal(got[1][b, :k], want[1][b, :k]) and torch.equal(got[2][b, :, :k], want[2][b, :, :k])
    assert moda.moda_last_status() == 0
