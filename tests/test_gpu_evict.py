"""Eviction from a sequence cache by accumulated weight on the GPU: positions, rows and weights are exact."""
import numpy as np
import pytest
import torch

import paper_2603_15619_b200 as moda
from oracle import moda_oracle as orc

pytestmark = pytest.mark.gpu


def inputs(B, T_cap, Hk, d, seed, weights="lognormal"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    K, V = (torch.randn((B, T_cap, Hk, d), generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    m = torch.randn((B, Hk, T_cap), generator=g, device="cuda")
    mass = {"lognormal": lambda: (2 * m).exp(), "ties": lambda: (m * 1.5).round(), "zeros": lambda: torch.zeros_like(m), "signed": lambda: m,
            "close": lambda: 1 + m * 1e-6, "tiny": lambda: m.abs() * 1e-42}[weights]()
    return K, V, mass


def check(K, V, mass, T, n_keep, n_recent, lens=None):
    B, _, Hk, _ = K.shape
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda") if lens is not None else None
    K_out, V_out, mass_out, index, lens_out = moda.moda_kv_evict(K, V, mass, T, n_keep, n_recent, seq_lens=seq)
    assert moda.moda_last_status() == 0
    m = mass.cpu().numpy()
    for b in range(B):
        n = T if lens is None else lens[b]
        assert int(lens_out[b]) == min(n_keep, n)
        for h in range(Hk):
            want = orc.kept_positions(m[b, h, :n], n_keep, n_recent)
            got = index[b, h].tolist()
            assert got[:len(want)] == want and all(i == -1 for i in got[len(want):]), (b, h)
            at = torch.tensor(want, device="cuda", dtype=torch.long)
            assert torch.equal(K_out[b, :len(want), h], K[b, at, h]) and torch.equal(V_out[b, :len(want), h], V[b, at, h])
            assert torch.equal(mass_out[b, h, :len(want)].view(torch.int32), mass[b, h, at].view(torch.int32))


SHAPES = [
    # B, T, T_cap, H_kv, d, n_keep, n_recent
    (1, 1, 1, 1, 64, 1, 0), (1, 1, 5, 2, 128, 3, 2), (2, 5, 5, 3, 64, 2, 1), (1, 33, 40, 1, 128, 32, 0), (1, 100, 100, 7, 64, 100, 7), (1, 100, 128, 2, 128, 50, 50),
    (3, 513, 513, 2, 64, 200, 30), (1, 1000, 1001, 16, 128, 1, 0), (1, 1000, 1001, 16, 128, 1, 1), (2, 2047, 2048, 4, 64, 2046, 5), (1, 4096, 4096, 2, 128, 1024, 100),
    (1, 4097, 4100, 2, 64, 1000, 0), (1, 9000, 9001, 3, 128, 3001, 77), (1, 20000, 20000, 1, 64, 5000, 17), (1, 40001, 40001, 2, 64, 39000, 0),
]


@pytest.mark.parametrize("B,T,T_cap,Hk,d,n_keep,n_recent", SHAPES)
def test_kept_rows(B, T, T_cap, Hk, d, n_keep, n_recent):
    K, V, mass = inputs(B, T_cap, Hk, d, seed=T)
    K[:, T:] = float("nan")
    mass[:, :, T:] = float("inf")                                            # past the length: never looked at
    check(K, V, mass, T, n_keep, n_recent)


@pytest.mark.parametrize("weights", ["ties", "zeros", "signed", "close", "tiny"])
@pytest.mark.parametrize("T,n_keep,n_recent", [(700, 300, 20), (9001, 4000, 0)])
def test_equal_negative_and_close_weights(weights, T, n_keep, n_recent):
    K, V, mass = inputs(2, T, 2, 64, seed=1, weights=weights)
    check(K, V, mass, T, n_keep, n_recent)


def test_weights_that_are_no_numbers():
    K, V, mass = inputs(1, 600, 2, 128, seed=2)
    mass[0, 0, ::3] = float("nan")
    mass[0, 0, 1::7] = float("inf")
    mass[0, 1, ::2] = -float("inf")
    mass[0, 1, 5::11] = -0.0
    mass[0, 1, 6::11] = 0.0
    for n_keep in (50, 300, 420, 599):
        check(K, V, mass, 600, n_keep, 10)
    mass.fill_(float("nan"))
    check(K, V, mass, 600, 100, 3)


@pytest.mark.parametrize("d", [64, 128])
def test_lengths_of_a_batch(d):
    lens = [0, 1, 2, 31, 100, 128, 129, 500]
    K, V, mass = inputs(len(lens), 512, 3, d, seed=7)
    for n_keep, n_recent in [(100, 10), (128, 128), (1, 0), (512, 4)]:
        check(K, V, mass, 500, n_keep, n_recent, lens)


def test_a_share_that_shared_memory_does_not_hold():
    # more keys than the shared memories of a cluster: the weights are read again from global memory
    T = 8 * 48 * 1024 + 4001
    g = torch.Generator(device="cuda").manual_seed(3)
    mass = torch.rand((1, 1, T), generator=g, device="cuda")
    K = torch.randn((1, T, 1, 64), generator=g, device="cuda", dtype=torch.bfloat16)
    K_out, V_out, mass_out, index, lens_out = moda.moda_kv_evict(K, K, mass, T, 1000, 100)
    want = torch.sort(torch.topk(mass[0, 0, :T - 100], 900).indices).values.int()
    assert torch.equal(index[0, 0, :900], want) and index[0, 0, 900:].tolist() == list(range(T - 100, T))
    assert torch.equal(K_out[0, :, 0], K[0, index[0, 0].long(), 0])


def test_outputs_of_the_callers_and_guard_bands():
    B, T, Hk, d, n_keep, T_out = 2, 300, 3, 128, 100, 160
    K, V, mass = inputs(B, T, Hk, d, seed=11)
    K_out, V_out = (torch.full((B, T_out, Hk, d), 7.0, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    mass_out = torch.full((B, Hk, T_out), 7.0, device="cuda")
    before = K.clone(), V.clone(), mass.clone()
    lens = torch.tensor([300, 40], dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    moda.moda_kv_evict(K, V, mass, T, n_keep, 5, seq_lens=lens, K_out=K_out, V_out=V_out, mass_out=mass_out, stream=s)
    s.synchronize()
    want = moda.moda_kv_evict(K, V, mass, T, n_keep, 5, seq_lens=lens)
    for b, n in enumerate((100, 40)):
        assert torch.equal(K_out[b, :n], want[0][b, :n]) and torch.equal(V_out[b, :n], want[1][b, :n]) and torch.equal(mass_out[b, :, :n], want[2][b, :, :n])
        assert bool((K_out[b, n:] == 7).all()) and bool((V_out[b, n:] == 7).all()) and bool((mass_out[b, :, n:] == 7).all())
    assert all(torch.equal(a, c) for a, c in zip(before, (K, V, mass)))      # the source is left as it was
    with pytest.raises(moda.ModaError, match=r"\[-3\]"):
        moda.moda_kv_evict(K, V, mass, T, n_keep, 5, K_out=K, V_out=torch.empty_like(K))
    with pytest.raises(moda.ModaError, match=r"\[-3\]"):
        moda.moda_kv_evict(K, V, mass, T, n_keep, 5, K_out=torch.empty_like(K), V_out=torch.empty_like(K), mass_out=mass)


@pytest.mark.parametrize("T,n_keep,n_recent,ragged", [(300, 100, 10, True), (4000, 1000, 0, False), (8100, 2000, 33, True), (13000, 4000, 100, False), (17003, 900, 5, True)])
def test_many_heads_at_once(T, n_keep, n_recent, ragged):
    # one CTA a head, with few to many keys a thread; against a stable sort of all heads
    B, Hk, d = 2, 80, 64
    K, V, mass = inputs(B, T, Hk, d, seed=T)
    mass = (mass * 8).round() / 8                                            # ties
    lens = [T // 3, T] if ragged else [T, T]
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    K_out, V_out, mass_out, index, lens_out = moda.moda_kv_evict(K, V, mass, T, n_keep, n_recent, seq_lens=seq)
    for b, n in enumerate(lens):
        kept = min(n_keep, n)
        recent = min(n_recent, kept)
        old = mass[b, :, :n - recent]
        order = torch.sort(old, dim=-1, descending=True, stable=True).indices[:, :kept - recent]
        want = torch.cat([torch.sort(order, dim=-1).values, torch.arange(n - recent, n, device="cuda").expand(Hk, -1)], -1)
        assert torch.equal(index[b, :, :kept].long(), want) and bool((index[b, :, kept:] == -1).all()) and int(lens_out[b]) == kept
        heads = torch.arange(Hk, device="cuda")[:, None].expand_as(want)
        assert torch.equal(K_out[b, :kept].transpose(0, 1), K[b, want, heads]) and torch.equal(V_out[b, :kept].transpose(0, 1), V[b, want, heads])
        assert torch.equal(mass_out[b, :, :kept], mass[b].gather(1, want))


@pytest.mark.parametrize("B,T,Hk,n_keep,n_recent", [
    (20, 12000, 8, 700, 50),        # more CTAs than SMs, two of them on one
    (5, 16001, 1, 300, 0),          # keys of a thread in registers, a CTA for each SM
    (19, 99001, 1, 100, 7),         # clusters of 4 with 1024 threads
    (1, 280000, 2, 64, 64),         # clusters of 16
])
def test_many_long_rows(B, T, Hk, n_keep, n_recent):
    K, V, mass = inputs(B, T, Hk, 64, seed=T)
    check(K, V, mass, T, n_keep, n_recent, lens=[T - (b * 997) % T for b in range(B)])
