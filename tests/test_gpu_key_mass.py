"""Attention weight of the sequence keys on the GPU: after a forward of many rows and in the decode step, against the fp64 oracle.

Tolerance of a weight: its exponent x = scale s log2(e) - LSE log2(e) is off by the roundings of s (fp32 accumulation of products
whose magnitudes sum to ~10 after scaling: 2^-22 of that), of the scaled LSE and of the sum (2^-24 of up to 32 each), together under 1e-5,
its exponential by 2^-22, and the sum over at most a few thousand rows in short chains by less than 1e-5: 1e-4 of the weight, and 1e-7
where weights vanish.  Scores that are g times larger have exponents off by g times more."""
import numpy as np
import pytest
import torch

import paper_2603_15619_b200 as moda
from paper_2603_15619_b200 import synthetic
from oracle import moda_oracle as orc

from parity import build_cache, f64

pytestmark = pytest.mark.gpu
RTOL, ATOL = 1e-4, 1e-7


def close(got, want, grow=1.0):
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    assert np.allclose(got[ok], want[ok], rtol=RTOL * grow, atol=ATOL), np.abs(got[ok] - want[ok]).max()


def inputs(B, T_q, T_kv, H, Hk, d, l, seed=0, grow=1.0, T_cap=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)
    Q, K, V = n(B, T_q, H, d) * grow, n(B, T_cap or T_kv, Hk, d), n(B, T_kv, Hk, d)
    Kd, Vd = n(l, B, T_q, Hk, d), n(l, B, T_q, Hk, d)
    _, LSE = moda.moda_attn_fwd_prefill(Q, K[:, :T_kv].contiguous(), V, build_cache(Kd, Vd) if l else None, l, d ** -0.5)
    return Q, K, LSE


SHAPES = [
    # B, T_q, T_kv, H, H_kv, d, l
    (1, 1, 1, 1, 1, 64, 0), (1, 1, 1, 2, 1, 128, 2), (2, 1, 129, 4, 2, 64, 1), (1, 2, 127, 3, 1, 128, 0), (1, 127, 127, 2, 2, 128, 3),
    (1, 128, 128, 8, 1, 64, 0), (2, 129, 129, 5, 1, 128, 1), (1, 257, 300, 6, 2, 64, 4), (1, 16, 16, 16, 1, 128, 0), (1, 40, 200, 32, 1, 64, 2),
    (1, 64, 1000, 8, 2, 128, 1), (3, 100, 513, 7, 7, 64, 0), (1, 600, 600, 12, 4, 128, 5), (1, 700, 1300, 3, 3, 64, 0), (2, 385, 385, 24, 8, 64, 1),
]


@pytest.mark.parametrize("B,T_q,T_kv,H,Hk,d,l", SHAPES)
def test_key_mass_matches_the_oracle(B, T_q, T_kv, H, Hk, d, l):
    Q, K, LSE = inputs(B, T_q, T_kv, H, Hk, d, l, seed=T_kv)
    mass = moda.moda_attn_key_mass(Q, K, LSE, d ** -0.5)
    again = moda.moda_attn_key_mass(Q, K, LSE, d ** -0.5)
    assert moda.moda_last_status() == 0
    close(f64(mass), orc.key_mass(f64(Q), f64(K), f64(LSE), d ** -0.5))
    assert torch.equal(mass, again)                                          # sums in a fixed order


def test_key_mass_of_a_long_prompt_adds_up():
    # every row's probabilities add up to 1: with no depth slots the weights of a head add up to rows times heads of the group
    B, T, H, Hk, d = 1, 9000, 8, 2, 128
    Q, K, LSE = inputs(B, T, T, H, Hk, d, 0, seed=8)
    mass = moda.moda_attn_key_mass(Q, K, LSE, d ** -0.5)
    assert np.allclose(f64(mass).sum(-1), T * H / Hk, rtol=1e-5)
    # the last rows of the last tile against the definition: only few rows see them
    tail = f64(Q)[:, -40:], f64(K), f64(LSE)[:, :, -40:]
    close(f64(mass)[:, :, -40:], orc.key_mass(*tail, d ** -0.5)[:, :, -40:])


LARGE = [
    # B, T_q, T_kv, H, H_kv, d: one to four units a tile and many of them, runs that share tiles and runs of whole tiles, several (b, head)
    (4, 64, 3000, 16, 4, 128), (3, 33, 2500, 24, 8, 128), (2, 1, 7000, 8, 8, 64), (2, 300, 4001, 14, 7, 64), (2, 500, 2049, 5, 5, 64), (3, 257, 1500, 6, 2, 128),
    (1, 1100, 3100, 32, 2, 64), (2, 1600, 1600, 6, 3, 128), (1, 3000, 3300, 5, 1, 128), (5, 129, 769, 4, 4, 128),
]


@pytest.mark.parametrize("B,T_q,T_kv,H,Hk,d", LARGE)
def test_key_mass_of_many_tiles(B, T_q, T_kv, H, Hk, d):
    Q, K, LSE = inputs(B, T_q, T_kv, H, Hk, d, 0, seed=T_q)
    mass = moda.moda_attn_key_mass(Q, K, LSE, d ** -0.5)
    assert moda.moda_last_status() == 0
    want = torch.zeros((B, Hk, T_kv), device="cuda", dtype=torch.float64)
    seen = torch.arange(T_kv, device="cuda") <= torch.arange(T_q, device="cuda")[:, None] + T_kv - T_q
    for h in range(H):
        s = torch.einsum("bid,bjd->bij", Q[:, :, h].double(), K[:, :, h // (H // Hk)].double()) * d ** -0.5
        want[:, h // (H // Hk)] += torch.where(seen, (s - LSE[:, h, :, None].double()).exp(), 0.0).sum(1)
    close(f64(mass), f64(want))


def test_key_mass_accumulates_over_the_chunks_of_a_prompt():
    B, T, H, Hk, d = 2, 500, 6, 3, 64
    Q, K, LSE = inputs(B, T, T, H, Hk, d, 0, seed=3, T_cap=512)
    whole = moda.moda_attn_key_mass(Q, K, LSE, d ** -0.5, T_kv=T)
    mass = torch.full((B, Hk, 512), 7.0, device="cuda")
    for at, end in [(0, 200), (200, 201), (201, 500)]:
        moda.moda_attn_key_mass(Q[:, at:end].contiguous(), K, LSE[:, :, at:end].contiguous(), d ** -0.5, T_kv=end, mass_in=mass, mass=mass)
    assert np.allclose(f64(mass)[:, :, :T], f64(whole)[:, :, :T], rtol=1e-5)
    assert bool((mass[:, :, T:] == 7.0).all())                               # positions that no key has are not touched


def test_key_mass_of_large_scores_and_of_rows_without_keys():
    B, T, H, Hk, d = 1, 260, 4, 2, 128
    Q, K, LSE = inputs(B, T, T, H, Hk, d, 0, seed=5, grow=8.0)
    close(f64(moda.moda_attn_key_mass(Q, K, LSE, d ** -0.5)), orc.key_mass(f64(Q), f64(K), f64(LSE), d ** -0.5), grow=8)
    LSE[0, 1, 17] = -float("inf")
    LSE[0, 2, 100:] = -float("inf")
    close(f64(moda.moda_attn_key_mass(Q, K, LSE, d ** -0.5)), orc.key_mass(f64(Q), f64(K), f64(LSE), d ** -0.5), grow=8)
    LSE.fill_(-float("inf"))
    assert bool((moda.moda_attn_key_mass(Q, K, LSE, d ** -0.5) == 0).all())


@pytest.mark.parametrize("d", [64, 128])
def test_what_a_key_does_not_see_does_not_reach_it(d):
    # NaN in cache rows past T_kv, in one key, and in the first query row reach only their own keys
    B, T_q, T, H, Hk = 1, 130, 300, 4, 2
    Q, K, LSE = inputs(B, T_q, T, H, Hk, d, 0, seed=9, T_cap=400)
    clean = moda.moda_attn_key_mass(Q, K, LSE, d ** -0.5, T_kv=T).clone()
    K[:, T:] = float("nan")
    K[:, 40, 1] = float("inf")
    Q[:, 0, 0] = float("nan")                                                # sees keys 0 .. 170 of head 0
    mass = moda.moda_attn_key_mass(Q, K, LSE, d ** -0.5, T_kv=T)
    assert torch.isnan(mass[0, 0, :171]).all() and torch.equal(mass[0, 0, 171:T], clean[0, 0, 171:T])
    others = [j for j in range(T) if j != 40]
    assert torch.equal(mass[0, 1, others], clean[0, 1, others]) and not torch.isfinite(mass[0, 1, 40])


def test_key_mass_on_another_stream_and_guard_bands():
    B, T_q, T, H, Hk, d = 2, 90, 333, 6, 2, 128
    Q, K, LSE = inputs(B, T_q, T, H, Hk, d, 0, seed=4)
    want = moda.moda_attn_key_mass(Q, K, LSE, d ** -0.5)
    buf = torch.full((B * Hk * T + 128,), 7.0, device="cuda")
    out = buf[64:64 + B * Hk * T].view(B, Hk, T)
    work = torch.full((moda.moda_key_mass_workspace_bytes(B, T_q, T, H, Hk, d) + 64,), 7, dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    moda.moda_attn_key_mass(Q, K, LSE, d ** -0.5, mass=out, workspace=work[:-64], stream=s)
    s.synchronize()
    assert torch.equal(out, want)
    assert bool((buf[:64] == 7.0).all()) and bool((buf[-64:] == 7.0).all()) and bool((work[-64:] == 7).all())


# ---------------------------------------------------------------------------------------------------------- decode step
DECODE = [
    # B, T_kv, T_cap, H, H_kv, d, l
    (1, 1, 1, 1, 1, 64, 0), (1, 1, 8, 2, 1, 128, 3), (2, 31, 31, 4, 2, 64, 2), (1, 255, 300, 2, 2, 128, 5), (2, 64, 64, 8, 1, 128, 1),
    (1, 257, 512, 6, 2, 128, 1), (3, 1000, 1024, 20, 4, 64, 7), (1, 1030, 1030, 32, 2, 128, 3), (1, 900, 1001, 32, 1, 64, 5), (16, 700, 700, 7, 7, 128, 0),
    (1, 5001, 5001, 8, 2, 128, 24),
]


@pytest.mark.parametrize("B,T_kv,T_cap,H,Hk,d,l", DECODE)
@pytest.mark.parametrize("ragged", [False, True])
def test_decode_mass_matches_the_oracle(B, T_kv, T_cap, H, Hk, d, l, ragged):
    x = synthetic.make_decode(B, T_kv, H, Hk, d, l, seed=13, device="cuda", T_cap=T_cap)
    x["K"][:, T_kv:] = float("nan")
    x["V"][:, T_kv:] = float("nan")
    scale, depth = d ** -0.5, x["depth"] if l else None
    lens = [max(1, T_kv * (b + 1) // B - b % 3) if ragged else T_kv for b in range(B)]
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda") if ragged else None
    old = torch.rand((B, Hk, T_cap), device="cuda")
    mass = torch.full((B, Hk, T_cap), 7.0, device="cuda")
    O, LSE, out = moda.moda_attn_decode_mass(x["q"], x["K"], x["V"], depth, T_kv, l, scale, seq_lens=seq, mass_in=old, mass=mass)
    assert moda.moda_last_status() == 0 and out is mass
    plain = (moda.moda_attn_decode_varlen(x["q"], x["K"], x["V"], seq, depth, T_kv, l, scale) if ragged
             else moda.moda_attn_decode(x["q"], x["K"], x["V"], depth, T_kv, l, scale))
    assert torch.equal(O, plain[0]) and torch.equal(LSE, plain[1])
    for b in range(B):
        n = lens[b]
        kd, vd = (f64(x["depth"][:, b:b + 1, :, i]) if l else None for i in (0, 1))
        q, K = f64(x["q"][b:b + 1]), f64(x["K"][b:b + 1, :n])
        _, lse = orc.decode_gqa(q, K, f64(x["V"][b:b + 1, :n]), kd, vd, scale)
        want = orc.key_mass(q[:, None], K, lse[:, :, None], scale)[0]
        want[:, :n - 1] += f64(old[b, :, :n - 1])
        close(f64(mass[b, :, :n]), want)
        assert bool((mass[b, :, n:] == 7.0).all())
    # in place, and without an accumulator
    moda.moda_attn_decode_mass(x["q"], x["K"], x["V"], depth, T_kv, l, scale, seq_lens=seq, mass_in=old, mass=old)
    for b in range(B):
        assert torch.equal(old[b, :, :lens[b]], mass[b, :, :lens[b]])
    _, _, alone = moda.moda_attn_decode_mass(x["q"], x["K"], x["V"], depth, T_kv, l, scale, seq_lens=seq)
    total = sum(float(alone[b, :, :lens[b]].sum()) for b in range(B))
    assert total <= B * H * (1 + 1e-4) and (l > 0 or total >= B * H * (1 - 1e-4))


def test_decode_mass_in_a_graph_accumulates_every_replay():
    B, T, H, Hk, d, l = 2, 500, 8, 2, 128, 3
    x = synthetic.make_decode(B, T, H, Hk, d, l, seed=2, device="cuda")
    _, _, one = moda.moda_attn_decode_mass(x["q"], x["K"], x["V"], x["depth"], T, l, d ** -0.5)
    mass = torch.zeros((B, Hk, T), device="cuda")
    work = torch.empty((moda.moda_decode_mass_workspace_bytes(B, T, H, Hk, d),), dtype=torch.uint8, device="cuda")
    O, LSE = torch.empty_like(x["q"]), torch.empty((B, H), device="cuda")
    call = lambda: moda.moda_attn_decode_mass(x["q"], x["K"], x["V"], x["depth"], T, l, d ** -0.5, mass_in=mass, mass=mass, O=O, LSE=LSE, workspace=work)
    call()
    torch.cuda.synchronize()
    mass.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for _ in range(4):
        g.replay()
    torch.cuda.synchronize()
    assert np.allclose(f64(mass)[:, :, :-1], 4 * f64(one)[:, :, :-1], rtol=1e-6)
    assert torch.equal(mass[:, :, -1], one[:, :, -1])                        # the newest key starts from 0 every time
