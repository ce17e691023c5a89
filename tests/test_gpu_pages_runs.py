"""Decode over pages in 8 bits and selection where there are more blocks than warps: every warp works through several, over the ends of groups and over empty sequences; the
forms that only large batches take; many depth pairs."""
import numpy as np
import pytest
import torch

import paper_2603_15619_b200 as moda
from oracle import moda_oracle as orc

import pages_ref as ref

pytestmark = pytest.mark.gpu


def _pool(num, sub, Hk, d, seed):
    """Full pages that sequences share (a step only reads them), value rows of sizes from 2^-6 to 2^6."""
    rng = np.random.default_rng(seed)
    pages = np.zeros((num, sub, Hk, 128 * d + 512), np.uint8)
    kc, vc, ks, vs = ref.split(pages, d)
    lead = (num, sub, Hk, 64)
    codes, scale = orc.quantize_e4m3_rows(ref.bf16(rng.standard_normal((*lead, d))))
    kc[...], ks[...] = codes, scale
    codes, scale = orc.quantize_e4m3_rows(ref.bf16(rng.standard_normal((*lead, d)) * 2.0 ** rng.integers(-6, 7, (*lead, 1))))
    vc[...], vs[...] = codes.swapaxes(-1, -2), scale
    return pages


def _case(lens, H, Hk, d, page, l, keep=None, seed=0, sharp=1.0, check=None):
    B, rng = len(lens), np.random.default_rng(seed)
    pages = _pool(40, page // 64, Hk, d, seed)
    most = max(-(-max(lens) // page), 1)
    table = rng.integers(0, 40, (B, most)).astype(np.int32)
    q = ref.bf16(rng.standard_normal((B, H, d)) * sharp)
    depth = ref.bf16(rng.standard_normal((l, B, Hk, 2, d)))
    index = None
    if keep is not None:
        index = np.full((B, Hk, keep), -1, np.int32)
        for b, n in enumerate(lens):
            for k in range(Hk):
                at = np.sort(rng.permutation(-(-n // 64))[:keep])
                index[b, k, :len(at)] = at
    put = lambda x: torch.from_numpy(x).cuda()
    O, LSE = moda.moda_attn_decode_e4m3(ref.put(q), put(pages), put(table), torch.tensor(lens, dtype=torch.int32, device="cuda"), ref.put(depth) if l else None, max(lens), l,
                                        d ** -0.5, index=None if index is None else put(index))
    assert moda.moda_last_status() == 0
    some = np.arange(B) if check is None else rng.permutation(B)[:check]
    o, lse, o_tol, lse_tol = ref.decode(q[some], pages, table[some], [lens[b] for b in some], depth[:, some], d ** -0.5, page, None if index is None else index[some])
    O, LSE = O.double().cpu().numpy()[some], LSE.double().cpu().numpy()[some]
    empty = np.isneginf(lse)
    assert np.array_equal(np.isneginf(LSE), empty) and (O[empty] == 0).all()
    assert (np.abs(O - o) <= o_tol).all(), float((np.abs(O - o) / np.maximum(o_tol, 1e-30)).max())
    assert (np.abs(LSE[~empty] - lse[~empty]) <= lse_tol[~empty]).all()


def _lens(B, low, high, empty, seed):
    rng = np.random.default_rng(seed)
    n = np.exp(rng.uniform(np.log(low), np.log(high), B)).astype(int)
    n[::empty] = 0
    n[1], n[-1] = high, 64 * (high // 64)
    return [int(x) for x in n]


RUNS = [  # sequences, shortest, longest, every how many is empty; H, Hk, d, page, l
    (40, 40, 3000, 7, 8, 4, 64, 64, 0), (40, 40, 3000, 7, 8, 4, 128, 128, 3),          # 1 to 3 units a warp
    (24, 2000, 5000, 5, 24, 8, 64, 64, 5), (24, 2000, 5000, 5, 16, 8, 128, 64, 0),     # 5 to 10
    (3, 20000, 40000, 9, 4, 4, 128, 256, 2), (3, 20000, 40000, 9, 4, 4, 64, 128, 33),  # few long ones
    (20, 500, 6000, 6, 32, 2, 128, 64, 4), (20, 500, 6000, 6, 64, 2, 64, 64, 0), (12, 900, 5000, 6, 64, 2, 128, 128, 1), (16, 500, 4000, 5, 32, 2, 64, 64, 0),   # groups of 16, 32
    (500, 1, 900, 3, 3, 1, 64, 64, 1),                                                   # more groups than a warp's units, empty ones between
]


@pytest.mark.parametrize("sharp", [1.0, 20.0])
@pytest.mark.parametrize("B,low,high,empty,H,Hk,d,page,l", RUNS)
def test_runs_of_several_blocks(B, low, high, empty, H, Hk, d, page, l, sharp):
    _case(_lens(B, low, high, empty, B + d), H, Hk, d, page, l, seed=d + H, sharp=sharp, check=10)


@pytest.mark.parametrize("B,low,high,H,Hk,d,keep", [(40, 300, 6000, 8, 4, 64, 20), (40, 300, 6000, 16, 8, 128, 33), (30, 40, 9000, 64, 2, 128, 50), (30, 40, 9000, 32, 2, 64, 50)])
def test_runs_of_several_named_blocks(B, low, high, H, Hk, d, keep):
    _case(_lens(B, low, high, 6, B + d), H, Hk, d, 64, 2, keep=keep, seed=keep, check=10)


@pytest.mark.parametrize("B,H,Hk,d,l", [(300, 8, 2, 128, 2), (150, 8, 8, 128, 0), (700, 2, 2, 64, 3), (2048, 1, 1, 64, 1), (1500, 2, 1, 128, 0)])
def test_merge_of_many_rows(B, H, Hk, d, l):
    _case(_lens(B, 1, 700, 11, B), H, Hk, d, 64, l, seed=B, check=25)


@pytest.mark.parametrize("l", [31, 32, 64, 65, 200, 256])
@pytest.mark.parametrize("H,Hk,d", [(8, 1, 128), (6, 2, 64)])
def test_many_depth_pairs(H, Hk, d, l):
    _case([0, 200, 65], H, Hk, d, 64, l, seed=l)


def test_runs_give_the_same_bits_and_replay():
    # the largest number of units a warp has here, captured: the second replay over other lengths
    H, Hk, d, page = 16, 4, 128, 64
    lens = [_lens(24, 500, 5000, 5, s) for s in range(2)]
    pages = torch.from_numpy(_pool(40, 1, Hk, d, 3)).cuda()
    table = torch.randint(0, 40, (24, 80), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    q = torch.randn((24, H, d), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()
    n = torch.tensor(lens[0], dtype=torch.int32, device="cuda")
    step = lambda: moda.moda_attn_decode_e4m3(q, pages, table, n, None, 5000, 0, 0.09)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for x in (lens[1], lens[0]):
        n.copy_(torch.tensor(x, dtype=torch.int32))
        graph.replay()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, step()))
    assert moda.moda_last_status() == 0


@pytest.mark.parametrize("few", [False, True])
@pytest.mark.parametrize("B,blocks,H,Hk,d,keep,recent", [(16, 2500, 16, 8, 128, 40, 2), (60, 2500, 6, 3, 64, 9, 0), (40, 4000, 10, 10, 128, 128, 3), (1, 3000, 2, 1, 128, 31, 1),
                                                         (2, 2048, 8, 4, 128, 64, 64)])
def test_selection_over_several_rounds(B, blocks, H, Hk, d, keep, recent, few):
    # two kernels, whose warps take several rounds; and one whose clusters do
    rng = np.random.default_rng(blocks + B)
    num, top = 3000, 2 if few else 127
    bounds = np.zeros((num, 1, Hk, 2 * d + 16), np.uint8)
    hi = rng.integers(-top, top + 1, (num, 1, Hk, d)).astype(np.int8)
    bounds[..., :d] = hi.view(np.uint8)
    bounds[..., d:2 * d] = np.minimum(hi, rng.integers(-top, top + 1, hi.shape).astype(np.int8)).view(np.uint8)
    bounds[..., 2 * d:2 * d + 4] = (np.ones(hi.shape[:3], np.float32) if few else np.exp(rng.standard_normal(hi.shape[:3]) * 0.3).astype(np.float32))[..., None].view(np.uint8)
    table = rng.integers(0, num, (B, blocks)).astype(np.int32)
    lens = [max(64 * blocks - 611 * b, 1) for b in range(B)]
    q = ref.bf16(rng.integers(-1, 2, (B, H, d)) if few else rng.standard_normal((B, H, d)))
    index = moda.moda_kv_select_blocks(ref.put(q), torch.from_numpy(bounds).cuda(), torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"),
                                       64 * blocks, keep, recent)
    assert moda.moda_last_status() == 0
    some = sorted({0, B // 2, B - 1})
    assert np.array_equal(index.cpu().numpy()[some], ref.select(q[some], bounds, table[some], [lens[b] for b in some], 64, keep, recent))
