"""The paged sequence cache in 8 bits on the GPU: written, read back, blocks selected, decode steps over all of it and over the selected blocks."""
import numpy as np
import pytest
import torch

import paper_2603_15619_b200 as moda
from paper_2603_15619_b200 import synthetic

import pages_ref as ref

pytestmark = pytest.mark.gpu

WRITES = [  # B, T, Hk, d, page, starts, n_new
    (1, 1, 1, 64, 64, [0], [1]),
    (3, 1, 2, 128, 64, [63, 64, 200], [1, 1, 1]),
    (2, 130, 3, 64, 128, [5, 61], [130, 77]),
    (2, 130, 3, 128, 64, [0, 64], [130, 128]),
    (4, 100, 1, 128, 256, [17, 0, 300, 48], [0, 100, 1, 16]),
    (1, 515, 5, 64, 64, [31], [515]),
]


@pytest.mark.parametrize("B,T,Hk,d,page,start,n_new", WRITES)
def test_write_gives_the_bytes_of_the_definition(B, T, Hk, d, page, start, n_new):
    rng = np.random.default_rng(T)
    lens = [s for s in start]
    most = max(s + n for s, n in zip(start, n_new))
    pages, bounds, table, _ = ref.make(B, most, Hk, d, page, [max(s + n, 1) for s, n in zip(start, n_new)], seed=T + d)
    K, V = (ref.bf16(rng.standard_normal((B, T, Hk, d)) * np.exp(rng.standard_normal((B, T, Hk, 1)) * 3)) for _ in range(2))
    K[0, 0, 0] = 0.0                                            # a row of zeros
    V[-1, -1, -1, 1:] = 0.0
    want = ref.write(pages, bounds, K, V, table, start, n_new, page)
    dev = [torch.from_numpy(x.copy()).cuda() for x in (pages, bounds, table)]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    moda.moda_kv_write_e4m3(dev[0], ref.put(K), ref.put(V), dev[2], start=i32(start), n_new=i32(n_new), bounds=dev[1])
    assert moda.moda_last_status() == 0
    assert np.array_equal(dev[0].cpu().numpy(), want[0])
    got, w = dev[1].cpu().numpy(), want[1]
    assert np.array_equal(got[..., :2 * d + 4], w[..., :2 * d + 4])
    # without bounds: the same pages
    again = torch.from_numpy(pages.copy()).cuda()
    moda.moda_kv_write_e4m3(again, ref.put(K), ref.put(V), dev[2], start=i32(start), n_new=i32(n_new))
    assert torch.equal(again, dev[0])


@pytest.mark.parametrize("d", [64, 128])
def test_rows_of_every_size_have_the_depth_caches_codes(d):
    # from bf16's smallest numbers to its largest, rows of one element, quotients that are ties: the oracle's codes and scales, and the bytes of the depth cache
    rng = np.random.default_rng(d)
    T = 261
    X = rng.standard_normal((1, T, 1, d)) * 2.0 ** (np.linspace(-138, 125, T)[None, :, None, None])
    X[0, ::7, 0, 1:] = 0.0
    X[0, 1::7] = rng.integers(-255, 256, X[0, 1::7].shape) * 2.0 ** rng.integers(-20, 20, X[0, 1::7].shape[:2] + (1,))
    X = ref.bf16(np.clip(X, -3e38, 3e38))
    dev = moda.alloc_kv_pages_e4m3(5, 64, 1, d)
    table = torch.arange(5, dtype=torch.int32, device="cuda")[None].contiguous()
    moda.moda_kv_write_e4m3(dev, ref.put(X), ref.put(-X), table)
    codes, scale = ref.orc.quantize_e4m3_rows(X[0, :, 0])
    negated, _ = ref.orc.quantize_e4m3_rows(-X[0, :, 0])
    kc, vc, ks, vs = ref.split(dev.cpu().numpy()[:, 0, 0], d)
    rows = lambda a: a.reshape(-1, *a.shape[2:])[:T]
    assert np.array_equal(rows(ks), scale) and np.array_equal(rows(vs), scale)
    assert np.array_equal(rows(kc), codes) and np.array_equal(rows(vc.swapaxes(-1, -2)), negated)
    cache = moda.alloc_depth_cache_e4m3(1, T, 1, d, 1)
    moda.moda_depth_cache_append_e4m3(cache, 0, ref.put(X), ref.put(-X))
    block = cache.cpu().numpy()[:3 * 2 * (128 * d + 512)].reshape(3, 2, -1)[:, 0]
    assert np.array_equal(block[:, :128 * d].reshape(3, d // 16, 128, 16).swapaxes(1, 2).reshape(-1, d)[:T], codes)


@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_are_not_finite(d):
    pages, bounds, table, dev = ref.make(1, 100, 2, d, 64, [100], seed=3)
    K, V = (ref.bf16(np.random.default_rng(i).standard_normal((1, 3, 2, d))) for i in range(2))
    K[0, 1, 0, 5], K[0, 2, 1, 7], V[0, 0, 0, 3] = np.nan, np.inf, -np.inf
    moda.moda_kv_write_e4m3(dev[0], ref.put(K), ref.put(V), dev[2], start=torch.tensor([100], dtype=torch.int32, device="cuda"), bounds=dev[1])
    b = dev[1].cpu().numpy().reshape(-1, 2, 2 * d + 16)[table[0, 1]]
    for h in range(2):
        assert not b[h, :2 * d].any() and np.isinf(b[h, 2 * d:2 * d + 4].copy().view(np.float32)[0])
    K2, _ = moda.moda_kv_read_e4m3(dev[0], dev[2], torch.tensor([103], dtype=torch.int32, device="cuda"), 103)
    K2 = K2.float().cpu().numpy()
    assert np.isnan(K2[0, 101, 0, 5]) and np.isfinite(np.delete(K2[0, 101, 0], 5)).all() and np.isnan(K2[0, 102, 1]).all() and np.isfinite(K2[0, 100]).all()


@pytest.mark.parametrize("B,T,Hk,d,page,lens,start", [(1, 1, 1, 64, 64, [1], None), (3, 200, 2, 128, 128, [0, 200, 77], None), (2, 70, 3, 64, 64, [150, 90], [90, 33]),
                                                      (2, 129, 1, 128, 256, [300, 60], [255, 0])])
def test_read_gives_the_rounded_products(B, T, Hk, d, page, lens, start):
    pages, _, table, dev = ref.make(B, max(lens), Hk, d, page, lens, seed=T)
    i32 = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")
    K, V = (torch.full((B, T, Hk, d), 7.0, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    out = moda.moda_kv_read_e4m3(dev[0], dev[2], i32(lens), T, start=i32(start), K_out=K, V_out=V)
    assert out[0] is K and out[1] is V and moda.moda_last_status() == 0
    for b in range(B):
        s = start[b] if start else 0
        n = min(max(lens[b] - s, 0), T)
        for k in range(Hk):
            for got, want in zip((K, V), ref.gather(pages, table, b, k, lens[b], page, d)):
                assert np.array_equal(got[b, :n, k].float().cpu().numpy(), ref.bf16(want[s:s + n].astype(np.float32)))
        assert (K[b, n:] == 7).all() and (V[b, n:] == 7).all()
    # the outputs that are made here: zeros behind
    K2, V2 = moda.moda_kv_read_e4m3(dev[0], dev[2], i32(lens), T, start=i32(start))
    assert torch.equal(K2, torch.where(K == 7, 0, K)) or (K == 7).float().mean() > 0


SELECTS = [  # B, lens, H, Hk, d, page, keep, recent
    (1, [64 * 40], 2, 2, 128, 64, 8, 1), (3, [0, 64 * 33 + 5, 64 * 9], 12, 3, 64, 128, 9, 2), (2, [64 * 300, 64 * 290 + 1], 8, 1, 128, 64, 40, 0),
    (1, [64 * 700 + 3], 32, 1, 64, 64, 100, 4), (2, [1, 64 * 70], 16, 1, 128, 256, 70, 70), (1, [64 * 1100], 5, 1, 64, 64, 1, 0),
]


def _bounds(num, sub, Hk, d, seed, few):
    """Bounds with many equal ratings (`few`) or of all kinds."""
    rng = np.random.default_rng(seed)
    out = np.zeros((num, sub, Hk, 2 * d + 16), np.uint8)
    top = 3 if few else 127
    out[..., :d] = rng.integers(-top, top + 1, out[..., :d].shape).astype(np.int8).view(np.uint8)
    out[..., d:2 * d] = np.minimum(out[..., :d].view(np.int8), rng.integers(-top, top + 1, out[..., :d].shape).astype(np.int8)).view(np.uint8)
    s = np.ones(out.shape[:3], np.float32) if few else np.exp(rng.standard_normal(out.shape[:3]) * (20 if seed % 2 else 0.1)).astype(np.float32)
    if few:
        out[..., :d] *= rng.integers(0, 2, (*out.shape[:3], 1), dtype=np.uint8)      # blocks with nothing in them
        out[..., d:2 * d] *= (out[..., :d].max(-1, keepdims=True) > 0).astype(np.uint8)
    out[..., 2 * d:2 * d + 4] = s[..., None].view(np.uint8)
    return out


@pytest.mark.parametrize("few", [False, True])
@pytest.mark.parametrize("B,lens,H,Hk,d,page,keep,recent", SELECTS)
def test_selection_is_the_definition(B, lens, H, Hk, d, page, keep, recent, few):
    rng = np.random.default_rng(keep)
    sub = page // 64
    most = -(-max(lens) // page)
    table = rng.permutation(B * most + 1).astype(np.int32)[:B * most].reshape(B, most)
    bounds = _bounds(B * most + 1, sub, Hk, d, keep, few)
    q = ref.bf16(rng.integers(-1, 2, (B, H, d)) if few else rng.standard_normal((B, H, d)))
    want = ref.select(q, bounds, table, lens, page, keep, recent)
    index = moda.moda_kv_select_blocks(ref.put(q), torch.from_numpy(bounds).cuda(), torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"),
                                       max(lens), keep, recent)
    assert moda.moda_last_status() == 0
    assert np.array_equal(index.cpu().numpy(), want)


@pytest.mark.parametrize("B,blocks,H,Hk,d,keep", [(40, 20, 32, 16, 64, 7), (20, 40, 160, 10, 128, 9), (2, 4200, 2, 1, 64, 33), (1, 11000, 3, 1, 128, 500), (9, 300, 256, 8, 128, 5),
                                                  (1, 4000, 6, 3, 64, 4)])
def test_selection_in_both_forms(B, blocks, H, Hk, d, keep):
    # many rows, very long ones, more heads than a CTA's warps, queries that take more shared memory than a kernel has without asking
    rng = np.random.default_rng(blocks)
    lens = [max(64 * blocks - 97 * b * b, 1) for b in range(B)]
    table = rng.permutation(B * blocks).astype(np.int32).reshape(B, blocks)
    bounds = _bounds(B * blocks, 1, Hk, d, 2, False)
    q = ref.bf16(rng.standard_normal((B, H, d)))
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    index = moda.moda_kv_select_blocks(ref.put(q), torch.from_numpy(bounds).cuda(), torch.from_numpy(table).cuda(), n, 64 * blocks, keep, 2).cpu().numpy()
    some = sorted({0, 1, B // 2, B - 1} & set(range(B)))
    assert np.array_equal(index[some], ref.select(q[some], bounds, table[some], [lens[b] for b in some], 64, keep, 2))


@pytest.mark.parametrize("B,Hk", [(1, 1), (2, 300), (400, 8)])
def test_selection_where_no_sequence_has_a_block(B, Hk):
    d = 64
    bounds = torch.zeros((1, 1, Hk, 2 * d + 16), dtype=torch.uint8, device="cuda")
    table, lens = torch.zeros((B, 1), dtype=torch.int32, device="cuda"), torch.zeros((B,), dtype=torch.int32, device="cuda")
    q = torch.ones((B, Hk, d), dtype=torch.bfloat16, device="cuda")
    for most in (0, 64):
        assert moda.moda_kv_select_blocks(q, bounds, table, lens, most, 3, 1).eq(-1).all()
    assert moda.moda_last_status() == 0


def test_selection_of_blocks_without_a_page_or_with_values_that_are_not_finite():
    d, n = 64, 50
    bounds = _bounds(n, 1, 1, d, 1, False)
    table = np.arange(n, dtype=np.int32)[None].copy()
    table[0, [3, 8]] = [-1, n]
    bounds[[20, 33], 0, 0, :2 * d] = 0
    bounds[[20, 33], 0, 0, 2 * d:2 * d + 4] = np.array([np.inf], np.float32).view(np.uint8)
    q = ref.bf16(np.random.default_rng(0).standard_normal((1, 4, d)))
    for keep in (2, 10, n - 1):
        got = moda.moda_kv_select_blocks(ref.put(q), torch.from_numpy(bounds).cuda(), torch.from_numpy(table).cuda(),
                                         torch.tensor([64 * n], dtype=torch.int32, device="cuda"), 64 * n, keep, 0).cpu().numpy()
        assert np.array_equal(got, ref.select(q, bounds, table, [64 * n], 64, keep, 0))
        assert {20, 33} <= set(got[0, 0])
    # queries that are zero or NaN: all ratings are equal, the lower blocks stay
    for v in (0.0, float("nan")):
        got = moda.moda_kv_select_blocks(ref.put(q * 0 + v), torch.from_numpy(bounds[:20]).cuda(), torch.arange(10, 20, dtype=torch.int32, device="cuda")[None].contiguous(),
                                         torch.tensor([640], dtype=torch.int32, device="cuda"), 640, 4, 1).cpu().numpy()
        assert got.tolist() == [[[0, 1, 2, 9]]]


DECODES = [  # B, lens, H, Hk, d, page, l
    (1, [1], 1, 1, 64, 64, 0), (1, [64], 2, 2, 128, 64, 3), (2, [63, 65], 6, 2, 64, 128, 0), (3, [0, 200, 1], 8, 1, 128, 64, 5), (4, [0, 0, 300, 0], 21, 3, 64, 256, 0),
    (2, [1000, 513], 4, 4, 128, 64, 33), (1, [3001], 5, 1, 64, 64, 2), (2, [700, 129], 16, 1, 128, 128, 4), (1, [400], 64, 2, 64, 64, 1), (3, [0, 0, 0], 4, 2, 64, 64, 2),
]


def _decode(B, lens, H, Hk, d, page, l, index=None, seed=0, scale=None, sharp=1.0, **kw):
    T = max(max(lens), 1)
    pages, _, table, dev = ref.make(B, T, Hk, d, page, lens, seed=seed + d + B)
    rng = np.random.default_rng(seed + 5)
    q = ref.bf16(rng.standard_normal((B, H, d)) * sharp)
    depth = ref.bf16(rng.standard_normal((l, B, Hk, 2, d)))
    scale = d ** -0.5 if scale is None else scale
    idx = None if index is None else torch.from_numpy(index).cuda()
    O, LSE = moda.moda_attn_decode_e4m3(ref.put(q), dev[0], dev[2], torch.tensor(lens, dtype=torch.int32, device="cuda"), ref.put(depth) if l else None, T, l, scale,
                                        index=idx, **kw)
    assert moda.moda_last_status() == 0
    return O, LSE, ref.decode(q, pages, table, lens, depth, scale, page, index)


def _check(O, LSE, want):
    o, lse, o_tol, lse_tol = want
    O, LSE = O.double().cpu().numpy(), LSE.double().cpu().numpy()
    empty = np.isneginf(lse)
    assert np.array_equal(np.isneginf(LSE), empty) and (O[empty] == 0).all()
    assert (np.abs(O - o) <= o_tol).all(), float((np.abs(O - o) / np.maximum(o_tol, 1e-30)).max())
    off = np.abs(LSE[~empty] - lse[~empty]) / lse_tol[~empty]
    assert (off <= 1).all(), float(off.max())


@pytest.mark.parametrize("sharp", [1.0, 30.0])
@pytest.mark.parametrize("B,lens,H,Hk,d,page,l", DECODES)
def test_decode_against_64_bits(B, lens, H, Hk, d, page, l, sharp):
    _check(*_decode(B, lens, H, Hk, d, page, l, sharp=sharp))


@pytest.mark.parametrize("H,Hk,d", [(8, 2, 128), (3, 1, 64), (32, 1, 64)])
def test_decode_over_named_blocks(H, Hk, d):
    rng = np.random.default_rng(H)
    lens = [64 * 30 + 7, 0, 64 * 3, 50]
    index = np.full((4, Hk, 9), -1, np.int32)
    for k in range(Hk):
        index[0, k] = np.sort(rng.permutation(31)[:9])
        index[2, k, :3] = [0, 2, 1]
        index[3, k, 0] = 0
    index[0, 0, 4] = 31                                         # no block of the sequence: passed over
    index[2, 0, 1] = -5
    _check(*_decode(4, lens, H, Hk, d, 64, 2, index=index))
    _check(*_decode(4, lens, H, Hk, d, 128, 0, index=index))


def test_blocks_without_a_page_have_no_weight():
    B, lens, H, Hk, d = 1, [64 * 6], 4, 2, 128
    pages, _, table, dev = ref.make(B, lens[0], Hk, d, 128, lens, seed=9)
    table[0, 1] = pages.shape[0]
    q = ref.bf16(np.random.default_rng(1).standard_normal((B, H, d)))
    t = torch.from_numpy(table).cuda()
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    _check(*moda.moda_attn_decode_e4m3(ref.put(q), dev[0], t, n, None, lens[0], 0, 0.1), ref.decode(q, pages, table, lens, None, 0.1, 128))
    K, V = moda.moda_kv_read_e4m3(dev[0], t, n, lens[0])
    assert (K[0, 128:256] == 0).all() and (V[0, 128:256] == 0).all() and (K[0, :128] != 0).any()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("power", [-60, 60])
def test_values_of_very_different_sizes(d, power):
    # value rows around 2^power and far from each other: their scales go into the weights, which must neither overflow nor vanish
    B, n, H, Hk = 1, 300, 4, 2
    rng = np.random.default_rng(d)
    K = ref.bf16(rng.standard_normal((B, n, Hk, d)))
    V = ref.bf16(rng.standard_normal((B, n, Hk, d)) * 2.0 ** (power + rng.integers(-20, 21, (B, n, Hk, 1))))
    pages, bounds, table, dev = ref.make(B, n, Hk, d, 64, [n], seed=1)
    pages, _ = ref.write(pages, None, K, V, table, [0], [n], 64)
    q = ref.bf16(rng.standard_normal((B, H, d)) * 2.0 ** 40)
    scale = 2.0 ** -40 * d ** -0.5
    got = moda.moda_attn_decode_e4m3(ref.put(q), torch.from_numpy(pages).cuda(), dev[2], torch.tensor([n], dtype=torch.int32, device="cuda"), None, n, 0, scale)
    _check(*got, ref.decode(q, pages, table, [n], None, scale, 64))


def test_many_sequences():
    # more than a thread per sequence, and empty ones among them
    lens = [(37 * i) % 130 for i in range(700)]
    _check(*_decode(700, lens, 2, 1, 64, 64, 1))


def test_nan_stays_where_it_is():
    B, lens, H, Hk, d = 2, [100, 100], 4, 2, 64
    pages, _, table, dev = ref.make(B, 100, Hk, d, 64, lens, seed=2)
    q = ref.bf16(np.random.default_rng(1).standard_normal((B, H, d)))
    q[0, 1, 3] = np.nan
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    O, LSE = moda.moda_attn_decode_e4m3(ref.put(q), dev[0], dev[2], n, None, 100, 0, 0.1)
    bad = torch.isnan(O).all(-1).cpu().numpy()
    assert bad.tolist() == [[False, True, False, False], [False] * 4] and torch.isfinite(O[1]).all() and torch.isnan(LSE[0, 1])


def test_same_bits_again_on_another_stream_and_captured():
    B, lens, H, Hk, d, l = 3, [700, 64, 333], 8, 2, 128, 3
    pages, bounds, table, dev = ref.make(B, 700, Hk, d, 64, lens, seed=4)
    rng = np.random.default_rng(2)
    q, depth = ref.put(ref.bf16(rng.standard_normal((B, H, d)))), ref.put(ref.bf16(rng.standard_normal((l, B, Hk, 2, d))))
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    work = torch.empty(moda.moda_decode_e4m3_workspace_bytes(B, H, Hk, d), dtype=torch.uint8, device="cuda")

    def step(**kw):
        index = moda.moda_kv_select_blocks(q, dev[1], dev[2], n, 700, 5, 1, **kw)
        return (index, *moda.moda_attn_decode_e4m3(q, dev[0], dev[2], n, depth, 700, l, 0.1, index=index, **kw))

    first = step()
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        second = step()
    third = step(stream=other)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        index = moda.moda_kv_select_blocks(q, dev[1], dev[2], n, 700, 5, 1)
        fourth = (index, *moda.moda_attn_decode_e4m3(q, dev[0], dev[2], n, depth, 700, l, 0.1, index=index, workspace=work))
    for t in fourth:
        t.zero_()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for got in (second, third, fourth):
        assert all(torch.equal(x, y) for x, y in zip(first, got))


def test_captured_behind_copies_and_other_streams():
    # the calls as a graph's first node, behind a copy, and behind two streams at once: replays see what is in the buffers then
    B, lens, H, Hk, d = 2, [400, 129], 4, 2, 64
    pages, bounds, table, dev = ref.make(B, 400, Hk, d, 64, lens, seed=7)
    rng = np.random.default_rng(3)
    q = [ref.put(ref.bf16(rng.standard_normal((B, H, d)))) for _ in range(2)]
    rows = [ref.put(ref.bf16(rng.standard_normal((B, 1, Hk, d)))) for _ in range(2)]
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ends = n - 1
    names = [torch.tensor([[[0, 2, 5], [1, 4, 6]], [[0, 1, 2], [1, 2, -1]]], dtype=torch.int32, device="cuda"),
             torch.tensor([[[3, 4, 6], [0, 1, 2]], [[2, -1, -1], [0, 2, -1]]], dtype=torch.int32, device="cuda")]
    own = [t.clone() for t in dev[:2]]
    qs, row, index, ix2 = q[0].clone(), rows[0].clone(), names[0].clone(), torch.empty_like(names[0])

    def first():
        return moda.moda_attn_decode_e4m3(qs, own[0], dev[2], n, None, 400, 0, 0.2, index=index)

    def copied():
        ix2.copy_(index)
        return moda.moda_attn_decode_e4m3(qs, own[0], dev[2], n, None, 400, 0, 0.2, index=ix2)

    def joined():
        here, beside = torch.cuda.current_stream(), torch.cuda.Stream()
        beside.wait_stream(here)
        with torch.cuda.stream(beside):
            ix2.copy_(index)
        moda.moda_kv_write_e4m3(own[0], row, row, dev[2], start=ends, bounds=own[1])
        here.wait_stream(beside)
        out = moda.moda_attn_decode_e4m3(qs, own[0], dev[2], n, None, 400, 0, 0.2, index=ix2)
        return (*out, moda.moda_kv_select_blocks(qs, own[1], dev[2], n, 400, 3, 1), *moda.moda_kv_read_e4m3(own[0], dev[2], n, 400))

    for step in (first, copied, joined):
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = step()
        for i in (1, 0):
            qs.copy_(q[i]), row.copy_(rows[i]), index.copy_(names[i])
            for t, src in zip(own, dev[:2]):
                t.copy_(src)
            graph.replay()
            got_i = [t.clone() for t in got]
            for t, src in zip(own, dev[:2]):
                t.copy_(src)
            assert all(torch.equal(a, b) for a, b in zip(got_i, step()))
        del graph
    assert moda.moda_last_status() == 0


@pytest.mark.parametrize("d", [64, 128])
def test_behind_calls_whose_kernels_start_early(d):
    # what the calls over the pages read is written by calls that launch their own last kernels beside one another: the same bits with and without a wait on the host in between
    B, T, H, l = 2, 700, 4, 3
    x = synthetic.make(synthetic.Workload("chain", B=B, T=T, H=H, d=d, l=l), seed=3, device="cuda:0")
    cache = moda.alloc_depth_cache(B, T, H, d, l, "cuda:0")
    for i in range(l):
        moda.moda_depth_cache_append(cache, i, x["Kd"][i].contiguous(), x["Vd"][i].contiguous())
    n = torch.tensor([T, T - 130], dtype=torch.int32, device="cuda")
    most = -(-T // 64)
    table = torch.arange(B * most, dtype=torch.int32, device="cuda").reshape(B, most)
    scale = d ** -0.5

    def chain(wait):
        pages, bounds = torch.zeros_like(moda.alloc_kv_pages_e4m3(B * most, 64, H, d)), torch.zeros_like(moda.alloc_kv_bounds(B * most, 64, H, d))
        steps = []
        def then(*out):
            if wait:
                torch.cuda.synchronize()
            steps.extend(out)
            return out
        O, LSE = then(*moda.moda_attn_fwd(x["Q"], x["K"], x["V"], cache, l, scale))
        _, dK, dV, _ = moda.moda_attn_bwd(x["Q"], x["K"], x["V"], cache, O, x["dO"], LSE, l, scale)
        then(dK, dV)
        moda.moda_kv_write_e4m3(pages, dK, dV, table, n_new=n, bounds=bounds)
        then(pages, bounds)
        q = dK[:, 5].contiguous()
        index, = then(moda.moda_kv_select_blocks(q, bounds, table, n, T, 4, 1))
        o, lse = then(*moda.moda_attn_decode_e4m3(q, pages, table, n, None, T, 0, scale, index=index))
        moda.moda_kv_write_e4m3(pages, o[:, None], o[:, None], table, start=n - 1, bounds=bounds)
        K, V = then(*moda.moda_kv_read_e4m3(pages, table, n, T))
        then(*moda.moda_attn_decode(q, K, V, x["Kd"].new_zeros((1, B, H, 2, d)), T, 1, scale))
        moda.moda_kv_write_e4m3(pages, K, V, table, n_new=n - 3, bounds=bounds)
        then(*moda.moda_attn_decode_e4m3(o, pages, table, n, None, T, 0, scale))
        return steps

    want = [t.clone() for t in chain(True)]
    for _ in range(20):
        got = chain(False)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert moda.moda_last_status() == 0


def test_pages_far_from_the_first():
    # more than 2^32 bytes into the pages
    d, Hk, page = 128, 8, 256
    num = (1 << 32) // moda.moda_kv_page_e4m3_bytes(page, Hk, d) + 40
    pages, bounds = moda.alloc_kv_pages_e4m3(num, page, Hk, d), moda.alloc_kv_bounds(num, page, Hk, d)
    n = 700
    table = torch.tensor([[num - 1, num - 30, num - 2]], dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(0)
    K, V = (ref.bf16(rng.standard_normal((1, n, Hk, d))) for _ in range(2))
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    moda.moda_kv_write_e4m3(pages, ref.put(K), ref.put(V), table, bounds=bounds)
    small, few = moda.alloc_kv_pages_e4m3(3, page, Hk, d), moda.alloc_kv_bounds(3, page, Hk, d)
    near = torch.tensor([[1, 0, 2]], dtype=torch.int32, device="cuda")
    moda.moda_kv_write_e4m3(small, ref.put(K), ref.put(V), near, bounds=few)
    q = ref.put(ref.bf16(rng.standard_normal((1, 16, d))))
    for a, b in zip(moda.moda_kv_read_e4m3(pages, table, lens, n), moda.moda_kv_read_e4m3(small, near, lens, n)):
        assert torch.equal(a, b) and a.any()
    index = moda.moda_kv_select_blocks(q, bounds, table, lens, n, 4, 1)
    assert torch.equal(index, moda.moda_kv_select_blocks(q, few, near, lens, n, 4, 1))
    for i in (None, index):
        got, want = (moda.moda_attn_decode_e4m3(q, x, t, lens, None, n, 0, 0.1, index=i) for x, t in ((pages, table), (small, near)))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_nothing_is_written_beside_the_outputs():
    B, H, Hk, d, l, lens = 3, 6, 2, 64, 2, [130, 0, 65]
    pages, bounds, table, dev = ref.make(B, 130, Hk, d, 64, lens, seed=11)
    rng = np.random.default_rng(3)
    q, depth = ref.put(ref.bf16(rng.standard_normal((B, H, d)))), ref.put(ref.bf16(rng.standard_normal((l, B, Hk, 2, d))))
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    band = lambda count, dtype: torch.full((count + 128,), 77, dtype=dtype, device="cuda")
    Ob, Lb, Ib = band(B * H * d, torch.bfloat16), band(B * H, torch.float32), band(B * Hk * 3, torch.int32)
    Wb = band(moda.moda_decode_e4m3_workspace_bytes(B, H, Hk, d), torch.uint8)
    Sb = band(moda.moda_kv_select_workspace_bytes(B, 130, Hk), torch.uint8)
    cut = lambda t, *s: t[64:-64].view(*s)
    moda.moda_kv_select_blocks(q, dev[1], dev[2], n, 130, 3, 1, index=cut(Ib, B, Hk, 3), workspace=cut(Sb, -1))
    moda.moda_attn_decode_e4m3(q, dev[0], dev[2], n, depth, 130, l, 0.1, O=cut(Ob, B, H, d), LSE=cut(Lb, B, H), workspace=cut(Wb, -1))
    torch.cuda.synchronize()
    for t in (Ob, Lb, Ib, Wb, Sb):
        assert (t[:64] == 77).all() and (t[-64:] == 77).all()
    assert np.array_equal(dev[0].cpu().numpy(), pages) and np.array_equal(dev[1].cpu().numpy(), bounds)
