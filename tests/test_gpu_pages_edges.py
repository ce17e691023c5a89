"""What the header says of the paged cache in 8 bits at its edges: table entries that are no page, positions behind the table's end, counts and starts outside their range, outputs
that a read makes."""
import numpy as np
import pytest
import torch

import paper_2603_15619_b200 as moda

import pages_ref as ref

pytestmark = pytest.mark.gpu

i32 = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("B,T,Hk,d,page,lens,start", [(1, 1, 1, 64, 64, [1], None), (3, 200, 2, 128, 128, [0, 200, 77], None), (2, 70, 3, 64, 64, [150, 90], [90, 33]),
                                                      (2, 129, 1, 128, 256, [300, 60], [255, 0]), (2, 65, 2, 64, 64, [70, 5], [70, 900])])
def test_a_read_fills_the_outputs_that_it_makes_with_zeros(B, T, Hk, d, page, lens, start):
    pages, _, table, dev = ref.make(B, max(lens), Hk, d, page, lens, seed=T)
    torch.full((2 * B * T * Hk * d * 2,), 7.0, device="cuda", dtype=torch.bfloat16)                    # what the next buffers are made of
    K, V = moda.moda_kv_read_e4m3(dev[0], dev[2], i32(lens), T, start=i32(start))
    assert K.shape == V.shape == (B, T, Hk, d) and moda.moda_last_status() == 0
    for b in range(B):
        s = start[b] if start else 0
        n = min(max(lens[b] - s, 0), T)
        for k in range(Hk):
            for got, want in zip((K, V), ref.gather(pages, table, b, k, lens[b], page, d)):
                assert np.array_equal(got[b, :n, k].float().cpu().numpy(), ref.bf16(want[s:s + n].astype(np.float32)))
        assert not K[b, n:].any() and not V[b, n:].any()


@pytest.mark.parametrize("d,page", [(64, 64), (128, 128)])
def test_writes_outside_the_table_and_its_ranges(d, page):
    # rows: a page that is none (two of them, either side of the range), behind the table's end, more rows than there are, fewer than none, a start before the first position and
    # one far behind the last
    B, T, Hk = 6, 150, 2
    start, n_new = [0, 3 * page - 70, 10, 7, -5, 2 ** 31 - 40], [150, 150, 10 ** 6, -3, 80, 150]
    pages, bounds, table, _ = ref.make(B, 3 * page, Hk, d, page, [3 * page] * B, seed=page)
    table[0, 0], table[1, 2], table[2, 1] = -1, pages.shape[0], 2 ** 31 - 1
    table[3, :] = -2 ** 31
    rng = np.random.default_rng(d)
    K, V = (ref.bf16(rng.standard_normal((B, T, Hk, d))) for _ in range(2))
    want = ref.write(pages, bounds, K, V, table, start, n_new, page)
    dev = [torch.from_numpy(x.copy()).cuda() for x in (pages, bounds, table)]
    moda.moda_kv_write_e4m3(dev[0], ref.put(K), ref.put(V), dev[2], start=i32(start), n_new=i32(n_new), bounds=dev[1])
    assert moda.moda_last_status() == 0
    assert np.array_equal(dev[0].cpu().numpy(), want[0]) and np.array_equal(dev[1].cpu().numpy()[..., :2 * d + 4], want[1][..., :2 * d + 4])
    assert not np.array_equal(want[0], pages)


def test_reads_outside_the_table_and_its_ranges():
    B, T, Hk, d, page = 4, 100, 2, 64, 64
    lens, start = [130, 10 ** 6, -4, 64], [-9, 150, 0, 2 ** 31 - 1]
    pages, _, table, dev = ref.make(B, 192, Hk, d, page, [192] * B, seed=1)
    K, V = (torch.full((B, T, Hk, d), 7.0, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    moda.moda_kv_read_e4m3(dev[0], dev[2], i32(lens), T, start=i32(start), K_out=K, V_out=V)
    rows = [(0, 100), (150, 42), (0, 0), (0, 0)]                         # first position, how many: the table ends at 192
    for b, (s, n) in enumerate(rows):
        for k in range(Hk):
            for got, want in zip((K, V), ref.gather(pages, table, b, k, 192, page, d)):
                assert np.array_equal(got[b, :n, k].float().cpu().numpy(), ref.bf16(want[s:s + n].astype(np.float32)))
        assert (K[b, n:] == 7).all() and (V[b, n:] == 7).all()
    assert moda.moda_last_status() == 0
