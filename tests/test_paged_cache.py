"""PagedCache: which sequence has which page, lengths and refusals (on the CPU, with the kernels' calls left out)."""
import pytest
import torch

import paper_2603_15619_b200 as moda
from paper_2603_15619_b200 import binding

BF16 = torch.bfloat16


@pytest.fixture
def calls(monkeypatch):
    made = []
    monkeypatch.setattr(binding, "moda_kv_write_e4m3", lambda pages, K, V, table, start, n_new, bounds: made.append((start.tolist(), None if n_new is None else n_new.tolist())))
    return made


def cache(**kw):
    return moda.PagedCache(**{**dict(B=3, H_kv=2, d=64, num_pages=7, max_len=300, page_size=128, device="cpu"), **kw})


def rows(T, B=3):
    return torch.zeros((B, T, 2, 64), dtype=BF16)


def used(c):
    return [[p for p in row if p >= 0] for row in c.table.tolist()]


def test_pages_go_to_the_sequences_that_need_them(calls):
    c = cache()
    assert c.table.shape == (3, 3) and c.free_pages == 7 and c.longest == 0
    c.write(rows(129), rows(129), n_new=[129, 0, 128])
    assert [len(x) for x in used(c)] == [2, 0, 1] and c.free_pages == 4 and c.lengths == [129, 0, 128] and c.lens.tolist() == c.lengths
    c.write(rows(1), rows(1))
    assert [len(x) for x in used(c)] == [2, 1, 2] and c.lengths == [130, 1, 129] and c.longest == 130
    flat = sum(used(c), [])
    assert len(set(flat)) == len(flat) == 5 and all(0 <= p < 7 for p in flat)
    assert calls == [([0, 0, 0], [129, 0, 128]), ([129, 0, 128], None)]
    c.release(0)
    assert c.free_pages == 4 and c.lengths == [0, 1, 129] and c.lens.tolist() == c.lengths and used(c)[0] == []
    c.write(rows(300), rows(300), n_new=[300, 0, 0])
    flat = sum(used(c), [])
    assert len(set(flat)) == len(flat) == 6 and c.lengths == [300, 1, 129]


def test_refusals_leave_the_cache_as_it_was(calls):
    c = cache()
    c.write(rows(200), rows(200))
    state = c.table.clone(), list(c.lengths), c.free_pages
    for K, V, n in ((rows(101), rows(101), None), (rows(100), rows(100), [100, 100, 101]), (rows(100), rows(100), [1, 1]), (rows(100), rows(100), [-1, 0, 0]),
                    (rows(5, B=2), rows(5, B=2), None), (rows(5), rows(4), None), (rows(5).float(), rows(5), None), (rows(10)[:, ::2], rows(10)[:, ::2], None),
                    (rows(60), rows(60), [60, 60, 60])):                                  # the last: two pages, one is free
        with pytest.raises(ValueError):
            c.write(K, V, n_new=n)
        assert torch.equal(c.table, state[0]) and c.lengths == state[1] and c.free_pages == state[2]
    with pytest.raises(ValueError):
        cache(page_size=100)
    with pytest.raises(ValueError):
        cache(max_len=0)
    with pytest.raises(ValueError):
        cache(bounds=False).select(torch.zeros((3, 2, 64), dtype=BF16), 4)
    with pytest.raises(ValueError):
        c.attend(torch.zeros((3, 2, 64), dtype=BF16), None, 0, 0.1, n_blocks=2, index=torch.zeros((3, 2, 2), dtype=torch.int32))
