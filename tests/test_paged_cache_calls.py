"""PagedCache: calls that are refused late, calls with nothing to do, an index that is older than a block (on the CPU, with the kernels' calls left out)."""
import pytest
import torch

import paper_2603_15619_b200 as moda
from paper_2603_15619_b200 import binding

BF16 = torch.bfloat16


def cache(**kw):
    return moda.PagedCache(**{**dict(B=3, H_kv=2, d=64, num_pages=7, max_len=300, page_size=128, device="cpu"), **kw})


def rows(T, B=3):
    return torch.zeros((B, T, 2, 64), dtype=BF16)


@pytest.fixture
def quiet(monkeypatch):
    made = []
    monkeypatch.setattr(binding, "moda_kv_write_e4m3", lambda *a, **k: made.append("write"))
    monkeypatch.setattr(binding, "moda_kv_select_blocks", lambda q, bounds, table, lens, longest, n, recent: torch.zeros((3, 2, n), dtype=torch.int32))
    monkeypatch.setattr(binding, "moda_attn_decode_e4m3", lambda *a, **k: made.append("attend"))
    return made


def state(c):
    return c.table.tolist(), c.lens.tolist(), list(c.lengths), [list(x) for x in c._owned], list(c._free)


def test_a_write_that_the_call_refuses_takes_no_pages(quiet, monkeypatch):
    c = cache()
    c.write(rows(100), rows(100), n_new=[100, 0, 128 - 28])
    before = state(c)

    def refuse(*a, **k):
        raise moda.ModaError(-2, "moda_kv_write_e4m3")

    for n_new in (None, [150, 130, 0], [0, 1, 0]):
        with monkeypatch.context() as m:
            m.setattr(binding, "moda_kv_write_e4m3", refuse)
            with pytest.raises(moda.ModaError):
                c.write(rows(150), rows(150), n_new=n_new)
        assert state(c) == before
    c.write(rows(1), rows(1))                                     # and the next one gets them
    assert c.lengths == [101, 1, 101] and [len(x) for x in c._owned] == [1, 1, 1]


def test_tensors_that_are_not_on_a_device_are_refused_without_effect():
    c = cache()
    before = state(c)
    with pytest.raises(ValueError):
        c.write(rows(200), rows(200))
    assert state(c) == before


def test_nothing_to_write_and_nothing_to_read(quiet):
    c = cache()
    K, V = c.read()
    assert K.shape == V.shape == (3, 0, 2, 64) and K.dtype == V.dtype == BF16
    c.write(rows(0), rows(0))
    c.write(rows(0), rows(0), n_new=[0, 0, 0])
    assert c.lengths == [0, 0, 0] and c.free_pages == 7 and quiet == []
    for bad in (dict(K=rows(0).float(), V=rows(0)), dict(K=rows(0), V=rows(1)), dict(K=rows(0), V=rows(0), n_new=[0, 0, 1]), dict(K=rows(0, B=2), V=rows(0, B=2))):
        with pytest.raises(ValueError):
            c.write(**bad)
    c.write(rows(5), rows(5))
    assert c.read(0)[0].shape == (3, 0, 2, 64)
    with pytest.raises(ValueError):
        c.read(-1)


def test_an_index_is_refused_once_a_sequence_has_opened_a_block(quiet):
    c, q = cache(), torch.zeros((3, 4, 64), dtype=BF16)
    attend = lambda index, cache=c: cache.attend(q, None, 0, 0.1, index=index)
    c.write(rows(100), rows(100), n_new=[63, 100, 0])
    index = c.select(q, 2)
    attend(index)
    c.write(rows(1), rows(1), n_new=[1, 1, 0])                     # 64 and 101 positions: the same blocks
    attend(index)
    c.write(rows(1), rows(1), n_new=[1, 0, 0])                     # the 65th position is not in it, whatever n_recent was
    with pytest.raises(ValueError, match="block"):
        attend(index)
    newer = c.select(q, 2)
    attend(newer)
    other = cache()                                                # a later layer's cache, with the same lengths and with others
    other.write(rows(101), rows(101), n_new=[65, 101, 0])
    attend(newer, other)
    with pytest.raises(ValueError, match="block"):
        attend(index, other)
    c.release(1)
    with pytest.raises(ValueError, match="block"):
        attend(newer)
    c.write(rows(100), rows(100), n_new=[0, 99, 0])
    newest = c.select(q, 2)
    c.release(1)
    c.write(rows(100), rows(100), n_new=[0, 99, 0])                # as many positions, of another sequence
    with pytest.raises(ValueError, match="sequence"):
        attend(newest)
    attend(torch.zeros((3, 2, 2), dtype=torch.int32))              # one of the caller's own making
    c.attend(q, None, 0, 0.1, n_blocks=2)
    assert quiet.count("attend") == 6
