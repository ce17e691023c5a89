"""The calls over the paged cache in 8 bits through the host extension: what it hands back, and that its results are those of the Python form."""
import pytest
import torch

import paper_2603_15619_b200 as moda
from paper_2603_15619_b200 import binding

from test_host_path import _Refuses

BF16 = torch.bfloat16
NAMES = ["write", "write_bounds", "read", "read_new", "select", "decode", "decode_index", "decode_l0"]


def test_what_is_not_plain_is_handed_back():
    host = binding.host()
    for t in (torch.zeros(1, 1, 2, 8704, dtype=torch.uint8), torch.empty(1, 1, 2, 8704, device="meta", dtype=torch.uint8), None, 3):
        assert host.kv_write(t, t, t, t, None, None, None) is None
        assert host.kv_read(t, t, t, 4, None, t, t) is None
        assert host.kv_select(t, t, t, t, 4, 2, 1, None, None) is None
        assert host.decode_e4m3(t, t, t, t, None, 4, 0, 0.1, None, None, None, None) is None
    assert host.kv_write() is None and host.kv_read() is None and host.kv_select() is None and host.decode_e4m3() is None


def calls():
    g = torch.Generator(device="cuda").manual_seed(1)
    n = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=BF16)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    B, T, H, Hk, d, l = 2, 300, 8, 2, 64, 3
    K, V, q, depth = n(B, T, Hk, d), n(B, T, Hk, d), n(B, H, d), n(l, B, Hk, 2, d)
    pages, bounds = moda.alloc_kv_pages_e4m3(6, 128, Hk, d).zero_(), moda.alloc_kv_bounds(6, 128, Hk, d).zero_()
    table, lens = i32([4, 0, 2], [1, 3, 5]), i32(300, 17)
    moda.moda_kv_write_e4m3(pages, K, V, table, bounds=bounds)
    index = i32([[0, 2], [1, 4]], [[0, -1], [0, -1]])
    p2, b2 = torch.zeros_like(pages), torch.zeros_like(bounds)

    def write(b, **k):
        moda.moda_kv_write_e4m3(p2.zero_(), K, V, table, start=i32(3, 70), n_new=i32(290, 33), bounds=None if b is None else b.zero_(), **k)
        return [p2] if b is None else [p2, b]

    return {
        "write": lambda **k: write(None, **k),
        "write_bounds": lambda **k: write(b2, **k),
        "read": lambda **k: moda.moda_kv_read_e4m3(pages, table, lens, 100, start=i32(7, 9), K_out=torch.zeros((B, 100, Hk, d), device="cuda", dtype=BF16),
                                                   V_out=torch.zeros((B, 100, Hk, d), device="cuda", dtype=BF16), **k),
        "read_new": lambda **k: moda.moda_kv_read_e4m3(pages, table, lens, 300, **k),
        "select": lambda **k: moda.moda_kv_select_blocks(q, bounds, table, lens, T, 3, 1, **k),
        "decode": lambda **k: moda.moda_attn_decode_e4m3(q, pages, table, lens, depth, T, l, 0.125, **k),
        "decode_index": lambda **k: moda.moda_attn_decode_e4m3(q, pages, table, lens, depth, T, l, 0.125, index=index, **k),
        "decode_l0": lambda **k: moda.moda_attn_decode_e4m3(q, pages, table, lens, None, T, 0, 0.125, **k),
    }


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_results_are_those_of_the_python_form(name, monkeypatch):
    f = calls()[name]
    served = []
    real = binding.host()

    class Watch:
        def __getattr__(self, fn):
            def call(*a):
                out = getattr(real, fn)(*a)
                served.append(out is not None)
                return out
            return call

    flat = lambda r: [x.clone() for x in (r if isinstance(r, (tuple, list)) else [r])]
    with monkeypatch.context() as m:
        m.setattr(binding, "host", lambda: Watch())
        fast = flat(f())
    assert served == [name != "read_new"]                                # outputs that are made for the caller: the Python form
    with monkeypatch.context() as m:
        m.setattr(binding, "host", lambda: _Refuses())
        slow = flat(f())
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = flat(f(stream=s))
    s.synchronize()
    assert len(fast) == len(slow) == len(other)
    for a, b, c in zip(fast, slow, other):
        assert torch.equal(a, b) and a.shape == b.shape and a.dtype == b.dtype and torch.equal(a, c)


@pytest.mark.gpu
def test_errors_come_as_from_the_python_form():
    g = torch.Generator(device="cuda").manual_seed(1)
    n = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=BF16)
    pages, bounds = moda.alloc_kv_pages_e4m3(2, 64, 2, 64), moda.alloc_kv_bounds(2, 64, 2, 64)
    q, K = n(1, 4, 64), n(1, 5, 2, 64)
    table, lens = torch.zeros((1, 2), dtype=torch.int32, device="cuda"), torch.zeros((1,), dtype=torch.int32, device="cuda")
    for f, code in [
        (lambda: moda.moda_kv_select_blocks(q, bounds, table, lens, 129, 2), -3), (lambda: moda.moda_kv_select_blocks(q, bounds, table, lens, 100, 2, 3), -3),
        (lambda: moda.moda_kv_select_blocks(n(1, 3, 64), bounds, table, lens, 100, 2), -12), (lambda: moda.moda_kv_select_blocks(q, bounds, table, lens, 100, 0), -3),
        (lambda: moda.moda_attn_decode_e4m3(q, pages, table, lens, None, 129, 0, 0.1), -3), (lambda: moda.moda_attn_decode_e4m3(q, pages, table, lens, None, 100, 0, 0.0), -13),
        (lambda: moda.moda_attn_decode_e4m3(q, pages, table, lens, None, 100, 0, 0.1, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), -7),
        (lambda: moda.moda_kv_read_e4m3(pages, table, lens, 0), -3),
    ]:
        with pytest.raises(moda.ModaError) as e:
            f()
        assert e.value.code == code
    with pytest.raises(ValueError):                                          # not contiguous
        moda.moda_kv_write_e4m3(pages, K.transpose(1, 2).contiguous().transpose(1, 2), K, table)
    with pytest.raises(ValueError):                                          # another width
        moda.moda_kv_write_e4m3(pages, n(1, 5, 2, 128), n(1, 5, 2, 128), table)
    torch.cuda.synchronize()
