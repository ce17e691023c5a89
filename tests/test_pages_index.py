"""An index that names no block is refused, not taken for the one that is not given (which means all blocks)."""
import pytest
import torch

import paper_2603_15619_b200 as moda
from paper_2603_15619_b200 import binding

from test_host_path import _Refuses

BF16 = torch.bfloat16


def tensors(device):
    pages = torch.zeros((2, 1, 2, 128 * 64 + 512), dtype=torch.uint8, device=device)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=device)
    return torch.zeros((1, 4, 64), dtype=BF16, device=device), pages, i32(1, 2), i32(1) + 70, i32(1, 2, 0)


def test_the_binding_says_so_before_it_looks_at_addresses():
    q, pages, table, lens, none = tensors("cpu")
    with pytest.raises(ValueError, match="no block"):
        moda.moda_attn_decode_e4m3(q, pages, table, lens, None, 100, 0, 0.1, index=none)


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["extension", "python", "stream"])
def test_refused_in_every_form(form, monkeypatch):
    q, pages, table, lens, none = tensors("cuda")
    O, LSE = torch.full_like(q, 7.0), torch.full((1, 4), 7.0, device="cuda")
    if form == "python":
        monkeypatch.setattr(binding, "host", lambda: _Refuses())
    with pytest.raises(ValueError, match="no block"):
        moda.moda_attn_decode_e4m3(q, pages, table, lens, None, 100, 0, 0.1, index=none, O=O, LSE=LSE, stream=torch.cuda.current_stream() if form == "stream" else None)
    torch.cuda.synchronize()
    assert (O == 7).all() and (LSE == 7).all()


@pytest.mark.gpu
def test_refused_by_the_class():
    cache = moda.PagedCache(1, 2, 64, num_pages=2, max_len=128)
    k = torch.ones((1, 70, 2, 64), dtype=BF16, device="cuda")
    cache.write(k, k)
    with pytest.raises(ValueError, match="no block"):
        cache.attend(torch.ones((1, 4, 64), dtype=BF16, device="cuda"), None, 0, 0.1, index=torch.empty((1, 2, 0), dtype=torch.int32, device="cuda"))
