"""What the calls over the paged cache in 8 bits refuse, before anything touches a device; the plain forms that the GPU tests compare with; launch rules."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

import paper_2603_15619_b200 as moda
from paper_2603_15619_b200 import binding, build

import pages_ref as ref

P = ctypes.c_void_p(4096)                   # aligned, never dereferenced: validation fails first
ODD = ctypes.c_void_p(4100)
CROOKED = ctypes.c_void_p(4098)
F = ctypes.c_float


def test_sizes():
    assert moda.moda_kv_page_e4m3_bytes(64, 2, 128) == 2 * (2 * 64 * 128 + 2 * 64 * 4)
    assert moda.moda_kv_page_e4m3_bytes(256, 3, 64) == 4 * 3 * (2 * 64 * 64 + 2 * 64 * 4)
    assert moda.moda_kv_page_bounds_bytes(128, 5, 64) == 2 * 5 * (2 * 64 + 16)
    for bad in ((0, 1, 64), (96, 1, 64), (64, 0, 64), (64, 1, 96)):
        assert moda.moda_kv_page_e4m3_bytes(*bad) == 0 and moda.moda_kv_page_bounds_bytes(*bad) == 0
        with pytest.raises(ValueError):
            moda.alloc_kv_pages_e4m3(1, *bad)
        with pytest.raises(ValueError):
            moda.alloc_kv_bounds(1, *bad)
    assert moda.moda_decode_e4m3_workspace_bytes(2, 8, 2, 64) > 0
    for bad in ((0, 8, 2, 64), (2049, 8, 2, 64), (2, 9, 2, 64), (2, 9, 1, 64), (2, 8, 2, 80)):
        assert moda.moda_decode_e4m3_workspace_bytes(*bad) == 0


def rows_call(f, pages=P, K=P, V=P, table=P, start=None, n=P, B=2, T=100, page=64, pages_n=10, most=4, Hk=2, d=64, bounds=None):
    if f == "write":
        return binding.load().moda_kv_write_e4m3(pages, bounds, K, V, table, start, n, B, T, page, pages_n, most, Hk, d, None)
    return binding.load().moda_kv_read_e4m3(pages, table, n, start, B, T, page, pages_n, most, Hk, d, K, V, None)


@pytest.mark.parametrize("f", ["write", "read"])
def test_rows_validation(f):
    call = lambda **k: rows_call(f, **k)
    for bad in (dict(B=0), dict(T=0), dict(T=-1), dict(page=0), dict(page=100), dict(page=32), dict(pages_n=0), dict(most=0), dict(Hk=0), dict(B=70000), dict(Hk=70000),
                dict(T=1 << 30), dict(page=1 << 20, pages_n=1 << 20), dict(page=1 << 20, most=1 << 20)):
        assert call(**bad) == -3, bad
    assert call(d=96) == -4
    for name in ("pages", "K", "V", "table"):
        assert call(**{name: None}) == -1, name
    for name in ("pages", "K", "V"):
        assert call(**{name: ODD}) == -2, name
    for name in ("table", "start", "n"):
        assert call(**{name: CROOKED}) == -2, name
    if f == "write":
        assert call(bounds=ODD) == -2
    else:
        assert call(n=None) == -1


def test_select_validation():
    need = moda.moda_kv_select_workspace_bytes(2, 200, 2)
    assert need >= 2 * 2 * 4 * 4 and moda.moda_kv_select_workspace_bytes(1, 64 * 32768 + 1, 1) == 0 and moda.moda_kv_select_workspace_bytes(0, 5, 1) == 0

    def call(q=P, bounds=P, table=P, lens=P, B=2, T=200, page=64, pages_n=10, most=4, H=4, Hk=2, d=64, n=3, recent=1, index=P, work=P, wb=need):
        return binding.load().moda_kv_select_blocks(q, bounds, table, lens, B, T, page, pages_n, most, H, Hk, d, n, recent, index, work, ctypes.c_size_t(wb), None)

    assert call(work=None) == -7 and call(work=ODD) == -7 and call(wb=need - 1) == -7

    for bad in (dict(B=0), dict(T=-1), dict(T=257), dict(page=65), dict(pages_n=0), dict(n=0), dict(recent=-1), dict(recent=4), dict(H=0), dict(n=1 << 30),
                dict(T=64 * 32768 + 1, most=1 << 20)):
        assert call(**bad) == -3, bad
    assert call(d=32) == -4 and call(H=5) == -12 and call(H=18) == -12
    for name in ("q", "bounds", "table", "lens", "index"):
        assert call(**{name: None}) == -1, name
        assert call(**{name: CROOKED}) == -2, name


def test_decode_validation():
    need = moda.moda_decode_e4m3_workspace_bytes(2, 4, 2, 64)

    def call(q=P, pages=P, table=P, lens=P, index=None, n=0, depth=P, B=2, T=200, page=64, pages_n=10, most=4, H=4, Hk=2, d=64, l=1, scale=0.1, O=P, LSE=P, work=P, wb=need):
        return binding.load().moda_attn_decode_e4m3(q, pages, table, lens, index, n, depth, B, T, page, pages_n, most, H, Hk, d, l, F(scale), O, LSE, work,
                                                    ctypes.c_size_t(wb), None)

    for bad in (dict(B=0), dict(B=2049), dict(T=-1), dict(T=257), dict(page=65), dict(pages_n=0), dict(index=P), dict(index=P, n=1 << 30), dict(H=0)):
        assert call(**bad) == -3, bad
    assert call(d=32) == -4 and call(H=5) == -12 and call(H=18) == -12 and call(l=-1) == -5 and call(l=257) == -5
    assert call(scale=0.0) == -13 and call(scale=float("nan")) == -13
    for name in ("q", "pages", "table", "lens", "depth", "O", "LSE"):
        assert call(**{name: None}) == -1, name
        assert call(**{name: CROOKED}) == -2, name
    assert call(index=CROOKED, n=1) == -2
    assert call(work=None) == -7 and call(work=ODD) == -7 and call(wb=need - 1) == -7


def test_the_binding_refuses_tensors_of_other_shapes_and_types():
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
    pages, bounds, table, lens = u8(5, 2, 3, 128 * 64 + 512), u8(5, 2, 3, 2 * 64 + 16), i32(2, 4), i32(2)
    q, K = bf(2, 6, 64), bf(2, 9, 3, 64)
    ok_write = dict(pages=pages, K=K, V=K, block_table=table)
    for bad in (dict(pages=pages.to(torch.int8)), dict(pages=u8(5, 2, 3, 8000)), dict(block_table=table.long()), dict(block_table=i32(3, 4)), dict(K=bf(2, 9, 2, 64)),
                dict(V=bf(2, 8, 3, 64)), dict(start=i32(3)), dict(n_new=lens.long()), dict(bounds=u8(5, 2, 3, 143)), dict()):
        with pytest.raises(ValueError):                                     # the last: no device tensors
            moda.moda_kv_write_e4m3(**{**ok_write, **bad})
    for bad in (dict(seq_lens=lens.long()), dict(start=i32(1)), dict(K_out=bf(2, 8, 3, 64)), dict(V_out=K.float())):
        with pytest.raises(ValueError):
            moda.moda_kv_read_e4m3(**{**dict(pages=pages, block_table=table, seq_lens=lens, T=9, K_out=K, V_out=K), **bad})
    for bad in (dict(q=bf(3, 6, 64)), dict(q=bf(2, 6, 128)), dict(bounds=pages), dict(seq_lens=i32(3)), dict(index=i32(2, 3, 4)), dict()):
        with pytest.raises(ValueError):
            moda.moda_kv_select_blocks(**{**dict(q=q, bounds=bounds, block_table=table, seq_lens=lens, max_seq_len=100, n_blocks=2, index=i32(2, 3, 2)), **bad})
    ok = dict(q=q, pages=pages, block_table=table, seq_lens=lens, depth_kv_token=None, max_seq_len=100, l=0, scale=0.1)
    for bad in (dict(q=bf(2, 6, 128)), dict(seq_lens=i32(2, 1)), dict(index=i32(2, 6, 2)), dict(l=1), dict(O=bf(2, 5, 64)), dict(LSE=torch.zeros(3)), dict()):
        with pytest.raises(ValueError):
            moda.moda_attn_decode_e4m3(**{**ok, **bad})


def test_plain_forms_agree_with_themselves():
    # written and read back: within half a step of e4m3 of the row's scale; a block's bounds hold its keys
    rng = np.random.default_rng(0)
    d, n = 64, 150
    K = ref.bf16(rng.standard_normal((1, n, 2, d)))
    pages, bounds = np.zeros((4, 1, 2, 128 * d + 512), np.uint8), np.zeros((4, 1, 2, 2 * d + 16), np.uint8)
    table = np.array([[2, 0, 3]], np.int32)
    pages, bounds = ref.write(pages, bounds, K, K, table, [0], [n], 64)
    for k in range(2):
        got, values = ref.gather(pages, table, 0, k, n, 64, d)
        assert np.array_equal(got, values)
        step = np.maximum(np.abs(K[0, :, k]) * 2.0 ** -4, np.abs(K[0, :, k]).max(-1, keepdims=True) / 448 * 2.0 ** -10)
        assert (np.abs(got - K[0, :, k]) <= step * 1.001).all()
        for j, page in enumerate(table[0]):
            keys = got[64 * j:64 * j + 64]
            b = bounds[page, 0, k]
            s = b[2 * d:2 * d + 4].view(np.float32)[0]
            assert (keys <= b[:d].view(np.int8) * s * 1.000001).all() and (keys >= b[d:2 * d].view(np.int8) * s * 1.000001).all()
    assert not pages[1].any() and not bounds[1].any()
    # a selection of all blocks changes nothing, and the chosen ones are the highest rated
    q = ref.bf16(rng.standard_normal((1, 4, d)))
    index = ref.select(q, bounds, table, [n], 64, 3, 1)
    assert index.tolist() == [[[0, 1, 2]] * 2]
    o, lse, *_ = ref.decode(q, pages, table, [n], None, 0.1, 64)
    o2, lse2, *_ = ref.decode(q, pages, table, [n], None, 0.1, 64, index)
    assert np.array_equal(o, o2) and np.array_equal(lse, lse2)
    assert ref.select(q, bounds, table, [0], 64, 2, 1).tolist() == [[[-1, -1]] * 2]


RULES = r"""
#include "launch_rules.h"
extern "C" int rate_rounds(int blocks, int step, int rows, int sms) { return moda::rate_rounds(blocks, step, rows, sms); }
extern "C" int select_ranks(int blocks, int rows, int sms) { return moda::select_ranks(blocks, rows, sms); }
"""


def test_forms_of_a_selection(tmp_path):
    src, so = tmp_path / "rules.cpp", tmp_path / "rules.so"
    src.write_text(RULES)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", f"-I{build.CSRC}", "-o", str(so), str(src)], check=True)
    lib = ctypes.CDLL(str(so))
    for blocks in (0, 1, 128, 129, 1000, 5000, 32768):
        for rows in (1, 8, 147, 148, 149, 592, 593, 10000):
            r = lib.rate_rounds(blocks, 128, rows, 148)
            ctas = lambda n: rows * -(-blocks // (128 * n))
            assert r in (1, 2, 4, 8) and (r == 8 or ctas(r) <= 8 * 148) and (r == 1 or ctas(r // 2) > 8 * 148)
            n = lib.select_ranks(blocks, rows, 148)
            assert n in (0, 1, 2, 4, 8) and rows * n <= 4 * 148 and (n < 2 or blocks > 64 * n)
            assert n > 0 or rows > 4 * 148 // 8 or blocks > 4096
    assert lib.select_ranks(1024, 8, 148) == 8 and lib.select_ranks(2048, 256, 148) == 0 and lib.select_ranks(32768, 1, 148) == 0
