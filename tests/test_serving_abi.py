"""What the serving entry points refuse, before anything touches a device, and what their sources show."""
import ctypes
import os
import re

import pytest
import torch

import paper_2603_15619_b200 as moda
from paper_2603_15619_b200 import binding, build

from test_wait_reporting import kernels, source

P = ctypes.c_void_p(4096)                   # aligned, never dereferenced: validation fails first
ODD = ctypes.c_void_p(4100)
FAR = ctypes.c_void_p(1 << 40)
F = ctypes.c_float


def test_key_mass_validation():
    lib = binding.load()
    need = moda.moda_key_mass_workspace_bytes(1, 10, 20, 8, 2, 128)
    assert need > 0 and moda.moda_key_mass_workspace_bytes(1, 30, 20, 8, 2, 128) == 0 and moda.moda_key_mass_workspace_bytes(1, 10, 20, 8, 3, 128) == 0

    def call(Q=P, K=P, LSE=P, old=None, B=1, T_q=10, T_kv=20, T_cap=24, H=8, Hk=2, d=128, scale=0.1, mass=P, work=P, wb=need):
        return lib.moda_attn_key_mass(Q, K, LSE, old, B, T_q, T_kv, T_cap, H, Hk, d, F(scale), mass, work, ctypes.c_size_t(wb), None)

    assert call(B=0) == -3 and call(T_q=0) == -3 and call(T_q=21) == -3 and call(T_cap=19) == -3 and call(T_cap=1 << 29) == -3
    assert call(d=96) == -4 and call(scale=0.0) == -13 and call(scale=float("nan")) == -13
    assert call(Hk=3) == -12 and call(H=12, Hk=1) == -12 and call(Hk=0) == -12
    assert call(Q=None) == -1 and call(K=None) == -1 and call(LSE=None) == -1 and call(mass=None) == -1
    assert call(K=ODD) == -2 and call(old=ODD) == -2 and call(mass=ODD) == -2
    assert call(work=None) == -7 and call(wb=need - 1) == -7 and call(work=ODD) == -7


def test_decode_mass_validation():
    lib = binding.load()
    need = moda.moda_decode_mass_workspace_bytes(2, 100, 8, 2, 64)
    assert need >= moda.moda_decode_workspace_bytes(2, 8, 64) + 2 * 8 * 100 * 4 and moda.moda_decode_mass_workspace_bytes(2, 0, 8, 2, 64) == 0

    def call(q=P, K=P, lens=None, depth=P, old=None, B=2, T=100, T_cap=128, H=8, Hk=2, d=64, l=2, scale=0.1, mass=P, work=P, wb=need):
        return lib.moda_attn_decode_mass(q, K, P, lens, depth, old, B, T, T_cap, H, Hk, d, l, F(scale), P, P, mass, work, ctypes.c_size_t(wb), None)

    assert call(B=0) == -3 and call(T=0) == -3 and call(T=129) == -3 and call(B=70000) == -3
    assert call(d=32) == -4 and call(l=-1) == -5 and call(l=257) == -5 and call(scale=-1.0) == -13
    assert call(Hk=3) == -12 and call(H=72, Hk=2) == -12
    assert call(q=None) == -1 and call(depth=None) == -1 and call(mass=None) == -1
    assert call(K=ODD) == -2 and call(lens=ctypes.c_void_p(4098)) == -2 and call(old=ODD) == -2
    assert call(work=None) == -7 and call(wb=need - 1) == -7


def test_evict_validation():
    lib = binding.load()

    def call(K=P, V=P, mass=P, lens=None, B=1, T=100, T_cap=128, Hk=2, d=64, keep=50, recent=10, T_out=64, K_out=FAR, V_out=FAR, index=FAR, mass_out=None):
        return lib.moda_kv_evict(K, V, mass, lens, B, T, T_cap, Hk, d, keep, recent, T_out, K_out, V_out, mass_out, index, None, None)

    assert call(B=0) == -3 and call(T=0) == -3 and call(T=129) == -3 and call(keep=0) == -3 and call(keep=65) == -3
    assert call(recent=-1) == -3 and call(recent=51) == -3 and call(Hk=0) == -3 and call(d=80) == -4
    assert call(K=None) == -1 and call(mass=None) == -1 and call(K_out=None) == -1 and call(index=None) == -1
    assert call(V=ODD) == -2 and call(V_out=ODD) == -2 and call(mass=ctypes.c_void_p(4097)) == -2 and call(lens=ctypes.c_void_p(4098)) == -2
    # outputs over inputs: also where only the ends meet
    at, size = 1 << 20, 128 * 2 * 64 * 2
    for out in (at, at + size - 16, at - 64 * 2 * 64 * 2 + 16):
        assert call(K=ctypes.c_void_p(at), K_out=ctypes.c_void_p(out)) == -3 and call(V=ctypes.c_void_p(at), K_out=ctypes.c_void_p(out)) == -3
        assert call(K=ctypes.c_void_p(at), V_out=ctypes.c_void_p(out)) == -3
    for out in (at, at + 2 * 128 * 4 - 4, at - 2 * 64 * 4 + 4):
        assert call(mass=ctypes.c_void_p(at), mass_out=ctypes.c_void_p(out)) == -3


def test_decode_shared_validation():
    lib = binding.load()
    need = moda.moda_decode_shared_workspace_bytes(4, 1000, 8, 2, 128)
    assert need > moda.moda_decode_workspace_bytes(4, 8, 128) and moda.moda_decode_shared_workspace_bytes(4, 0, 8, 2, 128) == moda.moda_decode_workspace_bytes(4, 8, 128)
    assert moda.moda_decode_shared_workspace_bytes(4, -1, 8, 2, 128) == 0 and moda.moda_decode_shared_workspace_bytes(4, 10, 9, 1, 128) == 0

    def call(q=P, Kp=P, K=P, lens=None, depth=P, B=4, Tp=1000, T=10, T_cap=16, H=8, Hk=2, d=128, l=1, scale=0.1, work=P, wb=need):
        return lib.moda_attn_decode_shared(q, Kp, P, K, P, lens, depth, B, Tp, T, T_cap, H, Hk, d, l, F(scale), P, P, work, ctypes.c_size_t(wb), None)

    assert call(B=0) == -3 and call(Tp=-1) == -3 and call(T=-1) == -3 and call(T=17) == -3 and call(Tp=1 << 30) == -3
    assert call(d=100) == -4 and call(l=257) == -5 and call(Hk=3) == -12 and call(scale=float("inf")) == -13
    assert call(q=None) == -1 and call(Kp=None) == -1 and call(K=None) == -1 and call(depth=None) == -1
    assert call(Kp=ODD) == -2 and call(K=ODD) == -2 and call(lens=ctypes.c_void_p(4097)) == -2
    assert call(work=None) == -7 and call(wb=need - 1) == -7


def test_the_binding_refuses_tensors_of_other_shapes_and_types():
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    fp = lambda *s: torch.zeros(s)
    Q, K = bf(1, 4, 4, 64), bf(1, 8, 2, 64)
    with pytest.raises(ValueError):
        moda.moda_attn_key_mass(Q, bf(2, 8, 2, 64), fp(1, 4, 4), 0.1)
    with pytest.raises(ValueError):
        moda.moda_attn_key_mass(Q, K, fp(1, 4, 5), 0.1)
    with pytest.raises(ValueError):
        moda.moda_attn_key_mass(Q, K, fp(1, 4, 4), 0.1, mass=fp(1, 2, 7))
    with pytest.raises(ValueError):
        moda.moda_attn_key_mass(Q, K, fp(1, 4, 4), 0.1)                      # no device tensors
    q = bf(1, 4, 64)
    with pytest.raises(ValueError):
        moda.moda_attn_decode_mass(q, K, K, None, 8, 1, 0.1)
    with pytest.raises(ValueError):
        moda.moda_attn_decode_mass(q, K, K, None, 8, 0, 0.1, seq_lens=torch.zeros(1, dtype=torch.int64))
    with pytest.raises(ValueError):
        moda.moda_attn_decode_mass(q, K, K, None, 8, 0, 0.1, mass_in=fp(1, 2, 9))
    with pytest.raises(ValueError):
        moda.moda_kv_evict(K, K, fp(1, 2, 7), 8, 4)
    with pytest.raises(ValueError):
        moda.moda_kv_evict(K, K, fp(1, 2, 8), 8, 4, index=torch.zeros((1, 2, 5), dtype=torch.int32))
    with pytest.raises(ValueError):
        moda.moda_kv_evict(K, K, fp(1, 2, 8), 8, 4, K_out=bf(1, 4, 2, 128))
    with pytest.raises(ValueError):
        moda.moda_attn_decode_shared(q, bf(5, 2, 128), bf(5, 2, 128), K, K, None, None, 8, 0, 0.1)
    with pytest.raises(ValueError):
        moda.moda_attn_decode_shared(q, bf(5, 4, 64), bf(5, 4, 64), K, K, None, None, 8, 0, 0.1)
    with pytest.raises(ValueError):
        moda.moda_attn_decode_shared(q, bf(5, 2, 64), bf(4, 2, 64), K, K, None, None, 8, 0, 0.1)


def test_every_serving_kernel_that_waits_tears_down_with_the_report():
    # PipeWait is mbar_wait with the CTA's abort word: the same tear-down
    seen = set()
    for f in sorted(os.listdir(build.CSRC)):
        if not f.endswith(".cuh"):
            continue
        for name, body in kernels(source(f)):
            if "PipeWait" not in body:
                continue
            seen.add(name)
            waits = [m.end() for m in re.finditer(r"\bwait\(", body)]
            calls = [m.start() for m in re.finditer(r"\babort_teardown\(", body)]
            assert len(calls) == 1 and calls[0] > max(waits), name
            assert re.search(r"__syncthreads\(\);\s*abort_teardown\(&?\w+, \d+\);\s*__syncthreads\(\);", body), name
            sites = re.findall(r"\bwait\([^;]*, (\d+)\);", body)
            assert len(sites) == len(set(sites)) == len(waits), (name, sites)
    assert seen == {"key_mass_kernel", "shared_prefix_kernel"}, seen
