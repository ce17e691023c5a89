"""The bounded sequence cache and the shared, cut prompt as a program uses them, on the GPU against the fp64 oracle."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import paper_2603_15619_b200 as moda
from oracle import moda_oracle as orc

from parity import TOL_LSE_ABS, TOL_O_MAX_ABS, TOL_O_REL_L2, build_cache, f64, rel_l2

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_limits_are_checked():
    for bad in [dict(capacity=8, keep=8), dict(capacity=8, keep=4, recent=5), dict(capacity=8, keep=4, recent=-1)]:
        with pytest.raises(ValueError):
            moda.BoundedCache(1, 1, 64, device="cpu", **bad)
    with pytest.raises(ValueError):
        moda.BoundedCache(1, 1, 64, 8, 4, device="cpu").attend(None, None, 0, 0.1)
    x = torch.zeros((2, 4, 1, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        moda.cut_prompt(x, x, x, x, 0.1, 2)


@pytest.mark.gpu
def test_every_step_is_the_operator_over_the_keys_that_stay():
    B, H, Hk, d, l, T, scale = 2, 4, 2, 64, 2, 150, 0.125
    g = torch.Generator(device="cuda").manual_seed(4)
    n = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)
    Q, K, V, Kd, Vd = n(B, T, H, d), n(B, T, Hk, d), n(B, T, Hk, d), n(l, B, T, Hk, d), n(l, B, T, Hk, d)
    _, LSE = moda.moda_attn_fwd_gqa(Q, K, V, build_cache(Kd, Vd), l, scale)
    cache = moda.BoundedCache(B, Hk, d, capacity=48, keep=40, recent=8)
    cache.load(K, V, Q, LSE, scale)
    # the same by the definitions: keys, values and weights per (sequence, head)
    mass = orc.key_mass(f64(Q), f64(K), f64(LSE), scale)
    sets = {}
    for b in range(B):
        for h in range(Hk):
            at = orc.kept_positions(mass[b, h], 40, 8)
            sets[b, h] = [f64(K)[b, at, h], f64(V)[b, at, h], mass[b, h, at]]
    for step in range(30):
        q, k, v, pairs = n(B, H, d), n(B, Hk, d), n(B, Hk, d), n(l, B, Hk, 2, d)
        full = cache.longest == cache.capacity
        cache.append(k, v)
        O, lse = cache.attend(q, pairs, l, scale)
        for b in range(B):
            for h in range(Hk):
                ks, vs, ms = sets[b, h]
                if full:
                    at = orc.kept_positions(ms, 40, 8)
                    ks, vs, ms = ks[at], vs[at], ms[at]
                ks, vs, ms = np.concatenate([ks, f64(k)[b, h:h + 1]]), np.concatenate([vs, f64(v)[b, h:h + 1]]), np.append(ms, 0.0)
                qs = f64(q)[b:b + 1, h * 2:h * 2 + 2]
                o_ref, lse_ref = orc.decode_gqa(qs, ks[None, :, None], vs[None, :, None], f64(pairs)[:, b:b + 1, h:h + 1, 0], f64(pairs)[:, b:b + 1, h:h + 1, 1], scale)
                got = f64(O)[b:b + 1, h * 2:h * 2 + 2]
                assert rel_l2(got, o_ref) <= TOL_O_REL_L2 and np.abs(got - o_ref).max() <= TOL_O_MAX_ABS
                assert np.abs(f64(lse)[b:b + 1, h * 2:h * 2 + 2] - lse_ref).max() <= TOL_LSE_ABS
                ms = ms + orc.key_mass(qs[:, None], ks[None, :, None], lse_ref[:, :, None], scale)[0, 0]
                assert int(cache.lens[b]) == len(ms)
                # a step adds weights that are off by 1e-4 of themselves at most
                assert np.allclose(f64(cache.mass)[b, h, :len(ms)], ms, rtol=1e-4, atol=1e-6 * (step + 2))
                sets[b, h] = [ks, vs, ms]
    assert moda.moda_last_status() == 0


@pytest.mark.gpu
def test_the_example_runs():
    spec = importlib.util.spec_from_file_location("continue_prompt", os.path.join(ROOT, "examples", "continue_prompt.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    O = m.main(T=700, B=5, H=4, H_kv=2, d=64, l=3, keep=100, recent=10, window=20, steps=7, capacity=110)
    assert torch.isfinite(O.float()).all()
