"""Pins of the oracle's serving functions: the attention weight of the sequence keys (a library softmax's probabilities, conservation,
equal scores), the keys that an eviction keeps (brute force over subsets, ties, NaN), the decode step over a shared prefix (a library softmax
over the concatenated keys, the plain decode step, empty rows)."""
import itertools

import numpy as np
import pytest
import torch

from oracle import moda_oracle as orc


@pytest.mark.parametrize("T_q,T_kv", [(6, 6), (1, 5), (3, 8)])
def test_key_mass_is_the_column_sum_of_a_library_softmax(T_q, T_kv):
    rng = np.random.default_rng(0)
    B, Hq, Hk, d, l, scale = 2, 4, 2, 3, 2, 0.4
    Q, K, V = rng.standard_normal((B, T_q, Hq, d)), rng.standard_normal((B, T_kv, Hk, d)), rng.standard_normal((B, T_kv, Hk, d))
    Kd, Vd = rng.standard_normal((l, B, T_q, Hk, d)), rng.standard_normal((l, B, T_q, Hk, d))
    _, LSE = orc.forward_prefill_gqa(Q, K, V, Kd, Vd, scale)
    mass = orc.key_mass(Q, K, LSE, scale)
    want = np.zeros((B, Hk, T_kv))
    depth = 0.0
    for h in range(Hq):
        s = torch.einsum("bid,bjd->bij", torch.tensor(Q[:, :, h]), torch.tensor(K[:, :, h // 2])) * scale
        s = s.masked_fill(torch.arange(T_kv) > torch.arange(T_q)[:, None] + T_kv - T_q, -torch.inf)
        u = torch.einsum("bid,lbid->bil", torch.tensor(Q[:, :, h]), torch.tensor(Kd[:, :, :, h // 2])) * scale
        p = torch.softmax(torch.cat([s, u], -1), -1)
        want[:, h // 2] += p[:, :, :T_kv].sum(1).numpy()
        depth += float(p[:, :, T_kv:].sum())
    assert np.allclose(mass, want, rtol=1e-12)
    assert np.isclose(mass.sum() + depth, B * Hq * T_q, rtol=1e-12)


def test_key_mass_of_equal_scores_and_of_rows_without_keys():
    B, T, H, d = 1, 7, 2, 4
    Q, K = np.zeros((B, T, H, d)), np.ones((B, T, 1, d))
    LSE = np.broadcast_to(np.log(np.arange(1, T + 1)), (B, H, T)).copy()
    mass = orc.key_mass(Q, K, LSE, 1.0)
    harmonic = np.array([sum(1 / (i + 1) for i in range(j, T)) for j in range(T)])
    assert np.allclose(mass[0, 0], 2 * harmonic, rtol=1e-13)
    LSE[0, 1] = -np.inf
    assert np.allclose(orc.key_mass(Q, K, LSE, 1.0)[0, 0], harmonic, rtol=1e-13)


def test_kept_positions_by_brute_force_over_subsets():
    rng = np.random.default_rng(3)
    for n, n_keep, n_recent in [(1, 1, 0), (5, 2, 1), (7, 4, 0), (7, 4, 4), (6, 9, 2), (8, 5, 3)]:
        mass = rng.integers(0, 4, n).astype(float)                           # many ties
        got = orc.kept_positions(mass, n_keep, n_recent)
        kept = min(n_keep, n)
        recent = min(n_recent, kept)
        old = n - recent
        # the largest sum; of several such subsets the first in lexicographic order is the one with the lower positions
        best = max(itertools.combinations(range(old), kept - recent), key=lambda c: (sum(mass[list(c)]), [-j for j in c]))
        assert got == list(best) + list(range(old, n))
    assert orc.kept_positions([np.nan, 1.0, np.nan, 0.0, np.inf, -np.inf], 4, 0) == [1, 3, 4, 5]
    assert orc.kept_positions([np.nan, -np.inf, np.nan], 2, 0) == [0, 1]


def test_decode_shared_is_a_library_softmax_over_all_keys():
    rng = np.random.default_rng(5)
    B, Hq, Hk, d, P, T, l, scale = 4, 4, 2, 3, 5, 3, 2, 0.7
    q, Kp, Vp = rng.standard_normal((B, Hq, d)), rng.standard_normal((P, Hk, d)), rng.standard_normal((P, Hk, d))
    K, V = rng.standard_normal((B, T, Hk, d)), rng.standard_normal((B, T, Hk, d))
    kd, vd = rng.standard_normal((l, B, Hk, d)), rng.standard_normal((l, B, Hk, d))
    lens = [0, 1, 3, 2]
    o, lse = orc.decode_shared(q, Kp, Vp, K, V, lens, kd, vd, scale)
    for b in range(B):
        for h in range(Hq):
            k = torch.tensor(np.concatenate([Kp[:, h // 2], K[b, :lens[b], h // 2], kd[:, b, h // 2]]))
            v = torch.tensor(np.concatenate([Vp[:, h // 2], V[b, :lens[b], h // 2], vd[:, b, h // 2]]))
            s = k @ torch.tensor(q[b, h]) * scale
            assert np.allclose(o[b, h], (torch.softmax(s, 0) @ v).numpy(), rtol=1e-12)
            assert np.isclose(lse[b, h], float(torch.logsumexp(s, 0)), rtol=1e-12)


def test_decode_shared_edges():
    rng = np.random.default_rng(6)
    B, Hq, Hk, d, T, l = 2, 2, 1, 3, 4, 3
    q, K, V = rng.standard_normal((B, Hq, d)), rng.standard_normal((B, T, Hk, d)), rng.standard_normal((B, T, Hk, d))
    kd, vd = rng.standard_normal((l, B, Hk, d)), rng.standard_normal((l, B, Hk, d))
    none = np.zeros((0, Hk, d))
    # no prefix: the plain decode step; the same keys as prefix and as own keys give the same
    a = orc.decode_shared(q, none, none, K, V, [T, T], kd, vd, 0.5)
    for x, y in zip(a, orc.decode_gqa(q, K, V, kd, vd, 0.5)):
        assert np.array_equal(x, y)
    same = np.repeat(K[:1], B, 0), np.repeat(V[:1], B, 0)
    for x, y in zip(orc.decode_shared(q, K[0], V[0], K, V, [0, 0], kd, vd, 0.5), orc.decode_gqa(q, *same, kd, vd, 0.5)):
        assert np.allclose(x, y, rtol=1e-13)
    # depth pairs alone, and no key at all
    o, lse = orc.decode_shared(q, none, none, K, V, [0, 0], kd, vd, 0.5)
    s = np.einsum("bhd,lbd->bhl", q, kd[:, :, 0]) * 0.5
    assert np.allclose(lse, np.log(np.exp(s).sum(-1)), rtol=1e-12)
    o, lse = orc.decode_shared(q, none, none, K, V, [0, 2], None, None, 0.5)
    assert (o[0] == 0).all() and (lse[0] == -np.inf).all() and np.isfinite(lse[1]).all()
