"""Decode over pages in 8 bits where value rows differ most (rows of zeros, whose scale is 1 by the format, beside small ones, and rows of one feature), or elements of a query."""
import numpy as np
import pytest
import torch

import paper_2603_15619_b200 as moda

import pages_ref as ref

pytestmark = pytest.mark.gpu


def _decode(K, V, q, scale, depth=None, index=None):
    """One sequence with keys K and values V [n,Hk,d]: O, LSE of the call, and the reference with its tolerances; the pages."""
    n, Hk, d = K.shape
    pages, _, table, dev = ref.make(1, n, Hk, d, 64, [n], seed=n)
    pages, _ = ref.write(pages, None, K[None], V[None], table, [0], [n], 64)
    idx = None if index is None else torch.from_numpy(index).cuda()
    O, LSE = moda.moda_attn_decode_e4m3(ref.put(q[None]), torch.from_numpy(pages).cuda(), dev[2], torch.tensor([n], dtype=torch.int32, device="cuda"),
                                        None if depth is None else ref.put(depth), n, 0 if depth is None else len(depth), scale, index=idx)
    assert moda.moda_last_status() == 0
    return O.double().cpu().numpy(), LSE.double().cpu().numpy(), ref.decode(q[None], pages, table, [n], depth, scale, 64, index), (pages, table)


def _check(O, LSE, want, more=0.0):
    o, lse, o_tol, lse_tol = want
    assert (np.abs(O - o) <= o_tol + more).all(), float((np.abs(O - o) / (o_tol + more)).max())
    assert (np.abs(LSE - lse) <= lse_tol).all()


def _keys(rng, n, Hk, H, d, sinks, share):
    """Keys, queries and a scale with which the keys `sinks` of every head have `share` of the weight together (None: all keys are alike)."""
    K, q = rng.standard_normal((n, Hk, d)), rng.standard_normal((H, d))
    K[:, :, 0], q[:, 0] = 0.0, 16.0
    if share is not None:
        # scores of the others are about normal in units of d^-1/2: their weight is that of about n exp(1 / 2)
        gap = np.log(share / (1 - share) * (n - len(sinks)) / len(sinks)) + 0.5
        K[sinks, :, :] = 0.0
        K[sinks, :, 0] = gap * d ** 0.5 / 16
    return ref.bf16(K), ref.bf16(q), d ** -0.5


ZEROS = {                                                       # n, rows of zeros
    "first": (64, [0]), "a_whole_block": (200, range(64, 128)), "earlier_block": (300, [5, 70]), "last_of_a_part": (131, [130]), "most": (150, [i for i in range(150) if i % 17]),
    "two_blocks_and_a_part": (129, range(129)),
}


@pytest.mark.parametrize("d,H,Hk", [(64, 3, 1), (128, 8, 2), (128, 32, 2)])
@pytest.mark.parametrize("size,share", [(1e-8, None), (1e-10, None), (0.05, 0.9999), (1e-6, 0.99), (1.0, None)])
@pytest.mark.parametrize("zeros", ZEROS)
def test_rows_of_zeros_beside_small_ones(zeros, size, share, d, H, Hk):
    # a row of zeros adds nothing to the output, whatever its weight is: the others keep the 2^-11 of theirs
    n, at = ZEROS[zeros][0], list(ZEROS[zeros][1])
    rng = np.random.default_rng(n + d)
    K, q, scale = _keys(rng, n, Hk, H, d, at[:1], share if len(at) < n else None)
    V = rng.standard_normal((n, Hk, d)) * size
    V[at] = 0.0
    V[at[-1], 0, 3] = -0.0
    _check(*_decode(K, ref.bf16(V), q, scale)[:3])


@pytest.mark.parametrize("d", [64, 128])
def test_a_row_of_zeros_in_one_head_alone_and_one_of_scale_1(d):
    # the heads of a position are rows of their own; a row whose largest element is 448 has scale 1 too and counts
    n, H, Hk = 90, 4, 2
    rng = np.random.default_rng(d)
    K, q, scale = _keys(rng, n, Hk, H, d, [], None)
    V = rng.standard_normal((n, Hk, d)) * 1e-9
    V[7, 0] = 0.0
    V[20:, 1] *= 1e9
    V[30, 1] = 0.0
    V[30, 1, d - 1] = 448.0
    V[31, 1] = np.where(np.arange(d) % 2, 448.0, -3.0)
    V[20:, 0] *= 1e3
    O, LSE, want, _ = _decode(K, ref.bf16(V), q, scale)
    _check(O, LSE, want)
    assert (np.abs(O[0, 2:, d - 1]) > 1e-3).all()


def test_rows_of_zeros_among_named_blocks_and_beside_depth_pairs():
    n, H, Hk, d, l = 500, 8, 2, 128, 3
    rng = np.random.default_rng(1)
    K, q, scale = _keys(rng, n, Hk, H, d, [], None)
    V = rng.standard_normal((n, Hk, d)) * 1e-9
    V[[64 * i + 3 * i for i in range(8)]] = 0.0
    depth = rng.standard_normal((l, 1, Hk, 2, d)) * 1e-9
    index = np.array([[[0, 3, 7, -1], [2, 5, 6, 7]]], np.int32)
    _check(*_decode(K, ref.bf16(V), q, scale, index=index)[:3])
    _check(*_decode(K, ref.bf16(V), q, scale, depth=ref.bf16(depth), index=index)[:3])


def _weights_left(q, pages, table, n, scale, d, Hk):
    """What the weights' f16 leaves of those that it holds with fewer bits, per element of O: half a step of 2^-24 of each, where the largest weight times scale, W, is held
    as 2^14 or more: 2^-25 2^-14 W |code|."""
    H = q.shape[0]
    out = np.zeros((1, H, d))
    for k in range(Hk):
        K, V = ref.gather(pages, table, 0, k, n, 64, d)
        s_v = np.array([ref.split(np.ascontiguousarray(pages[table[0, j // 64], 0, k]), d)[3][j % 64] for j in range(n)], np.float64)
        for h in range(k * (H // Hk), (k + 1) * (H // Hk)):
            s = K @ q[h].astype(np.float64) * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            W = (p * s_v * (V != 0).any(-1)).max()
            out[0, h] = 2.0 ** -39 * W * (np.abs(V) / s_v[:, None]).sum(0)
    return out


@pytest.mark.parametrize("power", [0, 10, 24, 32, 60])
@pytest.mark.parametrize("d", [64, 128])
def test_a_row_of_one_feature_far_above_the_others(d, power):
    # its weight times its scale is the largest; what is left of the others' in the features where it has codes 0 is what the header states
    n, H, Hk = 100, 4, 2
    rng = np.random.default_rng(power)
    K, q, scale = _keys(rng, n, Hk, H, d, [], None)
    V = rng.standard_normal((n, Hk, d))
    V[40] = 0.0
    V[40, :, 5] = 2.0 ** power
    O, LSE, want, (pages, table) = _decode(K, ref.bf16(V), q, scale)
    left = _weights_left(q, pages, table, n, scale, d, Hk)
    _check(O, LSE, want, left)
    # the scales are 2^power / 448 and about 2 / 448, no weight is 2^16 below another: to 2^10 all are above 2^-28 of the largest and keep 2^-11
    if power <= 10:
        _check(O, LSE, want)


@pytest.mark.parametrize("below", [20, 31, 33, 34])
@pytest.mark.parametrize("d", [64, 128])
def test_a_query_of_elements_of_very_different_sizes(d, below):
    # the largest element of the query meets codes that are 0: the scores are those of elements 2^-below of it.  To 2^-31 they are exact, below they are off by half a step of
    # f16 below its smallest normal number, 2^-25 where the largest is 2^14 or more: 2^-39 of the largest
    n, H, Hk = 150, 8, 2
    rng = np.random.default_rng(below)
    K, V, q = rng.standard_normal((n, Hk, d)), rng.standard_normal((n, Hk, d)), rng.uniform(1.0, 2.0, (H, d)) * rng.choice([-1, 1], (H, d)) * 2.0 ** -below
    K[:, :, 9], q[:, 9] = 0.0, 1.5
    q, scale = ref.bf16(q), 2.0 ** below * d ** -0.5 * 0.5
    O, LSE, (o, lse, o_tol, lse_tol), (pages, table) = _decode(ref.bf16(K), ref.bf16(V), q, scale)
    if below > 31:
        for k in range(Hk):
            keys, values = ref.gather(pages, table, 0, k, n, 64, d)
            ds = 1.5 * 2.0 ** -39 * np.abs(keys).sum(1).max() * scale          # of a score: all of its elements off by half a step
            for h in range(k * (H // Hk), (k + 1) * (H // Hk)):
                s = keys @ q[h].astype(np.float64) * scale
                p = np.exp(s - lse[0, h])
                lse_tol[0, h] += ds
                o_tol[0, h] += np.expm1(2 * ds) * (p @ np.abs(values)) * 1.01      # a weight is off by a factor of exp(ds), the sum by as much; 1.01: their rounding on top
    _check(O, LSE, (o, lse, o_tol, lse_tol))
