"""Decode step of a batch over a shared prefix on the GPU, against the fp64 oracle."""
import numpy as np
import pytest
import torch

import paper_2603_15619_b200 as moda
from oracle import moda_oracle as orc

from parity import TOL_LSE_ABS, TOL_O_MAX_ABS, TOL_O_REL_L2, f64, rel_l2

pytestmark = pytest.mark.gpu


def inputs(B, P, T_cap, H, Hk, d, l, seed, grow=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)
    return dict(q=n(B, H, d) * grow, Kp=n(P, Hk, d), Vp=n(P, Hk, d), K=n(B, T_cap, Hk, d), V=n(B, T_cap, Hk, d), depth=n(l, B, Hk, 2, d))


def call(x, lens, T, l, scale, **kw):
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda") if lens is not None else None
    out = moda.moda_attn_decode_shared(x["q"], x["Kp"], x["Vp"], x["K"], x["V"], seq, x["depth"] if l else None, T, l, scale, **kw)
    assert moda.moda_last_status() == 0
    return out


def check(x, lens, T, l, scale):
    O, LSE = call(x, lens, T, l, scale)
    B = x["q"].shape[0]
    kd, vd = (f64(x["depth"][:, :, :, i]) if l else None for i in (0, 1))
    o, lse = orc.decode_shared(f64(x["q"]), f64(x["Kp"]), f64(x["Vp"]), f64(x["K"]), f64(x["V"]), [T] * B if lens is None else lens, kd, vd, scale)
    O, LSE = f64(O), f64(LSE)
    there = np.isfinite(lse)
    assert np.array_equal(there, np.isfinite(LSE)) and (LSE[~there] == -np.inf).all() and (O[~there] == 0).all()
    if there.any():
        assert rel_l2(O, o) <= TOL_O_REL_L2 and np.abs(O - o).max() <= TOL_O_MAX_ABS * max(1.0, np.abs(o).max())
        assert np.abs(LSE[there] - lse[there]).max() <= TOL_LSE_ABS


SHAPES = [
    # B, P, T, T_cap, H, H_kv, d, l
    (1, 1, 1, 1, 1, 1, 64, 0), (1, 1, 0, 1, 2, 1, 128, 3), (2, 127, 5, 8, 4, 2, 64, 2), (3, 128, 64, 64, 6, 2, 128, 1), (5, 129, 65, 100, 3, 1, 64, 0),
    (7, 300, 200, 200, 16, 8, 128, 4), (16, 1000, 30, 32, 8, 1, 64, 5), (17, 1000, 30, 32, 8, 1, 128, 5),           # one row tile, one row more
    (33, 513, 20, 20, 8, 1, 64, 2), (40, 700, 33, 40, 28, 4, 128, 3), (130, 260, 10, 16, 1, 1, 64, 1), (9, 2000, 100, 128, 32, 1, 128, 2),   # G = 7, 1, 32
    (20, 1500, 50, 50, 16, 1, 64, 0), (26, 400, 7, 7, 10, 2, 128, 1), (64, 5000, 12, 16, 16, 2, 128, 2), (3, 9000, 300, 300, 5, 5, 64, 3),
]


@pytest.mark.parametrize("B,P,T,T_cap,H,Hk,d,l", SHAPES)
def test_matches_the_oracle(B, P, T, T_cap, H, Hk, d, l):
    x = inputs(B, P, T_cap, H, Hk, d, l, seed=P + B)
    lens = [T * b // max(B - 1, 1) for b in range(B)]                        # from none to T
    x["K"][:, T:] = float("nan")
    x["V"][:, T:] = float("nan")
    if lens[0] == 0:
        x["K"][0] = float("nan")                                             # a sequence without own keys: nothing of its cache is used
        x["V"][0] = float("nan")
    a = call(x, lens, T, l, d ** -0.5)
    x["K"].nan_to_num_(0.0)
    x["V"].nan_to_num_(0.0)
    b = call(x, lens, T, l, d ** -0.5)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    check(x, lens, T, l, d ** -0.5)
    if T > 0:
        check(x, None, T, l, d ** -0.5)


@pytest.mark.parametrize("d", [64, 128])
def test_without_a_prefix_it_is_the_plain_step(d):
    B, T, H, Hk, l = 6, 400, 8, 2, 4
    x = inputs(B, 0, T, H, Hk, d, l, seed=3)
    O, LSE = call(x, None, T, l, d ** -0.5)
    o, lse = moda.moda_attn_decode(x["q"], x["K"], x["V"], x["depth"], T, l, d ** -0.5)
    assert np.abs(f64(O) - f64(o)).max() <= 2 ** -8 * np.abs(f64(o)).max() and np.abs(f64(LSE) - f64(lse)).max() <= 1e-5
    check(x, [0, 400, 1, 2, 0, 63], T, l, d ** -0.5)


def test_rows_without_any_key():
    x = inputs(4, 0, 8, 4, 2, 64, 0, seed=5)
    check(x, [0, 3, 0, 8], 8, 0, 0.125)
    O, LSE = moda.moda_attn_decode_shared(x["q"], x["Kp"], x["Vp"], None, None, None, None, 0, 0, 0.125)
    assert bool((O == 0).all()) and bool((LSE == -float("inf")).all())


def test_only_a_prefix():
    for d, B, H, Hk in [(64, 3, 4, 2), (128, 50, 8, 1)]:
        x = inputs(B, 777, 1, H, Hk, d, 0, seed=6)
        O, LSE = moda.moda_attn_decode_shared(x["q"], x["Kp"], x["Vp"], None, None, None, None, 0, 0, d ** -0.5)
        o, lse = orc.decode_shared(f64(x["q"]), f64(x["Kp"]), f64(x["Vp"]), f64(x["K"]), f64(x["V"]), [0] * B, None, None, d ** -0.5)
        assert rel_l2(f64(O), o) <= TOL_O_REL_L2 and np.abs(f64(LSE) - lse).max() <= TOL_LSE_ABS


@pytest.mark.parametrize("where", ["first", "last", "rising"])
def test_scores_that_grow_along_the_prefix(where):
    # the running maximum moves late, early, or all the time: the rescaling of what has been summed
    B, P, H, Hk, d, l = 20, 3000, 16, 2, 128, 2
    x = inputs(B, P, 16, H, Hk, d, l, seed=8, grow=2.0)
    at = torch.linspace(0.1, 6.0, P, device="cuda") if where == "rising" else torch.ones(P, device="cuda")
    if where != "rising":
        at[0 if where == "first" else -1] = 20.0
    x["Kp"] = (x["Kp"].float() * at[:, None, None]).to(torch.bfloat16)
    check(x, [16] * B, 16, l, d ** -0.5)


LARGE = [
    # B, P, T, H, H_kv, d: one to many row tiles, teams of heads and of row tiles, side by side and one behind the other
    (4, 30000, 100, 8, 8, 64), (40, 12000, 40, 28, 4, 128), (130, 5000, 30, 16, 4, 64), (96, 2500, 3, 40, 8, 128), (200, 1300, 20, 32, 2, 64), (64, 40000, 10, 16, 2, 128),
    (33, 9000, 600, 12, 6, 128),
]


def check_on_device(x, lens, T, l):
    B, H, d = x["q"].shape
    P, Hk = x["Kp"].shape[:2]
    G = H // Hk
    O, LSE = call(x, lens, T, l, d ** -0.5)
    at = torch.tensor([T] * B if lens is None else lens, device="cuda")
    for k in range(Hk):
        q = x["q"][:, k * G:(k + 1) * G].double()
        s = torch.cat([torch.einsum("bgd,td->bgt", q, x["Kp"][:, k].double()), torch.einsum("bgd,btd->bgt", q, x["K"][:, :T, k].double()),
                       torch.einsum("bgd,lbd->bgl", q, x["depth"][:, :, k, 0].double())], -1) * d ** -0.5
        gone = torch.zeros(s.shape[-1], dtype=torch.bool, device="cuda").repeat(B, 1)
        gone[:, P:P + T] = torch.arange(T, device="cuda") >= at[:, None]
        s.masked_fill_(gone[:, None], -torch.inf)
        p = torch.softmax(s, -1)
        o = (torch.einsum("bgt,td->bgd", p[..., :P], x["Vp"][:, k].double()) + torch.einsum("bgt,btd->bgd", p[..., P:P + T], x["V"][:, :T, k].double()) +
             torch.einsum("bgl,lbd->bgd", p[..., P + T:], x["depth"][:, :, k, 1].double()))
        assert rel_l2(f64(O[:, k * G:(k + 1) * G]), f64(o)) <= TOL_O_REL_L2
        assert np.abs(f64(LSE[:, k * G:(k + 1) * G]) - f64(torch.logsumexp(s, -1))).max() <= TOL_LSE_ABS


@pytest.mark.parametrize("B,P,T,H,Hk,d", LARGE)
def test_large_batches_and_long_prefixes(B, P, T, H, Hk, d):
    x = inputs(B, P, T, H, Hk, d, 2, seed=B)
    check_on_device(x, [(37 * b) % (T + 1) for b in range(B)], T, 2)


NEAR = [
    # B, P, T, H, H_kv, d, l: four, two and one warp a row, with the last CTA full and not; the longest own caches that are read beside the depth pairs
    # and one key more; many depth pairs; no depth pairs; no prefix
    (3, 500, 192, 2, 1, 64, 256), (3, 500, 193, 2, 1, 64, 256), (25, 800, 48, 16, 2, 128, 1), (51, 800, 48, 8, 1, 64, 33), (50, 800, 49, 16, 2, 128, 7),
    (69, 300, 128, 32, 32, 64, 17), (70, 300, 192, 32, 16, 128, 0), (111, 300, 193, 20, 20, 128, 15), (183, 129, 96, 13, 13, 64, 256), (95, 0, 24, 32, 2, 128, 16),
    (95, 0, 25, 32, 1, 64, 9), (200, 64, 1, 12, 4, 128, 0),
]


@pytest.mark.parametrize("B,P,T,H,Hk,d,l", NEAR)
def test_short_own_caches_and_depth_pairs(B, P, T, H, Hk, d, l):
    x = inputs(B, P, T + 3, H, Hk, d, l, seed=T)
    for n in "KV":
        x[n][:, T:] = float("nan")                                           # not read beyond the longest cache
    check_on_device(x, [(31 * b + T) % (T + 1) for b in range(B)], T, l)
    check_on_device(x, None, T, l)


def test_numbers_behind_a_short_cache_are_not_used():
    B, P, T, H, Hk, d, l = 90, 200, 40, 32, 8, 64, 5
    x = inputs(B, P, T, H, Hk, d, l, seed=2)
    lens = [b % (T + 1) for b in range(B)]
    a = call(x, lens, T, l, 0.125)
    for b, n in enumerate(lens):
        x["K"][b, n:] = float("inf")
        x["V"][b, n:] = float("nan")
    c = call(x, lens, T, l, 0.125)
    assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])


def test_a_query_that_is_no_number_has_no_result():
    for B, l in ((3, 0), (3, 2), (20, 0)):
        x = inputs(B, 200, 10, 16, 2, 64, l, seed=3)
        x["q"][1, 5] = float("nan")
        O, LSE = call(x, [10] * B, 10, l, 0.125)
        assert torch.isnan(O[1, 5]).all() and torch.isnan(LSE[1, 5])
        O[1, 5], LSE[1, 5] = 0, 0
        assert torch.isfinite(O.float()).all() and torch.isfinite(LSE).all()


def test_repeatable_on_another_stream_and_guard_bands():
    B, P, T, H, Hk, d, l = 9, 1000, 40, 12, 4, 128, 3
    x = inputs(B, P, T, H, Hk, d, l, seed=9)
    want = call(x, None, T, l, d ** -0.5)
    n, m = B * H * d, B * H
    Ob, Lb = torch.full((n + 128,), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((m + 128,), 7.0, device="cuda")
    work = torch.full((moda.moda_decode_shared_workspace_bytes(B, P, H, Hk, d) + 64,), 7, dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    moda.moda_attn_decode_shared(x["q"], x["Kp"], x["Vp"], x["K"], x["V"], None, x["depth"], T, l, d ** -0.5, O=Ob[64:64 + n].view(B, H, d),
                                 LSE=Lb[64:64 + m].view(B, H), workspace=work[:-64], stream=s)
    s.synchronize()
    assert torch.equal(Ob[64:64 + n].view(B, H, d), want[0]) and torch.equal(Lb[64:64 + m].view(B, H), want[1])
    assert bool((Ob[:64] == 7).all() and (Ob[-64:] == 7).all() and (Lb[:64] == 7).all() and (Lb[-64:] == 7).all() and (work[-64:] == 7).all())
