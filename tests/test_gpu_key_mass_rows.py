"""Key weights with rows that saw no key (LSE -inf): nothing of such a row reaches a key, whatever its query holds (padding of a batch, say)."""
import numpy as np
import pytest
import torch

import paper_2603_15619_b200 as moda
from oracle import moda_oracle as orc

from parity import f64

pytestmark = pytest.mark.gpu
# as for finite queries: the exponent is off by less than 1e-5, its exponential by 2^-22, the sum in short chains by less than 1e-5
RTOL, ATOL = 1e-4, 1e-7

CASES = [
    # B, T_q, T_kv, H, H_kv, d: one row, few units a tile and many of them, groups that do not fill a unit, several tiles and heads
    (1, 1, 1, 1, 1, 64), (2, 1, 300, 4, 4, 128), (1, 40, 300, 8, 2, 128), (2, 64, 1500, 16, 4, 128), (2, 130, 700, 6, 2, 64), (1, 257, 513, 5, 1, 128),
    (1, 700, 1300, 3, 3, 64), (3, 385, 385, 24, 8, 64), (1, 600, 900, 12, 4, 128), (1, 50, 200, 32, 1, 64), (1, 1100, 1100, 7, 1, 128),
]


@pytest.mark.parametrize("which", ["one", "some", "first_half", "all"])
@pytest.mark.parametrize("B,T_q,T_kv,H,Hk,d", CASES)
def test_rows_that_saw_no_key(B, T_q, T_kv, H, Hk, d, which):
    g = torch.Generator(device="cuda").manual_seed(T_q)
    n = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)
    Q, K, V = n(B, T_q, H, d), n(B, T_kv, Hk, d), n(B, T_kv, Hk, d)
    _, LSE = moda.moda_attn_fwd_prefill(Q, K, V, None, 0, d ** -0.5)
    gone = torch.zeros((B, H, T_q), dtype=torch.bool, device="cuda")
    if which == "one":
        gone[B - 1, H // 2, T_q // 2] = True
    elif which == "some":
        gone |= torch.rand((B, H, T_q), generator=g, device="cuda") < 0.2
    elif which == "first_half":
        gone[:, :, :(T_q + 1) // 2] = True
    else:
        gone[:] = True
    LSE.masked_fill_(gone, -torch.inf)
    want = orc.key_mass(f64(Q), f64(K), f64(LSE), d ** -0.5)
    clean = moda.moda_attn_key_mass(Q, K, LSE, d ** -0.5)
    assert np.allclose(f64(clean), want, rtol=RTOL, atol=ATOL)
    rows = gone.transpose(1, 2)                                              # [B, T_q, H]
    for junk in (float("nan"), float("inf"), -3e38):
        Q[rows] = junk
        mass = moda.moda_attn_key_mass(Q, K, LSE, d ** -0.5)
        assert moda.moda_last_status() == 0 and torch.equal(mass, clean)
    if which == "one" and T_q > 1:                                           # a query that is no number in a row that did see keys still shows
        b, h, i = B - 1, 0, T_q - 1
        Q[b, i, h] = float("nan")
        mass = moda.moda_attn_key_mass(Q, K, LSE, d ** -0.5)
        assert bool(torch.isnan(mass[b, 0]).all()) and torch.equal(mass[:b], clean[:b])
