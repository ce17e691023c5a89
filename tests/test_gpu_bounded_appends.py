"""A bounded cache whose tokens are not all attended: a key starts from no weight, whatever its place in the buffers held before."""
import pytest
import torch

import paper_2603_15619_b200 as moda
from oracle import moda_oracle as orc

from parity import f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,Hk", [(2, 2), (40, 9)])
def test_tokens_that_are_not_attended(B, Hk):
    # cuts with keys among them whose token had no step of its own; with 360 heads a cut has more CTAs than fit at once
    H, d, scale, T = 2 * Hk, 64, 0.125, 60
    g = torch.Generator(device="cuda").manual_seed(B)
    n = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)
    Q, K, V = n(B, T, H, d), n(B, T, Hk, d), n(B, T, Hk, d)
    _, LSE = moda.moda_attn_fwd_gqa(Q, K, V, None, 0, scale)
    cache = moda.BoundedCache(B, Hk, d, capacity=48, keep=40, recent=4)
    cache.load(K, V, Q, LSE, scale)
    assert bool((cache.mass[:, :, 40:] == 0).all())
    cache.load(K, V, Q, LSE, scale)                                          # the other set of buffers
    assert bool((cache.mass[:, :, 40:] == 0).all())
    for step in range(40):
        before, full = cache.mass.clone(), cache.longest == cache.capacity
        length = cache.longest
        k = n(B, Hk, d)
        cache.append(k, k)
        if full:
            for b in (0, B - 1):
                for h in (0, Hk - 1):
                    at = orc.kept_positions(f64(before)[b, h, :length], 40, 4)
                    assert cache.index[b, h].tolist() == at
                    assert torch.equal(cache.mass[b, h, :40], before[b, h, at])
            before, length = cache.mass.clone(), 40
        assert cache.longest == length + 1 and cache.lens.tolist() == [length + 1] * B
        assert bool((cache.mass[:, :, length:] == 0).all()) and torch.equal(cache.mass[:, :, :length], before[:, :, :length])
        assert torch.equal(cache.K[:, length], k)
        if step % 3 == 2:                                                    # of three tokens two are given, the third is asked for
            q = n(B, H, d)
            before = cache.mass.clone()
            _, lse = cache.attend(q, None, 0, scale)
            # a step's weights: of the same exponential in 64 bits, off by 1e-4 of themselves at most
            s = torch.einsum("bkgd,btkd->bkgt", q.double().view(B, Hk, 2, d), cache.K[:, :length + 1].double()) * scale
            want = torch.softmax(s, -1).sum(2)
            assert torch.allclose(cache.mass[:, :, :length + 1].double(), before[:, :, :length + 1].double() + want, rtol=1e-4, atol=1e-6)
    assert moda.moda_last_status() == 0
