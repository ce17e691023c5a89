"""A bounded cache that several queries in turn attend to: the newest key keeps what the queries before gave to it."""
import pytest
import torch

import paper_2603_15619_b200 as moda

pytestmark = pytest.mark.gpu


def test_every_query_adds_to_every_key():
    B, H, Hk, d, T, scale = 3, 8, 2, 64, 50, 0.125
    g = torch.Generator(device="cuda").manual_seed(2)
    n = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)
    Q, K, V = n(B, T, H, d), n(B, T, Hk, d), n(B, T, Hk, d)
    _, LSE = moda.moda_attn_fwd_gqa(Q, K, V, None, 0, scale)
    cache = moda.BoundedCache(B, Hk, d, capacity=48, keep=40, recent=4)
    cache.load(K, V, Q, LSE, scale)

    def attend():
        q, length = n(B, H, d), cache.longest
        before = cache.mass[:, :, :length].double()
        cache.attend(q, None, 0, scale)
        s = torch.einsum("bkgd,btkd->bkgt", q.double().view(B, Hk, H // Hk, d), cache.K[:, :length].double()) * scale
        want = before + torch.softmax(s, -1).sum(2)
        # a step's weights are off by 1e-4 of themselves at most
        assert torch.allclose(cache.mass[:, :, :length].double(), want, rtol=1e-4, atol=1e-6)

    attend()                                                                 # another query of the prompt, before any token
    attend()
    for _ in range(12):                                                      # over a cut
        cache.append(n(B, Hk, d), n(B, Hk, d))
        attend()
        attend()
        attend()
    assert moda.moda_last_status() == 0
