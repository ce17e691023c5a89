"""The calls over the paged cache in 8 bits as they are used together."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import paper_2603_15619_b200 as moda

import pages_ref as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("H,Hk,d,page", [(8, 2, 128, 64), (3, 3, 64, 128)])
def test_prompt_tokens_release_and_reuse(H, Hk, d, page):
    B, l, scale = 3, 2, d ** -0.5
    rng = np.random.default_rng(d)
    cache = moda.PagedCache(B, Hk, d, num_pages=12, max_len=400, page_size=page)
    pages, bounds = (np.zeros(x.shape, np.uint8) for x in (cache.pages, cache.bounds))
    cache.pages.zero_()
    cache.bounds.zero_()
    lengths = [0] * B

    def write(T, n_new):
        K, V = (ref.bf16(rng.standard_normal((B, T, Hk, d))) for _ in range(2))
        cache.write(ref.put(K), ref.put(V), n_new=None if n_new is None else n_new)
        n = [T] * B if n_new is None else n_new
        nonlocal pages, bounds
        pages, bounds = ref.write(pages, bounds, K, V, cache.table.cpu().numpy(), lengths, n, page)
        for b in range(B):
            lengths[b] += n[b]
        assert cache.lengths == lengths and cache.lens.tolist() == lengths
        assert np.array_equal(cache.pages.cpu().numpy(), pages)
        assert np.array_equal(cache.bounds.cpu().numpy()[..., :2 * d + 4], bounds[..., :2 * d + 4])

    def step(**kw):
        q = ref.bf16(rng.standard_normal((B, H, d)))
        depth = ref.bf16(rng.standard_normal((l, B, Hk, 2, d)))
        O, LSE = cache.attend(ref.put(q), ref.put(depth), l, scale, **kw)
        table, index = cache.table.cpu().numpy(), None
        if kw:
            index = ref.select(q, bounds, table, lengths, page, kw["n_blocks"], kw["n_recent"])
            assert np.array_equal(cache.index.cpu().numpy(), index)
        o, lse, o_tol, lse_tol = ref.decode(q, pages, table, lengths, depth, scale, page, index)
        assert (np.abs(O.double().cpu().numpy() - o) <= o_tol).all() and (np.abs(LSE.double().cpu().numpy() - lse) <= lse_tol).all()

    write(200, [200, 77, 0])
    step()
    for _ in range(3):
        write(1, None)
        step()
        step(n_blocks=2, n_recent=1)
    K, V = cache.read()
    table = cache.table.cpu().numpy()
    for b in range(B):
        for k in range(Hk):
            for got, want in zip((K, V), ref.gather(pages, table, b, k, lengths[b], page, d)):
                assert np.array_equal(got[b, :lengths[b], k].float().cpu().numpy(), ref.bf16(want.astype(np.float32)))
        assert not K[b, lengths[b]:].any() and not V[b, lengths[b]:].any()
    cache.release(0)
    lengths[0] = 0
    step()
    write(130, [130, 0, 130])
    step()
    step(n_blocks=3, n_recent=0)
    assert moda.moda_last_status() == 0


def test_a_captured_step_takes_the_lengths_of_its_replay():
    B, H, Hk, d, l, scale = 2, 8, 2, 128, 2, 0.1
    g = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *n: torch.randn(n, generator=g, device="cuda", dtype=torch.bfloat16)
    cache = moda.PagedCache(B, Hk, d, num_pages=20, max_len=600)
    cache.write(new(B, 190, Hk, d), new(B, 190, Hk, d), n_new=[190, 40])
    q, depth = new(B, H, d), new(l, B, Hk, 2, d)

    def step(**kw):
        return (*cache.attend(q, depth, l, scale, **kw), *cache.attend(q, depth, l, scale, n_blocks=3, n_recent=1, **kw), cache.index)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(longest=cache.max_len)
    for T in (1, 130, 64):
        cache.write(new(B, T, Hk, d), new(B, T, Hk, d))
        q.copy_(new(B, H, d))
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, step()))
    cache.release(0)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(got, step())) and torch.isfinite(got[1][1]).all() and (got[0][0] != 0).any()


def test_example_runs():
    spec = importlib.util.spec_from_file_location("paged_cache_example", os.path.join(ROOT, "examples", "paged_cache.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    O = module.main(B=2, T=300, chunk=64, H=4, H_kv=2, l=2, steps=2, n_blocks=3)
    assert torch.isfinite(O).all()
