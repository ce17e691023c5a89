"""An index that is used again: over the end of a block, by another layer's cache, and one that a graph selects anew with every replay."""
import pytest
import torch

import paper_2603_15619_b200 as moda

pytestmark = pytest.mark.gpu


def test_an_index_serves_until_a_sequence_opens_a_block():
    B, H, Hk, d, scale = 2, 4, 2, 64, 0.125
    g = torch.Generator(device="cuda").manual_seed(3)
    new = lambda *n: torch.randn(n, generator=g, device="cuda", dtype=torch.bfloat16)
    layers = [moda.PagedCache(B, Hk, d, num_pages=12, max_len=300) for _ in range(2)]
    K = new(B, 200, Hk, d)
    for c in layers:
        c.write(K, K, n_new=[190, 40])
    q = new(B, H, d)
    index = layers[0].select(q, 2, 1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        anew = layers[0].select(q, 2, 1, longest=300)
    for i in range(5):                                          # positions 190 .. 194: the last three are in a block that the index does not have
        k = new(B, 1, Hk, d) * 0 + 4.0
        for c in layers:
            c.write(k, k)
        graph.replay()
        for c in layers:
            fresh = c.attend(q, None, 0, scale, n_blocks=2, n_recent=1)
            assert all(torch.equal(a, b) for a, b in zip(c.attend(q, None, 0, scale, index=anew), fresh))
            if 190 + i < 192:
                c.attend(q, None, 0, scale, index=index)
            else:
                with pytest.raises(ValueError, match="block"):
                    c.attend(q, None, 0, scale, index=index)
                assert (index[0] != 3).all() and (c.index[0] == 3).any(-1).all()
    assert moda.moda_last_status() == 0
