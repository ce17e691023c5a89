"""A batch of prompts of different lengths, taken in two chunks, then decoded from a paged cache in 8 bits, over all positions and over selected blocks: one layer, synthetic data.

    python examples/paged_cache.py

1. The first chunk of every prompt: its forward, and its keys and values written into the pages.
2. The second chunk, behind the first one read back from the pages.
3. Tokens, each attending to every position of its sequence.
4. Tokens that attend to a few blocks of it, and what that leaves out.
5. A sequence ends; a new one takes its place and its pages.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2603_15619_b200 as moda  # noqa: E402


def main(B=4, T=4096, chunk=512, H=16, H_kv=8, d=128, l=8, steps=16, n_blocks=16, n_recent=2):
    g = torch.Generator(device="cuda").manual_seed(0)
    new = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)
    scale = d ** -0.5
    cache = moda.PagedCache(B, H_kv, d, num_pages=B * -(-(T + chunk + 2 * steps) // 64), max_len=T + chunk + 2 * steps)

    # 1. the first chunk
    K, V = new(B, T, H_kv, d), new(B, T, H_kv, d)
    lengths = [T - 64 * b - b for b in range(B)]
    cache.write(K, V, n_new=lengths)
    print(f"{sum(lengths)} positions in {cache.pages.shape[0] - cache.free_pages} pages: {cache.pages.nbytes / 2 ** 20:.0f} MB, as bf16 {2 * K.nbytes / 2 ** 20:.0f} MB")

    # 2. the second chunk of each, behind the first
    depth = moda.alloc_depth_cache(1, chunk, H_kv, d, l)
    for b in range(B):
        for i in range(l):
            moda.moda_depth_cache_append(depth, i, new(1, chunk, H_kv, d), new(1, chunk, H_kv, d))
        Q, k, v = new(1, chunk, H, d), new(1, chunk, H_kv, d), new(1, chunk, H_kv, d)
        had = moda.moda_kv_read_e4m3(cache.pages, cache.table[b:b + 1], cache.lens[b:b + 1], lengths[b])
        O, LSE = moda.moda_attn_fwd_prefill(Q, torch.cat([had[0], k], 1), torch.cat([had[1], v], 1), depth, l, scale)
        rows, counts = torch.zeros((B, chunk, H_kv, d), device="cuda", dtype=torch.bfloat16), [chunk * (i == b) for i in range(B)]
        vals = rows.clone()
        rows[b], vals[b] = k[0], v[0]
        cache.write(rows, vals, n_new=counts)
    print(f"second chunks: output norm {float(O.float().norm()):.2f}, lengths {cache.lengths}")

    # 3. and 4. tokens
    token = lambda: (new(B, H, d), new(B, 1, H_kv, d), new(B, 1, H_kv, d), new(l, B, H_kv, 2, d))
    for _ in range(steps):
        q, k, v, pairs = token()
        cache.write(k, v)
        O, LSE = cache.attend(q, pairs, l, scale)
    print(f"{steps} tokens over every position: LSE {float(LSE.mean()):.3f}")
    for _ in range(steps):
        q, k, v, pairs = token()
        cache.write(k, v)
        whole, lse = cache.attend(q, pairs, l, scale)
        O, LSE = cache.attend(q, pairs, l, scale, n_blocks=n_blocks, n_recent=n_recent)
    kept = float((LSE - lse).exp().mean())
    print(f"{steps} tokens over {n_blocks} of {-(-cache.longest // 64)} blocks: they hold {100 * kept:.1f} % of the weight of all")

    # 5. a place is taken over
    cache.release(1)
    k, v = new(B, 100, H_kv, d), new(B, 100, H_kv, d)
    cache.write(k, v, n_new=[100 * (b == 1) for b in range(B)])
    O, LSE = cache.attend(q, pairs, l, scale)
    assert moda.moda_last_status() == 0
    print(f"a new sequence of 100 positions beside the others: lengths {cache.lengths}, LSE {[round(float(x), 2) for x in LSE.mean(1)]}")
    return O


if __name__ == "__main__":
    main()
