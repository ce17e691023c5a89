"""Several continuations of one long prompt, then one long generation, with a sequence cache of bounded length: one layer, synthetic data.

    python examples/continue_prompt.py

1. The prompt's forward (its depth slots as a stack of layers left them).
2. Its cache is cut to the keys that its last rows used most; all continuations share what stays.
3. Every continuation decodes on the shared prefix with a cache of its own.
4. One continuation goes on in a bounded cache that is cut whenever it is full.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2603_15619_b200 as moda  # noqa: E402


def main(T=8192, B=16, H=16, H_kv=8, d=128, l=8, keep=1024, recent=128, window=64, steps=48, capacity=1152):
    g = torch.Generator(device="cuda").manual_seed(0)
    new = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)
    scale = d ** -0.5
    token = lambda n: (new(n, H, d), new(n, H_kv, d), new(n, H_kv, d), new(l, n, H_kv, 2, d))

    # 1. the prompt
    Q, K, V = new(1, T, H, d), new(1, T, H_kv, d), new(1, T, H_kv, d)
    depth = moda.alloc_depth_cache(1, T, H_kv, d, l)
    for i in range(l):
        moda.moda_depth_cache_append(depth, i, new(1, T, H_kv, d), new(1, T, H_kv, d))
    O, LSE = moda.moda_attn_fwd_gqa(Q, K, V, depth, l, scale)

    # 2. the keys that stay: rated by the last rows of the prompt
    last = Q[:, -window:].contiguous(), LSE[:, :, -window:].contiguous()
    K_prefix, V_prefix, index = moda.cut_prompt(K, V, *last, scale, keep, recent)
    weight = moda.moda_attn_key_mass(last[0], K, last[1], scale)
    kept = weight[0].gather(1, index.long()).sum() / weight.sum()
    print(f"prompt of {T} keys cut to {K_prefix.shape[0]}: they hold {100 * float(kept):.1f} % of the weight of its last {window} rows")

    # 3. continuations on the shared prefix
    own_K, own_V = torch.zeros((B, steps, H_kv, d), device="cuda", dtype=torch.bfloat16), torch.zeros((B, steps, H_kv, d), device="cuda", dtype=torch.bfloat16)
    lens = torch.zeros((B,), device="cuda", dtype=torch.int32)
    work = torch.empty((moda.moda_decode_shared_workspace_bytes(B, K_prefix.shape[0], H, H_kv, d),), device="cuda", dtype=torch.uint8)
    for t in range(steps):
        q, k, v, pairs = token(B)
        own_K[:, t], own_V[:, t] = k, v
        lens += 1
        O, LSE = moda.moda_attn_decode_shared(q, K_prefix, V_prefix, own_K, own_V, lens, pairs, t + 1, l, scale, workspace=work)
    print(f"{B} continuations of {steps} tokens: output norm {float(O.float().norm()):.3f}, LSE {float(LSE.mean()):.3f}")

    # 4. one of them in a bounded cache
    cache = moda.BoundedCache(1, H_kv, d, capacity, keep, recent)
    cache.load(K, V, *last, scale)
    cuts = 0
    for t in range(4 * (capacity - keep)):
        q, k, v, pairs = token(1)
        before = cache.longest
        cache.append(k, v)
        cuts += cache.longest <= before
        O, LSE = cache.attend(q, pairs, l, scale)
    assert moda.moda_last_status() == 0
    print(f"{4 * (capacity - keep)} more tokens in a cache of {capacity}: cut {cuts} times, {int(cache.lens[0])} keys now, LSE {float(LSE.mean()):.3f}")
    return O


if __name__ == "__main__":
    main()
