"""A sequence cache of bounded length for serving: the keys that the queries use most, and the most recent ones, stay.

The mechanisms are the library's: ``moda_attn_key_mass`` rates a prompt's keys by the attention weight that its rows gave to them,
``moda_attn_decode_mass`` adds every token's weights, ``moda_kv_evict`` cuts the cache when it is full.  This class keeps the buffers and
the lengths.  Attention does not depend on the order of the keys; positional information has to be in them.

    cache = BoundedCache(B, H_kv, d, capacity=4096, keep=3072, recent=512)
    cache.load(K, V, Q, LSE, scale)                      # after the prompt's forward: cut to `keep` if it is longer
    for token in ...:
        cache.append(k, v)                               # the token's own key and value
        O, LSE = cache.attend(q, depth_kv_token, l, scale)

``cut_prompt`` cuts one prompt to a prefix that several continuations share (``moda_attn_decode_shared``).
"""
from __future__ import annotations

import torch

from . import binding


class BoundedCache:
    def __init__(self, B: int, H_kv: int, d: int, capacity: int, keep: int, recent: int = 0, device="cuda"):
        if not 0 <= recent <= keep < capacity:
            raise ValueError("0 <= recent <= keep < capacity required")
        self.B, self.H_kv, self.d, self.capacity, self.keep, self.recent = B, H_kv, d, capacity, keep, recent
        bf = dict(device=device, dtype=torch.bfloat16)
        # two sets of buffers: a cut writes from one into the other
        self._sets = [(torch.empty((B, capacity, H_kv, d), **bf), torch.empty((B, capacity, H_kv, d), **bf),
                       torch.zeros((B, H_kv, capacity), device=device)) for _ in range(2)]
        self.index = torch.empty((B, H_kv, keep), device=device, dtype=torch.int32)    # of the last cut: where its keys were
        self.lens = torch.zeros((B,), device=device, dtype=torch.int32)
        self.longest = 0                                       # no length is above this (known without asking the device)
        self._rows = torch.arange(B, device=device)
        self._attended = False                                 # the newest key has taken part in a step

    @property
    def K(self):
        return self._sets[0][0]

    @property
    def V(self):
        return self._sets[0][1]

    @property
    def mass(self):
        """Accumulated weights [B, H_kv, capacity] of a sequence's first ``lens`` keys; 0 behind them."""
        return self._sets[0][2]

    def _cut_into(self, K, V, mass, longest, lens):
        Ko, Vo, mo = self._sets[1]
        mo.zero_()                                             # behind the keys that stay it holds weights of an earlier cut: a new key has none
        binding.moda_kv_evict(K, V, mass, longest, self.keep, self.recent, seq_lens=lens, K_out=Ko, V_out=Vo, mass_out=mo, index=self.index, lens_out=self.lens)
        self._sets.reverse()
        self.longest = min(longest, self.keep)

    def load(self, K, V, Q, LSE, scale):
        """Takes over a prompt's K, V [B,T,H_kv,d], rated by the rows Q [B,T_q,H,d] at its end (all of them, or the last ones) with the
        LSE [B,H,T_q] of their forward, and cut to ``keep`` keys."""
        if tuple(K.shape[::2]) + (K.shape[3],) != (self.B, self.H_kv, self.d):
            raise ValueError("K must be [B, T, H_kv, d] of this cache")
        mass = binding.moda_attn_key_mass(Q, K, LSE, scale)
        self._cut_into(K, V, mass, K.shape[1], None)
        self._attended = True

    def append(self, k, v):
        """The next token's key and value rows [B,H_kv,d]; cuts the cache first if it is full."""
        if self.longest == self.capacity:
            self._cut_into(*self._sets[0], self.longest, self.lens)
        at = self.lens.long()
        self.K[self._rows, at] = k
        self.V[self._rows, at] = v
        self.lens += 1
        self.longest += 1
        self._attended = False

    def attend(self, q, depth_kv_token, l, scale, O=None, LSE=None, workspace=None):
        """The step of the token appended last, or of another query over the same keys: O [B,H,d], LSE [B,H]; its weights are added to the
        accumulated ones."""
        if self.longest < 1:
            raise ValueError("append the token's key and value first")
        # the call starts the newest key from 0, which is right for a token's first step alone
        newest = (self._rows, slice(None), self.lens.long() - 1) if self._attended else None
        had = self.mass[newest] if self._attended else None
        O, LSE, _ = binding.moda_attn_decode_mass(q, self.K, self.V, depth_kv_token, self.longest, l, scale, seq_lens=self.lens, mass_in=self.mass, mass=self.mass,
                                                  O=O, LSE=LSE, workspace=workspace)
        if self._attended:
            self.mass[newest] += had
        self._attended = True
        return O, LSE


def cut_prompt(K, V, Q, LSE, scale, keep: int, recent: int = 0):
    """A prompt's K, V [1,T,H_kv,d] cut to min(keep, T) keys by the weight that its rows Q gave to them: K_prefix, V_prefix [keep,H_kv,d] for
    ``moda_attn_decode_shared``, and where they were [H_kv,keep]."""
    if K.shape[0] != 1:
        raise ValueError("one prompt: K and V must be [1, T, H_kv, d]")
    keep = min(int(keep), K.shape[1])
    mass = binding.moda_attn_key_mass(Q, K, LSE, scale)
    Ko, Vo, _, index, _ = binding.moda_kv_evict(K, V, mass, K.shape[1], keep, min(int(recent), keep))
    return Ko[0], Vo[0], index[0]
