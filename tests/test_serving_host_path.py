"""The serving calls through the host extension: what it hands back, and that its results are those of the Python form."""
import pytest
import torch

import paper_2603_15619_b200 as moda
from paper_2603_15619_b200 import binding

from test_host_path import _Refuses

BF16 = torch.bfloat16


def test_what_is_not_plain_is_handed_back():
    host = binding.host()
    for t in (torch.zeros(1, 4, 2, 64, dtype=BF16), torch.empty(1, 4, 2, 64, dtype=BF16, device="meta"), None, 3):
        assert host.key_mass(t, t, t, 0.1, None, None, None, None) is None
        assert host.decode_mass(t, t, t, None, None, 4, 0, 0.1, None, None, None, None, None) is None
        assert host.evict(t, t, t, 4, 2, 0, None, None, None, None, None, None) is None
        assert host.decode_shared(t, t, t, t, t, None, None, 4, 0, 0.1, None, None, None) is None
    assert host.key_mass() is None and host.decode_mass() is None and host.evict() is None and host.decode_shared() is None


def calls():
    g = torch.Generator(device="cuda").manual_seed(1)
    n = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=BF16)
    B, T, H, Hk, d, l = 2, 300, 8, 2, 64, 3
    Q, K, V, q, Kp = n(B, 40, H, d), n(B, T, Hk, d), n(B, T, Hk, d), n(B, H, d), n(500, Hk, d)
    depth, mass = n(l, B, Hk, 2, d), torch.rand((B, Hk, T), device="cuda")
    LSE = torch.full((B, H, 40), 6.0, device="cuda")
    lens = torch.tensor([300, 17], dtype=torch.int32, device="cuda")
    buf = torch.zeros((B, Hk, T), device="cuda")
    return {
        "mass": lambda **k: moda.moda_attn_key_mass(Q, K, LSE, 0.125, **k),
        "mass_in": lambda **k: moda.moda_attn_key_mass(Q, K, LSE, 0.125, T_kv=200, mass_in=mass, mass=buf.zero_(), **k)[:, :, :200].clone(),
        "step": lambda **k: moda.moda_attn_decode_mass(q, K, V, depth, T, l, 0.125, **k),
        "step_lens": lambda **k: moda.moda_attn_decode_mass(q, K, V, depth, T, l, 0.125, seq_lens=lens, mass_in=mass, mass=buf.zero_(), **k),
        "step_l0": lambda **k: moda.moda_attn_decode_mass(q, K, V, None, T, 0, 0.125, **k),
        "evict": lambda **k: [x[:1] for x in moda.moda_kv_evict(K, V, mass, T, 100, 10, **k)],
        "evict_lens": lambda **k: moda.moda_kv_evict(K, V, mass, T, 17, 3, seq_lens=lens, **k),
        "shared": lambda **k: moda.moda_attn_decode_shared(q, Kp, Kp, K, V, lens, depth, T, l, 0.125, **k),
        "shared_l0": lambda **k: moda.moda_attn_decode_shared(q, Kp, Kp, K, V, None, None, T, 0, 0.125, **k),
    }


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["mass", "mass_in", "step", "step_lens", "step_l0", "evict", "evict_lens", "shared", "shared_l0"])
def test_results_are_those_of_the_python_form(name, monkeypatch):
    f = calls()[name]
    served = []
    real = binding.host()

    class Watch:
        def __getattr__(self, fn):
            def call(*a):
                out = getattr(real, fn)(*a)
                served.append(out is not None)
                return out
            return call

    flat = lambda r: [x.clone() for x in (r if isinstance(r, (tuple, list)) else [r])]
    with monkeypatch.context() as m:
        m.setattr(binding, "host", lambda: Watch())
        fast = flat(f())
    assert served == [True]
    with monkeypatch.context() as m:
        m.setattr(binding, "host", lambda: _Refuses())
        slow = flat(f())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = flat(f(stream=s))
    s.synchronize()
    assert len(fast) == len(slow) == len(other)
    for a, b, c in zip(fast, slow, other):
        assert torch.equal(a, b) and a.shape == b.shape and a.dtype == b.dtype and torch.equal(a, c)


@pytest.mark.gpu
def test_errors_come_as_from_the_python_form():
    g = torch.Generator(device="cuda").manual_seed(1)
    n = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=BF16)
    K, q, mass = n(1, 64, 2, 64), n(1, 4, 64), torch.rand((1, 2, 64), device="cuda")
    LSE = torch.zeros((1, 4, 64), device="cuda")
    for f, code in [
        (lambda: moda.moda_attn_key_mass(n(1, 64, 4, 64), K, LSE, 0.0), -13), (lambda: moda.moda_attn_key_mass(n(1, 64, 4, 64), K, LSE, 0.1, T_kv=63), -3),
        (lambda: moda.moda_attn_key_mass(n(1, 64, 4, 64), K, LSE, 0.1, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), -7),
        (lambda: moda.moda_attn_decode_mass(q, K, K, None, 65, 0, 0.1), -3), (lambda: moda.moda_attn_decode_mass(n(1, 3, 64), K, K, None, 64, 0, 0.1), -12),
        (lambda: moda.moda_kv_evict(K, K, mass, 64, 20, 30), -3), (lambda: moda.moda_kv_evict(K, K, mass, 65, 20, 3), -3), (lambda: moda.moda_kv_evict(K, K, mass, 64, 0, 0), -3),
        (lambda: moda.moda_attn_decode_shared(q, n(8, 2, 64), n(8, 2, 64), K, K, None, None, -1, 0, 0.1), -3),
    ]:
        with pytest.raises(moda.ModaError) as e:
            f()
        assert e.value.code == code
    with pytest.raises(ValueError):                                          # not contiguous
        moda.moda_kv_evict(K.transpose(1, 2), K.transpose(1, 2), mass, 2, 1)
    with pytest.raises(ValueError):
        moda.moda_attn_decode_mass(q, K, K, None, 64, 0, 0.1, mass_in=torch.rand((1, 64, 2), device="cuda").transpose(1, 2))
    torch.cuda.synchronize()
