"""Eviction in every form of its selection kernel (csrc/launch_rules.h), against a stable sort: positions, rows, weights and lengths are exact."""
import pytest
import torch

import paper_2603_15619_b200 as moda

from test_evict_forms import form  # noqa: F401

CASES = [
    # ranks, most keys of a thread, threads, CTAs of an SM; B, T, H_kv, n_keep, n_recent
    ((1, 5, 512, 2), 3, 2500, 60, 700, 9), ((2, 5, 512, 2), 2, 5000, 2, 900, 0), ((1, 9, 512, 2), 5, 4500, 50, 1000, 20), ((4, 9, 512, 2), 1, 16001, 8, 500, 30),
    ((1, 17, 512, 2), 10, 8600, 16, 2000, 1), ((8, 17, 512, 2), 1, 60001, 2, 777, 5), ((1, 33, 512, 2), 19, 16500, 8, 300, 40), ((4, 33, 512, 2), 20, 50000, 3, 500, 0),
    # the keys of a thread in registers, an SM to each CTA: one CTA a row, and clusters
    ((1, 33, 512, 1), 100, 13000, 1, 1500, 11), ((8, 33, 512, 1), 1, 131001, 8, 16001, 1001), ((8, 33, 512, 1), 2, 130000, 1, 129000, 0),
    ((4, 33, 1024, 1), 19, 99001, 2, 100, 7), ((8, 33, 1024, 1), 1, 250001, 1, 64, 64), ((16, 33, 1024, 1), 1, 397217, 1, 1000, 100),
    # more keys than the shared memories of a cluster hold: they are read again for every pass
    ((16, 0, 512, 1), 1, 600001, 1, 1000, 100), ((16, 0, 512, 1), 2, 545001, 1, 5000, 3),
]


@pytest.mark.parametrize("name,B,T,Hk,n_keep,n_recent", CASES)
def test_the_cases_take_the_forms_that_they_name(form, name, B, T, Hk, n_keep, n_recent):  # noqa: F811
    assert form(T, B * Hk)[:4] == name


def test_no_form_is_left_out(form):  # noqa: F811
    named = {c[0][1:] for c in CASES}
    taken = {form(T, rows)[1:4] for T in list(range(1, 40000, 611)) + list(range(40000, 700000, 9973)) for rows in (1, 8, 100, 148, 149, 5000)}
    assert taken == named


@pytest.mark.gpu
@pytest.mark.parametrize("weights", ["lognormal", "ties", "few_values_and_nan"])
@pytest.mark.parametrize("name,B,T,Hk,n_keep,n_recent", CASES)
def test_positions_rows_weights_and_lengths(name, B, T, Hk, n_keep, n_recent, weights):
    d, T_cap = 64, T + 3
    g = torch.Generator(device="cuda").manual_seed(T)
    K, V = (torch.randn((B, T_cap, Hk, d), generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    m = torch.randn((B, Hk, T_cap), generator=g, device="cuda")
    mass = {"lognormal": lambda: (2 * m).exp(), "ties": lambda: (m * 3).round(), "few_values_and_nan": lambda: m.sign()}[weights]()
    if weights == "few_values_and_nan":
        mass[:, :, 5::7] = float("nan")
        mass[:, :, 6::1001] = float("inf")
    mass[:, :, T:] = float("inf")                                            # past the length: never looked at
    lens = [T - (b * 997) % T for b in range(B)]
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    K_out, V_out, mass_out, index, lens_out = moda.moda_kv_evict(K, V, mass, T, n_keep, n_recent, seq_lens=seq)
    assert moda.moda_last_status() == 0
    for b, n in enumerate(lens):
        kept = min(n_keep, n)
        recent = min(n_recent, kept)
        assert int(lens_out[b]) == kept
        old = mass[b, :, :n - recent].double()
        old = torch.where(old.isnan(), -torch.inf, old)                      # no weight here is -inf: NaN below every number
        order = torch.sort(old, dim=-1, descending=True, stable=True).indices[:, :kept - recent]
        want = torch.cat([torch.sort(order, dim=-1).values, torch.arange(n - recent, n, device="cuda").expand(Hk, -1)], -1)
        assert torch.equal(index[b, :, :kept].long(), want) and bool((index[b, :, kept:] == -1).all())
        heads = torch.arange(Hk, device="cuda")[:, None].expand_as(want)
        assert torch.equal(K_out[b, :kept].transpose(0, 1), K[b, want, heads]) and torch.equal(V_out[b, :kept].transpose(0, 1), V[b, want, heads])
        assert torch.equal(mass_out[b, :, :kept].view(torch.int32), mass[b].gather(1, want).view(torch.int32))
