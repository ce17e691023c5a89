"""Serving operators that bound and share the sequence cache, as cases that can be timed and compared.

``listed()`` names the cases, ``draw(rng)`` gives more of the same ranges, ``prepare`` makes what a program has in hand
before the call and ``run`` is one pass: through the package's entry points where ``own`` is true, else the operator's
plain form in 32 bits.  ``exact`` is the operator's definition in 64 bits.

Kinds of case (group ``k`` = the query heads that share key/value head ``k``):

    mass     attention weight that the last Tq rows give to each of T keys, summed over rows and the group's heads
             (``moda_attn_key_mass``): after a prompt, or of a window of its last rows
    step     a decode step that also adds its weights to an accumulator per key (``moda_attn_decode_mass``)
    evict    the keys of largest accumulated weight and the most recent ones, with their K, V rows (``moda_kv_evict``)
    shared   a decode step of a batch over one shared prefix, a cache of each sequence's own and the token's depth pairs
             (``moda_attn_decode_shared``)

Queries, keys and values are Gaussians, accumulated weights are log-normal (a few keys hold most of the weight).  Lengths
of the sequences of a batch are a permutation of evenly spaced ones, so that a case's work does not depend on the seed.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
BF16 = torch.bfloat16
F32 = torch.float32
F64 = torch.float64


def listed():
    return [
        # the window of a prompt's last rows that picks the keys to keep: all keys read for few rows
        dict(name="mass_window", kind="mass", B=4, Tq=64, T=8192, H=32, Hk=8, d=128),
        # a chunk of a ragged prompt over what is cached already, narrow heads, odd sizes
        dict(name="mass_chunk", kind="mass", B=3, Tq=1000, T=5003, H=16, Hk=16, d=64),
        # every row of a long prompt: the largest
        dict(name="mass_prompt", kind="mass", B=1, Tq=32768, T=32768, H=16, Hk=8, d=128),
        # one sequence, one token: latency
        dict(name="step_one", kind="step", B=1, T=2048, H=16, Hk=8, d=128, l=24, ragged=False),
        # a batch of sequences of different lengths, eight query heads per key/value head
        dict(name="step_ragged", kind="step", B=32, T=8192, H=64, Hk=8, d=128, l=24, ragged=True),
        # many short sequences, narrow heads, an odd group
        dict(name="step_narrow", kind="step", B=96, T=1500, H=24, Hk=8, d=64, l=32, ragged=True),
        # the cache of one sequence that has reached its limit
        dict(name="evict_one", kind="evict", B=1, T=2176, Hk=8, d=128, keep=2048, recent=256, ragged=False),
        # a batch after its prompts, each cut to an eighth of the longest
        dict(name="evict_batch", kind="evict", B=32, T=8192, Hk=8, d=128, keep=1024, recent=128, ragged=True),
        # a very long prompt, narrow heads, odd sizes
        dict(name="evict_long", kind="evict", B=1, T=131001, Hk=8, d=64, keep=16001, recent=1001, ragged=False),
        # four continuations of a short prompt: latency
        dict(name="shared_few", kind="shared", B=4, P=2048, T=64, H=16, Hk=8, d=128, l=24),
        # an odd number of continuations, an odd group, narrow heads
        dict(name="shared_odd", kind="shared", B=37, P=10007, T=301, H=24, Hk=8, d=64, l=32),
        # a large batch on a very long prefix
        dict(name="shared_long", kind="shared", B=128, P=131072, T=512, H=32, Hk=8, d=128, l=24),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6.5e12, w["flops"] / 1.6e15)


def draw(rng):
    top = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["mass", "step", "evict", "shared"])
        d = rng.choice([64, 128])
        G, Hk = rng.choice([1, 2, 3, 4, 5, 8]), rng.choice([1, 2, 4, 7, 8, 16])
        if kind == "mass":
            T = _log_int(rng, 1, 40000)
            case = dict(kind=kind, B=rng.randint(1, 4), Tq=min(T, _log_int(rng, 1, 40000)), T=T, H=Hk * G, Hk=Hk, d=d)
        elif kind == "step":
            case = dict(kind=kind, B=_log_int(rng, 1, 128), T=_log_int(rng, 1, 32768), H=Hk * G, Hk=Hk, d=d, l=rng.randint(0, 40),
                        ragged=rng.choice([False, True]))
        elif kind == "evict":
            T = _log_int(rng, 1, 140000)
            keep = rng.randint(1, T)
            case = dict(kind=kind, B=_log_int(rng, 1, 64), T=T, Hk=Hk, d=d, keep=keep, recent=rng.randint(0, keep), ragged=rng.choice([False, True]))
        else:
            case = dict(kind=kind, B=_log_int(rng, 1, 192), P=_log_int(rng, 1, 140000), T=_log_int(rng, 1, 2048), H=Hk * G, Hk=Hk, d=d,
                        l=rng.randint(0, 40))
        held = 4 * case["B"] * case["T"] * Hk * d + 4 * case.get("P", 0) * Hk * d
        scores = 4 * case["B"] * Hk * G * (case.get("P", 0) + case["T"] * (min(case["Tq"], 1024) if kind == "mass" else 1))
        if _cost(case) <= top and held <= 4e9 and scores <= 9e9:
            return case


def _lengths(case):
    """Lengths of a batch's sequences, in no order: evenly spaced over what the kind allows."""
    B, T = case["B"], case["T"]
    if case["kind"] == "shared":                         # a continuation may have no key of its own yet
        return [T * i // max(B - 1, 1) for i in range(B)] if B > 1 else [T]
    if not case.get("ragged"):
        return [T] * B
    return [max(1, T * (i + 1) // B) for i in range(B)]


def work(case):
    B, T, Hk, d = case["B"], case["T"], case["Hk"], case["d"]
    kind, n = case["kind"], sum(_lengths(case))
    if kind == "mass":
        H, Tq = case["H"], case["Tq"]
        pairs = Tq * (T - Tq) + Tq * (Tq + 1) // 2
        return {"bytes": 2 * B * d * (Tq * H + T * Hk) + 4 * B * (Tq * H + T * Hk), "flops": 2 * B * H * d * pairs}
    if kind == "evict":
        kept = sum(min(case["keep"], m) for m in _lengths(case))
        return {"bytes": 4 * Hk * n + Hk * kept * (8 * d + 8), "flops": 0}
    H, l = case["H"], case["l"]
    token = 4 * B * H * d + 4 * B * H + 4 * l * B * Hk * d
    if kind == "step":
        return {"bytes": 4 * Hk * d * n + 8 * Hk * n + token, "flops": 4 * H * d * (n + l * B)}
    return {"bytes": 4 * Hk * d * (case["P"] + n) + token, "flops": 4 * H * d * (B * case["P"] + n + l * B)}


# ---------------------------------------------------------------------------------------------------------------------
def _inputs(case, seed):
    """The case's inputs alone."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 6113 + 29)
    host = torch.Generator()
    host.manual_seed(seed * 7 + 3)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV, dtype=BF16)

    B, T, Hk, d, kind = case["B"], case["T"], case["Hk"], case["d"], case["kind"]
    x = {"case": case, "scale": d ** -0.5}
    lens = torch.tensor(_lengths(case), dtype=torch.int32)[torch.randperm(B, generator=host)]
    x["lens"] = lens.to(DEV)
    if kind == "mass":
        x["Q"], x["K"] = normal(B, case["Tq"], case["H"], d), normal(B, T, Hk, d)
        x["LSE"] = _lse(x["Q"], x["K"], x["scale"])
        return x
    x["K"], x["V"] = normal(B, T, Hk, d), normal(B, T, Hk, d)
    if kind in ("step", "evict"):
        x["mass_in"] = torch.randn((B, Hk, T), generator=g, device=DEV, dtype=F32).mul_(2).exp_()
    if kind != "evict":
        x["q"] = normal(B, case["H"], d)
        x["depth"] = normal(case["l"], B, Hk, 2, d)
    if kind == "shared":
        x["Kp"], x["Vp"] = normal(case["P"], Hk, d), normal(case["P"], Hk, d)
    return x


def _rows(case):
    """Rows of a mass case at a time: scores of one key/value head's group within 256 MB or so."""
    return max(1, min(case["Tq"], (1 << 26) // max(1, case["T"] * (case["H"] // case["Hk"]))))


def _lse(Q, K, scale):
    """LSE of causal attention of the last Tq positions, as the prefill call before this one left it."""
    B, Tq, H, d = Q.shape
    T, Hk = K.shape[1], K.shape[2]
    G, off = H // Hk, T - Tq
    out = torch.empty((B, H, Tq), device=DEV, dtype=F32)
    step = _rows(dict(Tq=Tq, T=T, H=H, Hk=Hk))
    for b in range(B):
        for k in range(Hk):
            keys = K[b, :, k].float()
            for i in range(0, Tq, step):
                n = min(step, Tq - i)
                seen = i + n + off
                s = (Q[b, i:i + n, k * G:(k + 1) * G].float().transpose(0, 1) @ keys[:seen].T) * scale
                s.masked_fill_(torch.arange(seen, device=DEV) > torch.arange(i, i + n, device=DEV)[:, None] + off, -math.inf)
                out[b, k * G:(k + 1) * G, i:i + n] = torch.logsumexp(s, -1)
    return out


def prepare(case, seed):
    """Inputs, and the buffers that a serving program keeps between steps."""
    x = _inputs(case, seed)
    B, T, Hk, d, kind = case["B"], case["T"], case["Hk"], case["d"], case["kind"]
    if kind in ("mass", "step"):
        x["mass"] = torch.zeros((B, Hk, T), device=DEV, dtype=F32)
    if kind == "evict":
        n = case["keep"]
        x["K_out"], x["V_out"] = torch.zeros((B, n, Hk, d), device=DEV, dtype=BF16), torch.zeros((B, n, Hk, d), device=DEV, dtype=BF16)
        x["mass_out"] = torch.zeros((B, Hk, n), device=DEV, dtype=F32)
        x["index"] = torch.full((B, Hk, n), -1, device=DEV, dtype=torch.int32)
        x["lens_out"] = torch.zeros((B,), device=DEV, dtype=torch.int32)
    if kind in ("step", "shared"):
        x["O"] = torch.empty((B, case["H"], d), device=DEV, dtype=BF16)
        x["LSE"] = torch.empty((B, case["H"]), device=DEV, dtype=F32)
    if own:
        import paper_2603_15619_b200 as moda
        x["moda"] = moda
        if kind == "step":
            n = moda.moda_decode_mass_workspace_bytes(B, T, case["H"], Hk, d)
        elif kind == "shared":
            n = moda.moda_decode_shared_workspace_bytes(B, case["P"], case["H"], Hk, d)
        elif kind == "mass":
            n = moda.moda_key_mass_workspace_bytes(B, case["Tq"], T, case["H"], Hk, d)
        else:
            n = 0
        x["work"] = torch.empty((max(n, 16),), device=DEV, dtype=torch.uint8)
    return x


def run(x):
    kind = x["case"]["kind"]
    if not own:
        return {"mass": _plain_mass, "step": _plain_step, "evict": _plain_evict, "shared": _plain_shared}[kind](x)
    moda, case = x["moda"], x["case"]
    if kind == "mass":
        return moda.moda_attn_key_mass(x["Q"], x["K"], x["LSE"], x["scale"], mass=x["mass"], workspace=x["work"])
    if kind == "step":
        return moda.moda_attn_decode_mass(x["q"], x["K"], x["V"], x["depth"], case["T"], case["l"], x["scale"],
                                          seq_lens=x["lens"] if case["ragged"] else None, mass_in=x["mass_in"], mass=x["mass"],
                                          O=x["O"], LSE=x["LSE"], workspace=x["work"])
    if kind == "evict":
        return moda.moda_kv_evict(x["K"], x["V"], x["mass_in"], case["T"], case["keep"], case["recent"],
                                  seq_lens=x["lens"] if case["ragged"] else None, K_out=x["K_out"], V_out=x["V_out"],
                                  mass_out=x["mass_out"], index=x["index"], lens_out=x["lens_out"])
    return moda.moda_attn_decode_shared(x["q"], x["Kp"], x["Vp"], x["K"], x["V"], x["lens"], x["depth"], case["T"], case["l"], x["scale"],
                                        O=x["O"], LSE=x["LSE"], workspace=x["work"])


# ------------------------------------------------------------------------------------------------ plain forms, 32 bits
def _plain_mass(x):
    case, Q, K, scale = x["case"], x["Q"], x["K"], x["scale"]
    B, Tq, H, d = Q.shape
    T, Hk = K.shape[1], K.shape[2]
    G, off = H // Hk, T - Tq
    mass = torch.zeros((B, Hk, T), device=DEV, dtype=F32)
    step = _rows(case)
    for b in range(B):
        for k in range(Hk):
            keys = K[b, :, k].float()
            for i in range(0, Tq, step):
                n = min(step, Tq - i)
                seen = i + n + off                                           # keys that some row of the block sees
                s = (Q[b, i:i + n, k * G:(k + 1) * G].float().transpose(0, 1) @ keys[:seen].T) * scale
                p = (s - x["LSE"][b, k * G:(k + 1) * G, i:i + n, None]).exp_()
                p.masked_fill_(torch.arange(seen, device=DEV) > torch.arange(i, i + n, device=DEV)[:, None] + off, 0.0)
                mass[b, k, :seen] += p.sum((0, 1))
    return mass


def _softmax_parts(parts):
    """Weights of one softmax over several score tensors (last dim), and its LSE; a row without keys has weights 0."""
    m = torch.stack([p.amax(-1) for p in parts if p.shape[-1]]).amax(0)
    base = torch.where(m == -math.inf, torch.zeros_like(m), m)
    e = [(p - base[..., None]).exp() for p in parts]
    total = sum(v.sum(-1) for v in e)
    safe = torch.where(total == 0, torch.ones_like(total), total)
    return [v / safe[..., None] for v in e], base + total.log()


def _own_scores(x, q):
    """Scores of a batch's queries [B, Hk, G, d] over its own cache, -inf past each length."""
    K = x["K"].float()
    s = torch.einsum("bkgd,btkd->bkgt", q, K) * x["scale"]
    return s.masked_fill_(torch.arange(K.shape[1], device=DEV) >= x["lens"][:, None, None, None], -math.inf)


def _depth_scores(x, q):
    return torch.einsum("bkgd,lbkd->bkgl", q, x["depth"][:, :, :, 0].float()) * x["scale"]


def _own_values(x, w):
    return torch.einsum("bkgt,btkd->bkgd", w, x["V"].float())


def _depth_values(x, w):
    return torch.einsum("bkgl,lbkd->bkgd", w, x["depth"][:, :, :, 1].float())


def _plain_step(x):
    case = x["case"]
    B, H, Hk, d = case["B"], case["H"], case["Hk"], case["d"]
    q = x["q"].float().view(B, Hk, H // Hk, d)
    (w, wd), lse = _softmax_parts([_own_scores(x, q), _depth_scores(x, q)])
    o = _own_values(x, w) + _depth_values(x, wd)
    at = torch.arange(case["T"], device=DEV)
    lens = x["lens"][:, None, None]
    mass = torch.where(at < lens - 1, x["mass_in"], 0.0) + torch.where(at < lens, w.sum(2), 0.0)
    return o.view(B, H, d).to(BF16), lse.view(B, H), mass


def _plain_evict(x):
    case, K, V, mass, lens = x["case"], x["K"], x["V"], x["mass_in"], x["lens"].long()[:, None, None]
    T, n = case["T"], case["keep"]
    at = torch.arange(T, device=DEV).expand_as(mass)
    kept = lens.clamp(max=n)
    rank = mass.masked_fill(at >= lens - kept.clamp(max=case["recent"]), math.inf).masked_fill(at >= lens, -math.inf)
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :n]
    index = torch.sort(order.masked_fill(torch.arange(n, device=DEV) >= kept, T), dim=-1).values
    there = index < T
    safe = index.clamp(max=T - 1)
    rows = safe.transpose(1, 2)[..., None].expand(-1, -1, -1, case["d"])
    mask = there.transpose(1, 2)[..., None]
    K_out, V_out = K.gather(1, rows) * mask, V.gather(1, rows) * mask
    mass_out = torch.where(there, mass.gather(2, safe), 0.0)
    return K_out, V_out, mass_out, torch.where(there, index, -1).int(), kept.view(-1).int()


def _plain_shared(x):
    case = x["case"]
    B, H, Hk, d = case["B"], case["H"], case["Hk"], case["d"]
    G = H // Hk
    q = x["q"].float().view(B, Hk, G, d)
    rows = q.transpose(0, 1).reshape(Hk, B * G, d)
    prefix = torch.bmm(rows, x["Kp"].float().permute(1, 2, 0)).mul_(x["scale"]).view(Hk, B, G, -1).transpose(0, 1)
    (wp, w, wd), lse = _softmax_parts([prefix, _own_scores(x, q), _depth_scores(x, q)])
    o = torch.bmm(wp.transpose(0, 1).reshape(Hk, B * G, -1), x["Vp"].float().transpose(0, 1)).view(Hk, B, G, d).transpose(0, 1)
    o = o + _own_values(x, w) + _depth_values(x, wd)
    return o.reshape(B, H, d).to(BF16), lse.reshape(B, H)


# ------------------------------------------------------------------------------------------- the definitions, 64 bits
def exact(case, seed):
    x = _inputs(case, seed)
    kind, scale = case["kind"], x["scale"]
    B, T, Hk, d = case["B"], case["T"], case["Hk"], case["d"]
    if kind == "evict":
        return None, None, _exact_kept_mass(x), None, None
    H = case["H"]
    G = H // Hk
    if kind == "mass":
        mass = torch.zeros((B, Hk, T), device=DEV, dtype=F64)
        first = T - case["Tq"]                                               # position of row 0
        block = max(1, (1 << 25) // T)
        for b in range(B):
            for h in range(H):
                keys = x["K"][b, :, h // G].to(F64)
                for lo in range(0, case["Tq"], block):
                    rows = x["Q"][b, lo:lo + block, h].to(F64)
                    logp = rows @ keys.T * scale - x["LSE"][b, h, lo:lo + block, None].to(F64)
                    mass[b, h // G] += torch.tril(logp.exp(), diagonal=first + lo).sum(0)
        return mass
    O = torch.zeros((B, H, d), device=DEV, dtype=F64)
    LSE = torch.zeros((B, H), device=DEV, dtype=F64)
    mass = torch.zeros((B, Hk, T), device=DEV, dtype=F64)
    lens = x["lens"].tolist()
    for k in range(Hk):
        shared = [x[n][:, k].to(F64) for n in ("Kp", "Vp")] if kind == "shared" else []
        for b in range(B):
            n = lens[b]
            keys = torch.cat([x["K"][b, :n, k].to(F64), x["depth"][:, b, k, 0].to(F64)] + shared[:1])
            values = torch.cat([x["V"][b, :n, k].to(F64), x["depth"][:, b, k, 1].to(F64)] + shared[1:])
            s = x["q"][b, k * G:(k + 1) * G].to(F64) @ keys.T * scale
            lse = torch.logsumexp(s, -1)
            p = (s - lse[:, None]).exp()
            O[b, k * G:(k + 1) * G], LSE[b, k * G:(k + 1) * G] = p @ values, lse
            if kind == "step":
                mass[b, k, :n] = p[:, :n].sum(0)
                mass[b, k, :n - 1] += x["mass_in"][b, k, :n - 1].to(F64)
    return (O, LSE, mass) if kind == "step" else (O, LSE)


def _exact_kept_mass(x):
    """Weights of the kept keys by counting, for every key, the keys that go before it."""
    case, lens = x["case"], x["lens"].tolist()
    out = torch.zeros((case["B"], case["Hk"], case["keep"]), device=DEV, dtype=F64)
    for b, n in enumerate(lens):
        kept = min(case["keep"], n)
        recent = min(case["recent"], kept)
        for k in range(case["Hk"]):
            mass = x["mass_in"][b, k, :n].to(F64)
            old = n - recent
            place = torch.full((n,), -1, device=DEV, dtype=torch.long)       # of an old key in order of weight
            place[:old][torch.argsort(mass[:old], descending=True, stable=True)] = torch.arange(old, device=DEV)
            out[b, k, :kept] = mass[place < kept - recent]
    return out
