"""The paged sequence cache in 8 bits, as cases that can be timed and compared.

``listed()`` names the cases, ``draw(rng)`` gives more of the same ranges, ``prepare`` makes what a program has in hand
before the call and ``run`` is one pass: through the package's entry points where ``own`` is true, else the operator's
plain form in 32 bits.  ``exact`` is the operator's definition in 64 bits.

Kinds of case (group ``k`` = the query heads that share key/value head ``k``; a block = 64 positions):

    write    new K, V rows quantised into the pages, and the bounds of every block that they touch (``moda_kv_write_e4m3``)
    read     rows of the pages as bf16 K, V again, for a prefill behind a cached prefix (``moda_kv_read_e4m3``)
    select   the blocks that a token attends to, by the bounds of their keys (``moda_kv_select_blocks``)
    decode   a decode step over the pages and the token's depth pairs (``moda_attn_decode_e4m3``)
    sparse   the blocks' selection and a decode step over them (both calls)

Pages: uint8 [num_pages][page_size / 64][Hk][128 d + 512], of a block the key codes [64][d], the value codes [d][64], 64 fp32
scales of the keys and 64 of the values.  Bounds: uint8 [num_pages][page_size / 64][Hk][2 d + 16], of a block's keys the largest
of each feature as int8 [d], the smallest as int8 [d], their fp32 scale and 12 bytes of nothing.

Queries, keys and values are Gaussians.  Lengths of the sequences of a batch are a permutation of evenly spaced ones, so that a
case's work does not depend on the seed, and their pages lie in no order.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
BF16 = torch.bfloat16
F32 = torch.float32
F64 = torch.float64
E4M3 = torch.float8_e4m3fn
BLOCK = 64


def listed():
    return [
        # a decode step's append: one token of each sequence of a batch
        dict(name="write_step", kind="write", B=64, T=1, at=2047, Hk=8, d=128, page=64, ragged=True),
        # chunks of prompts behind what is cached, of different lengths, narrow heads, odd sizes
        dict(name="write_chunk", kind="write", B=5, T=1000, at=777, Hk=7, d=64, page=128, ragged=True),
        # a long prompt: the largest
        dict(name="write_prompt", kind="write", B=1, T=65536, at=0, Hk=8, d=128, page=64, ragged=False),
        # short prefixes of a batch, narrow heads, odd sizes
        dict(name="read_few", kind="read", B=6, T=3001, Hk=5, d=64, page=64, ragged=True),
        # a long prefix before its next chunk
        dict(name="read_prompt", kind="read", B=1, T=65536, Hk=8, d=128, page=256, ragged=False),
        # one sequence: latency
        dict(name="select_one", kind="select", B=1, T=65536, H=16, Hk=8, d=128, page=64, keep=32, recent=2, ragged=False),
        # a batch of long sequences of different lengths
        dict(name="select_batch", kind="select", B=32, T=131072, H=32, Hk=8, d=128, page=64, keep=128, recent=4, ragged=True),
        # one sequence, one token: latency
        dict(name="decode_one", kind="decode", B=1, T=2048, H=16, Hk=8, d=128, l=24, page=64, ragged=False),
        # a batch of sequences of different lengths, eight query heads per key/value head
        dict(name="decode_ragged", kind="decode", B=32, T=8192, H=64, Hk=8, d=128, l=24, page=64, ragged=True),
        # many short sequences, narrow heads, an odd group
        dict(name="decode_narrow", kind="decode", B=96, T=1500, H=24, Hk=8, d=64, l=32, page=128, ragged=True),
        # one long sequence: latency
        dict(name="sparse_one", kind="sparse", B=1, T=65536, H=16, Hk=8, d=128, l=24, page=64, keep=32, recent=2, ragged=False),
        # a batch of long sequences of different lengths
        dict(name="sparse_batch", kind="sparse", B=16, T=131072, H=32, Hk=8, d=128, l=24, page=64, keep=128, recent=4, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6.5e12, w["flops"] / 1.6e15)


def draw(rng):
    top = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["write", "read", "select", "decode", "sparse"])
        d = rng.choice([64, 128])
        G, Hk = rng.choice([1, 2, 3, 4, 5, 7, 8, 16]), rng.choice([1, 2, 4, 7, 8, 16])
        case = dict(kind=kind, Hk=Hk, d=d, page=rng.choice([64, 128, 256]), ragged=rng.choice([False, True]))
        if kind == "write":
            case.update(B=_log_int(rng, 1, 128), T=_log_int(rng, 1, 65536), at=rng.choice([0, _log_int(rng, 1, 8192)]))
        elif kind == "read":
            case.update(B=_log_int(rng, 1, 64), T=_log_int(rng, 1, 65536))
        else:
            case.update(B=_log_int(rng, 1, 128), T=_log_int(rng, 1, 131072), H=Hk * G)
            if kind != "select":
                case["l"] = rng.randint(0, 40)
            if kind != "decode":
                keep = _log_int(rng, 1, 256)
                case.update(keep=keep, recent=rng.randint(0, min(keep, 8)))
                if kind == "select" and (keep == case["recent"] or _blocks(case["T"]) < keep + 4):
                    continue                             # nothing to choose
        positions = case["B"] * (case["T"] + case.get("at", 0))
        rated = positions // BLOCK * (Hk * d + Hk * G) if kind in ("select", "sparse") else 0
        read = positions if kind != "sparse" else case["B"] * case["keep"] * BLOCK
        if _cost(case) <= top and positions * Hk * d <= 1.2e9 and read * Hk * max(d, G) <= 6e8 and rated <= 6e8:
            return case


def _spread(B, most, least):
    """Evenly spaced lengths from about `least` to `most`."""
    return [least + (most - least) * i // (B - 1) for i in range(B)] if B > 1 else [most]


def _lengths(case):
    """Rows that a write brings, or lengths of the sequences, in no order; a batch may hold an empty place."""
    B, T = case["B"], case["T"]
    if not case["ragged"]:
        return [T] * B
    return _spread(B, T, 1 if case["kind"] == "write" else 0)


def _starts(case):
    """Positions that the rows of a write start at."""
    return _spread(case["B"], case["at"], case["at"] // 2 if case["ragged"] else case["at"])


def _blocks(n):
    return -(-n // BLOCK)


def work(case):
    Hk, d, kind = case["Hk"], case["d"], case["kind"]
    row, bound = 2 * d + 8, 2 * d + 16
    lens = _lengths(case)
    n = sum(lens)
    if kind == "write":
        return {"bytes": Hk * n * (4 * d + row) + Hk * bound * sum(_blocks(m) for m in lens), "flops": 0}
    if kind == "read":
        return {"bytes": Hk * n * (4 * d + row), "flops": 0}
    B, H = case["B"], case["H"]
    got = {"bytes": 2 * B * H * d, "flops": 0}
    if kind != "decode":
        blocks = sum(_blocks(m) for m in lens)
        got["bytes"] += Hk * bound * blocks + 4 * B * Hk * case["keep"]
        got["flops"] += 4 * H * d * blocks
    if kind != "select":
        l = case["l"]
        if kind == "sparse":
            n = sum(min(m, case["keep"] * BLOCK) for m in lens)
        got["bytes"] += Hk * row * n + 2 * B * H * d + 4 * B * H + 4 * l * B * Hk * d
        got["flops"] += 4 * H * d * (n + l * B)
    return got


# ------------------------------------------------------------------------------------------------------- the pages
def _views(pages, d):
    """Key codes [.., 64, d], value codes [.., d, 64], scales of the keys and of the values [.., 64] of a pages tensor."""
    n = BLOCK * d
    lead = pages.shape[:-1]
    return (pages[..., :n].unflatten(-1, (BLOCK, d)).view(E4M3), pages[..., n:2 * n].unflatten(-1, (d, BLOCK)).view(E4M3),
            pages[..., 2 * n:2 * n + 4 * BLOCK].view(F32), pages[..., 2 * n + 4 * BLOCK:].view(F32).reshape(*lead, BLOCK))


def _bound_views(bounds, d):
    """Largest and smallest [.., d] int8, and the scale [..]."""
    return bounds[..., :d].view(torch.int8), bounds[..., d:2 * d].view(torch.int8), bounds[..., 2 * d:2 * d + 4].view(F32)[..., 0]


def _full(v):
    """A number to divide (by): torch multiplies by the reciprocal where a plain one is given, which rounds twice."""
    return torch.full((), v, device=DEV)


def _quantise(x):
    """Codes and scales of rows [.., d]."""
    x = x.float()
    most = x.abs().amax(-1)
    scale = torch.where(most > 0, most / _full(448.0), torch.ones_like(most))
    return (x / scale[..., None]).clamp(-448.0, 448.0).to(E4M3), scale


def _bounds_of(K, valid):
    """Largest and smallest of each feature as int8, and their scale, of dequantised keys [.., 64, d] where `valid` [.., 64]."""
    hi = K.masked_fill(~valid[..., None], -math.inf).amax(-2)
    lo = K.masked_fill(~valid[..., None], math.inf).amin(-2)
    scale = torch.maximum(hi.abs(), lo.abs()).amax(-1) / _full(127.0)
    safe = torch.where(scale > 0, scale, torch.ones_like(scale))[..., None]
    return (hi / safe).ceil().clamp(max=127.0).to(torch.int8), (lo / safe).floor().clamp(min=-127.0).to(torch.int8), scale


def _table(case, lens, host):
    """A page for every place of the sequences, in no order: block table [B, most], and the number of pages."""
    sub = case["page"] // BLOCK
    need = [-(-_blocks(n) // sub) for n in lens]
    # a write's sequences have room for the longest, whatever start meets whatever length
    most = -(-_blocks(case["at"] + case["T"]) // sub) if case["kind"] == "write" else 0
    total = max(sum(need), most * case["B"], 1)
    order = torch.randperm(total, generator=host, dtype=torch.int32).tolist()
    table = torch.zeros((case["B"], max(max(need), 1)), dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    return table, total


def _tiles(table, j, sub):
    """Number of the block of 64 that holds block j [B, n] of each sequence, over all pages."""
    return table.gather(1, (j // sub)).long() * sub + j % sub


def _fill(x, g):
    """Pages (and bounds) of the sequences' cached positions, a sequence at a time."""
    case, sub = x["case"], x["case"]["page"] // BLOCK
    Hk, d = case["Hk"], case["d"]
    views = _views(x["pages"].flatten(0, 1), d)
    bounds = _bound_views(x["bounds"].flatten(0, 1), d) if "bounds" in x else None
    for b, n in enumerate(x["cached"]):
        if n == 0:
            continue
        blocks = _blocks(n)
        tile = _tiles(x["table"][b:b + 1].long(), torch.arange(blocks, device=DEV)[None], sub)[0]
        valid = (torch.arange(blocks * BLOCK, device=DEV) < n).view(blocks, 1, BLOCK)
        for i in range(2):
            codes, scale = _quantise(torch.randn((blocks, Hk, BLOCK, d), generator=g, device=DEV, dtype=F32).to(BF16))
            codes = codes.view(torch.uint8) * valid[..., None]
            scale = scale * valid
            views[i].view(torch.uint8)[tile] = codes if i == 0 else codes.transpose(-1, -2)
            views[2 + i][tile] = scale
            if i == 0 and bounds is not None:
                for to, v in zip(bounds, _bounds_of(codes.view(E4M3).float() * scale[..., None], valid.expand(-1, Hk, -1))):
                    to[tile] = v


# ---------------------------------------------------------------------------------------------------------- inputs
def _inputs(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 101)
    host = torch.Generator()
    host.manual_seed(seed * 13 + 5)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV, dtype=BF16)

    B, T, Hk, d, kind = case["B"], case["T"], case["Hk"], case["d"], case["kind"]
    sub = case["page"] // BLOCK
    x = {"case": case, "scale": d ** -0.5}
    order = torch.randperm(B, generator=host)
    lens = torch.tensor(_lengths(case), dtype=torch.int32)[order]
    x["lens"] = lens.to(DEV)
    if kind == "write":
        start = torch.tensor(_starts(case), dtype=torch.int32)[torch.randperm(B, generator=host)]
        x["start"], x["cached"], ends = start.to(DEV), start.tolist(), (start + lens).tolist()
        x["K"], x["V"] = normal(B, T, Hk, d), normal(B, T, Hk, d)
    else:
        x["cached"] = ends = lens.tolist()
    table, pages = _table(case, ends, host)
    x["table"] = table.to(DEV)
    if kind in ("write", "select", "sparse"):
        x["bounds"] = torch.zeros((pages, sub, Hk, 2 * d + 16), device=DEV, dtype=torch.uint8)
    if kind != "select":
        x["pages"] = torch.zeros((pages, sub, Hk, 2 * BLOCK * d + 8 * BLOCK), device=DEV, dtype=torch.uint8)
        _fill(x, g)
    else:
        # what Gaussian keys leave: extremes of 64 of them
        hi, lo, scale = _bound_views(x["bounds"], d)
        for to, sign in ((hi, 1), (lo, -1)):
            to.copy_((torch.rand(to.shape, generator=g, device=DEV) * 77 + 50).mul_(sign).to(torch.int8))
        scale.copy_(torch.randn(scale.shape, generator=g, device=DEV).mul_(0.1).exp_() * (3.6 / 127))
    if kind in ("select", "decode", "sparse"):
        x["q"] = normal(B, case["H"], d)
    if kind in ("decode", "sparse"):
        x["depth"] = normal(case["l"], B, Hk, 2, d)
    return x


def prepare(case, seed):
    """Inputs, and the buffers that a serving program keeps between steps."""
    x = _inputs(case, seed)
    B, T, Hk, d, kind = case["B"], case["T"], case["Hk"], case["d"], case["kind"]
    if kind == "read":
        x["K_out"], x["V_out"] = (torch.zeros((B, T, Hk, d), device=DEV, dtype=BF16) for _ in range(2))
    if kind in ("select", "sparse"):
        x["index"] = torch.full((B, Hk, case["keep"]), -1, device=DEV, dtype=torch.int32)
    if kind in ("decode", "sparse"):
        x["O"] = torch.empty((B, case["H"], d), device=DEV, dtype=BF16)
        x["LSE"] = torch.empty((B, case["H"]), device=DEV, dtype=F32)
    if own:
        import paper_2603_15619_b200 as moda
        x["moda"] = moda
        if kind in ("decode", "sparse"):
            x["work"] = torch.empty((moda.moda_decode_e4m3_workspace_bytes(B, case["H"], Hk, d),), device=DEV, dtype=torch.uint8)
    return x


def run(x):
    kind = x["case"]["kind"]
    if own:
        return _call(x)
    return {"write": _plain_write, "read": _plain_read, "select": _plain_select, "decode": _plain_decode, "sparse": _plain_sparse}[kind](x)


def _call(x):
    moda, case = x["moda"], x["case"]
    kind, T = case["kind"], case["T"]
    if kind == "write":
        moda.moda_kv_write_e4m3(x["pages"], x["K"], x["V"], x["table"], start=x["start"], n_new=x["lens"], bounds=x["bounds"])
        return _views(x["pages"], case["d"]) + _bound_views(x["bounds"], case["d"])
    if kind == "read":
        return moda.moda_kv_read_e4m3(x["pages"], x["table"], x["lens"], T, K_out=x["K_out"], V_out=x["V_out"])
    index = None
    if kind != "decode":
        index = moda.moda_kv_select_blocks(x["q"], x["bounds"], x["table"], x["lens"], T, case["keep"], case["recent"], index=x["index"])
    if kind == "select":
        return index
    O, LSE = moda.moda_attn_decode_e4m3(x["q"], x["pages"], x["table"], x["lens"], x["depth"], T, case["l"], x["scale"], index=index,
                                        O=x["O"], LSE=x["LSE"], workspace=x["work"])
    return (O, LSE) if index is None else (index, O, LSE)


# ------------------------------------------------------------------------------------------------ plain forms, 32 bits
def _plain_write(x):
    case, sub = x["case"], x["case"]["page"] // BLOCK
    B, T, d = case["B"], case["T"], case["d"]
    Kc, Vc, sk, sv = _views(x["pages"].flatten(0, 1), d)
    hi, lo, scale = _bound_views(x["bounds"].flatten(0, 1), d)
    # rows that are padding repeat the last one
    i = torch.minimum(torch.arange(T, device=DEV)[None], x["lens"][:, None].long() - 1)
    at = x["start"][:, None].long() + i
    tile, row = _tiles(x["table"], at // BLOCK, sub), at % BLOCK
    each = torch.arange(B, device=DEV)[:, None]
    codes, s = _quantise(x["K"][each, i])
    Kc.view(torch.uint8)[tile, :, row] = codes.view(torch.uint8)
    sk[tile, :, row] = s
    codes, s = _quantise(x["V"][each, i])
    Vc.view(torch.uint8)[tile, :, :, row] = codes.view(torch.uint8)
    sv[tile, :, row] = s
    first = x["start"][:, None].long() // BLOCK
    end = (x["start"] + x["lens"])[:, None].long()
    j = torch.minimum(first + torch.arange((T + BLOCK - 2) // BLOCK + 1, device=DEV)[None], (end - 1) // BLOCK)
    tile = _tiles(x["table"], j, sub)
    keys = Kc.view(torch.uint8)[tile].view(E4M3).float() * sk[tile][..., None]
    valid = j[..., None] * BLOCK + torch.arange(BLOCK, device=DEV) < end[..., None]
    hi[tile], lo[tile], scale[tile] = _bounds_of(keys, valid[:, :, None].expand(-1, -1, case["Hk"], -1))
    return _views(x["pages"], d) + _bound_views(x["bounds"], d)


def _plain_read(x):
    case, sub = x["case"], x["case"]["page"] // BLOCK
    T, d = case["T"], case["d"]
    Kc, Vc, sk, sv = _views(x["pages"].flatten(0, 1), d)
    at = torch.arange(T, device=DEV)[None].expand(case["B"], -1)
    there = (at < x["lens"][:, None])[..., None, None]
    at = torch.minimum(at, (x["lens"][:, None].long() - 1).clamp(min=0))
    tile, row = _tiles(x["table"], at // BLOCK, sub), at % BLOCK
    K = Kc.view(torch.uint8)[tile, :, row].view(E4M3).float() * sk[tile, :, row][..., None]
    V = Vc.view(torch.uint8)[tile, :, :, row].contiguous().view(E4M3).float() * sv[tile, :, row][..., None]
    return torch.where(there, K.to(BF16), x["K_out"]), torch.where(there, V.to(BF16), x["V_out"])


def _plain_select(x):
    case, sub = x["case"], x["case"]["page"] // BLOCK
    B, T, H, Hk, d, keep = (case[n] for n in ("B", "T", "H", "Hk", "d", "keep"))
    blocks = _blocks(T)
    hi, lo, scale = _bound_views(x["bounds"].flatten(0, 1), d)
    have = (x["lens"].long() + BLOCK - 1) // BLOCK
    at = torch.arange(blocks, device=DEV)[None].expand(B, -1)
    tile = _tiles(x["table"], torch.minimum(at, (have[:, None] - 1).clamp(min=0)), sub)
    q = x["q"].float().view(B, Hk, H // Hk, d)
    q = (q * (_full(127.0) / q.abs().amax((2, 3), keepdim=True))).round()
    # whole numbers below 2^24: any order of the sums gives the same
    dots = torch.einsum("bkgd,bnkd->bkgn", q.clamp(min=0), hi[tile].float()) + torch.einsum("bkgd,bnkd->bkgn", q.clamp(max=0), lo[tile].float())
    rating = dots.amax(2) * scale[tile].transpose(1, 2)
    at, have = at[:, None], have[:, None, None]
    kept = have.clamp(max=keep)
    rating = rating.masked_fill(at >= have - kept.clamp(max=case["recent"]), math.inf).masked_fill(at >= have, -math.inf)
    order = torch.sort(rating, dim=-1, descending=True, stable=True).indices[..., :keep]
    order = torch.nn.functional.pad(order, (0, keep - order.shape[-1]))
    order = torch.sort(order.masked_fill(torch.arange(keep, device=DEV) >= kept, blocks), dim=-1).values
    return torch.where(order < blocks, order, -1).int()


def _attend(q, K, V, there, depth, scale):
    """O and LSE of queries [B, Hk, G, d] over keys [B, Hk, n, d] where `there` [B, Hk, n], and depth pairs [l, B, Hk, 2, d]."""
    s = (q @ K.transpose(-1, -2)).mul_(scale).masked_fill_(~there[:, :, None], -math.inf)
    sd = torch.einsum("bkgd,lbkd->bkgl", q, depth[:, :, :, 0].float()) * scale
    m = s.amax(-1)
    if sd.shape[-1]:
        m = torch.maximum(m, sd.amax(-1))
    base = torch.where(m == -math.inf, torch.zeros_like(m), m)[..., None]
    s, sd = s.sub_(base).exp_(), (sd - base).exp()
    total = s.sum(-1) + sd.sum(-1)
    o = s @ V + torch.einsum("bkgl,lbkd->bkgd", sd, depth[:, :, :, 1].float())
    o = o / torch.where(total == 0, torch.ones_like(total), total)[..., None]
    B, Hk, G, d = q.shape
    return o.reshape(B, Hk * G, d).to(BF16), (base[..., 0] + total.log()).reshape(B, Hk * G)


def _plain_decode(x):
    case, sub = x["case"], x["case"]["page"] // BLOCK
    B, H, Hk, d = case["B"], case["H"], case["Hk"], case["d"]
    Kc, Vc, sk, sv = _views(x["pages"].flatten(0, 1), d)
    have = (x["lens"][:, None].long() + BLOCK - 1) // BLOCK
    j = torch.minimum(torch.arange(max(_blocks(case["T"]), 1), device=DEV)[None], (have - 1).clamp(min=0))
    tile = _tiles(x["table"], j, sub)
    K = (Kc.view(torch.uint8)[tile].view(E4M3).float() * sk[tile][..., None]).transpose(1, 2).flatten(2, 3)
    V = (Vc.view(torch.uint8)[tile].view(E4M3).float() * sv[tile][..., None, :]).permute(0, 2, 1, 4, 3).flatten(2, 3)
    there = (torch.arange(K.shape[2], device=DEV) < x["lens"][:, None])[:, None].expand(-1, Hk, -1)
    return _attend(x["q"].float().view(B, Hk, H // Hk, d), K, V, there, x["depth"], x["scale"])


def _plain_sparse(x):
    case, sub = x["case"], x["case"]["page"] // BLOCK
    B, H, Hk, d = case["B"], case["H"], case["Hk"], case["d"]
    index = _plain_select(x)
    Kc, Vc, sk, sv = _views(x["pages"].flatten(0, 1), d)
    j = index.long()
    tile = _tiles(x["table"], j.clamp(min=0).flatten(1), sub).view_as(j)
    head = torch.arange(Hk, device=DEV)[None, :, None]
    K = (Kc.view(torch.uint8)[tile, head].view(E4M3).float() * sk[tile, head][..., None]).flatten(2, 3)
    V = (Vc.view(torch.uint8)[tile, head].view(E4M3).float() * sv[tile, head][..., None, :]).transpose(-1, -2).flatten(2, 3)
    at = j[..., None] * BLOCK + torch.arange(BLOCK, device=DEV)
    there = ((j >= 0)[..., None] & (at < x["lens"][:, None, None, None])).flatten(2)
    return (index,) + _attend(x["q"].float().view(B, Hk, H // Hk, d), K, V, there, x["depth"], x["scale"])


# ------------------------------------------------------------------------------------------- the definitions, 64 bits
_CODES = None


def _values():
    """What the 256 codes stand for."""
    global _CODES
    if _CODES is None:
        v = []
        for c in range(256):
            e, m = c >> 3 & 15, c & 7
            a = math.nan if c & 127 == 127 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
            v.append(-a if c & 128 else a)
        _CODES = torch.tensor(v, dtype=F64, device=DEV)
    return _CODES


def _nearest(y):
    """The e4m3 values nearest to y, ties to the even mantissa."""
    v = _values()[:127]
    mid = (v[1:] + v[:-1]) / 2
    a = y.abs()
    up, down = torch.bucketize(a, mid, right=True), torch.bucketize(a, mid)       # they differ on a tie
    return v[torch.where(up % 2 == 0, up, down)].copysign(y)


def exact(case, seed):
    kind = case["kind"]
    if kind == "select":
        return None
    x = _inputs(case, seed)
    if kind == "write":
        return _exact_write(x)
    B, T, Hk, d, sub = case["B"], case["T"], case["Hk"], case["d"], case["page"] // BLOCK
    n = BLOCK * d
    raw, table, lens, scale = x["pages"].flatten(0, 1), x["table"].long(), x["lens"].tolist(), x["scale"]

    def rows(b, k, blocks):
        """Keys and values of blocks of a sequence's head."""
        block = torch.as_tensor(blocks, device=DEV, dtype=torch.long)
        r = raw[table[b, block // sub] * sub + block % sub, k]
        s = r[:, 2 * n:].contiguous().view(F32).to(F64)
        K = _values()[r[:, :n].long()].view(-1, BLOCK, d) * s[:, :BLOCK, None]
        V = _values()[r[:, n:2 * n].long()].view(-1, d, BLOCK) * s[:, None, BLOCK:]
        return K.reshape(-1, d), V.transpose(1, 2).reshape(-1, d)

    if kind == "read":
        K, V = (torch.zeros((B, T, Hk, d), device=DEV, dtype=F64) for _ in range(2))
        for b in range(B):
            for k in range(Hk):
                kb, vb = rows(b, k, range(_blocks(lens[b])))
                K[b, :lens[b], k], V[b, :lens[b], k] = kb[:lens[b]], vb[:lens[b]]
        return K, V
    H = case["H"]
    G = H // Hk
    O = torch.zeros((B, H, d), device=DEV, dtype=F64)
    LSE = torch.full((B, H), -math.inf, device=DEV, dtype=F64)
    for b in range(B):
        for k in range(Hk):
            own_q = x["q"][b, k * G:(k + 1) * G]
            blocks = list(range(_blocks(lens[b]))) if kind == "decode" else _exact_blocks(x, b, k, own_q, lens[b])
            keys, values = rows(b, k, blocks) if blocks else (torch.zeros((0, d), device=DEV, dtype=F64),) * 2
            at = (torch.tensor(blocks, device=DEV, dtype=torch.long)[:, None] * BLOCK + torch.arange(BLOCK, device=DEV)).flatten()
            keys, values = keys[at < lens[b]], values[at < lens[b]]
            keys = torch.cat([keys, x["depth"][:, b, k, 0].to(F64)])
            values = torch.cat([values, x["depth"][:, b, k, 1].to(F64)])
            if len(keys):
                s = own_q.to(F64) @ keys.T * scale
                LSE[b, k * G:(k + 1) * G] = torch.logsumexp(s, -1)
                O[b, k * G:(k + 1) * G] = torch.softmax(s, -1) @ values
    return (O, LSE) if kind == "decode" else (None, O, LSE)


def _exact_blocks(x, b, k, q, n):
    """The blocks that a head's queries [G, d] attend to, by whole numbers."""
    case, d = x["case"], x["case"]["d"]
    blocks = _blocks(n)
    kept = min(case["keep"], blocks)
    recent = min(case["recent"], kept)
    old = blocks - recent
    if kept - recent == 0 or old == 0:
        return list(range(old, blocks))
    sub = case["page"] // BLOCK
    block = torch.arange(old, device=DEV)
    r = x["bounds"].flatten(0, 1)[x["table"][b].long()[block // sub] * sub + block % sub, k]
    hi, lo = r[:, :d].view(torch.int8).to(F64), r[:, d:2 * d].view(torch.int8).to(F64)
    q = q.float()
    q = torch.round(q * (127.0 / q.abs().max().to(F64)).float()).to(F64)
    best = torch.stack([torch.maximum(hi * row, lo * row).sum(-1) for row in q]).amax(0)
    rating = (best.float() * r[:, 2 * d:2 * d + 4].contiguous().view(F32)[:, 0]).tolist()
    return sorted(sorted(range(old), key=lambda i: (-rating[i], i))[:kept - recent]) + list(range(old, blocks))


def _exact_write(x):
    case, sub = x["case"], x["case"]["page"] // BLOCK
    Hk, d = case["Hk"], case["d"]
    Kc, Vc, sk, sv = (v.flatten(0, 1).to(F64) for v in (t.float() for t in _views(x["pages"], d)))
    scale = _bound_views(x["bounds"], d)[2].flatten(0, 1).to(F64)
    lead = x["pages"].shape[:2]
    for b, (start, n) in enumerate(zip(x["start"].tolist(), x["lens"].tolist())):
        at = torch.arange(start, start + n, device=DEV)
        tile = x["table"][b].long()[at // case["page"]] * sub + at // BLOCK % sub
        for codes, scales, rows, turned in ((Kc, sk, x["K"], False), (Vc, sv, x["V"], True)):
            r = rows[b, :n].to(F64)
            s = r.abs().amax(-1) / 448
            s = torch.where(s > 0, s, torch.ones_like(s))
            c = _nearest((r / s.float().to(F64)[..., None]).float().to(F64))         # a quotient of 32 bits, as the format has it
            scales[tile, :, at % BLOCK] = s
            if turned:
                codes[tile, :, :, at % BLOCK] = c
            else:
                codes[tile, :, at % BLOCK] = c
        for j in range(start // BLOCK, _blocks(start + n)):
            t = int(x["table"][b, j // sub]) * sub + j % sub
            rows = min(BLOCK, start + n - j * BLOCK)
            scale[t] = (Kc[t, :, :rows] * sk[t, :, :rows, None]).abs().amax((1, 2)) / 127
    return tuple(v.unflatten(0, lead) for v in (Kc, Vc, sk, sv)) + (None, None, scale.unflatten(0, lead))
