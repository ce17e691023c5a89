"""Plain forms of the paged sequence cache in 8 bits, in numpy: the layout, the quantisation, the bounds, the selection, the decode step in 64 bits."""
import numpy as np
import torch

from oracle import moda_oracle as orc

BLOCK = 64
F32 = np.float32


def split(pages, d):
    """Writable views of pages uint8 [..., 128 d + 512]: key codes [..., 64, d], value codes [..., d, 64], scales of the keys and the values [..., 64]."""
    n, lead = BLOCK * d, pages.shape[:-1]
    scales = pages.view(F32)[..., 2 * n // 4:]
    return pages[..., :n].reshape(*lead, BLOCK, d), pages[..., n:2 * n].reshape(*lead, d, BLOCK), scales[..., :BLOCK], scales[..., BLOCK:]


def write(pages, bounds, K, V, table, start, n_new, page_size):
    """moda_kv_write_e4m3 on copies: pages and bounds after the call."""
    pages, bounds = pages.copy(), None if bounds is None else bounds.copy()
    B, T, Hk, d = K.shape
    sub = page_size // BLOCK
    flat = pages.reshape(-1, Hk, pages.shape[-1])
    n = BLOCK * d
    for b in range(B):
        s = max(int(start[b]), 0)
        end = min(s + min(max(int(n_new[b]), 0), T), table.shape[1] * page_size)
        for p in range(s, end):
            page = table[b, p // page_size]
            if not 0 <= page < pages.shape[0]:
                continue
            at = page * sub + p % page_size // BLOCK
            for X, off, turned in ((K, 0, False), (V, n, True)):
                codes, scale = orc.quantize_e4m3_rows(X[b, p - s])
                row = p % BLOCK
                if turned:
                    flat[at, :, off + row:off + n:BLOCK] = codes
                else:
                    flat[at, :, off + row * d:off + (row + 1) * d] = codes
                lo = 2 * n + 4 * (row + (BLOCK if turned else 0))
                flat[at, :, lo:lo + 4] = scale.astype(F32)[:, None].view(np.uint8)
        if bounds is not None:
            for j in range(s // BLOCK, -(-end // BLOCK) if end > s else 0):
                page = table[b, j // sub]
                if 0 <= page < pages.shape[0]:
                    at = page * sub + j % sub
                    bounds.reshape(-1, Hk, 2 * d + 16)[at, :, :2 * d + 4] = bounds_of(flat[at], d, min(BLOCK, end - j * BLOCK))
    return pages, bounds


def bounds_of(block, d, rows):
    """Bytes [Hk, 2 d + 4] of the bounds of a block's first `rows` keys."""
    codes, _, scale, _ = split(np.ascontiguousarray(block), d)
    with np.errstate(invalid="ignore", over="ignore"):
        keys = (orc.e4m3_decode_table().astype(F32)[codes[:, :rows]] * scale[:, :rows, None]).astype(F32)
    out = np.zeros((block.shape[0], 2 * d + 4), np.uint8)
    for h, k in enumerate(keys):
        if not np.isfinite(k).all():
            out[h, 2 * d:] = np.array([np.inf], F32).view(np.uint8)
            continue
        hi, lo = k.max(0), k.min(0)
        s = F32(max(np.abs(hi).max(), np.abs(lo).max())) / F32(127)
        if s > 0:
            out[h, :d] = np.minimum(np.ceil((hi / s).astype(F32)), 127).astype(np.int8).view(np.uint8)
            out[h, d:2 * d] = np.maximum(np.floor((lo / s).astype(F32)), -127).astype(np.int8).view(np.uint8)
        out[h, 2 * d:] = np.array([s], F32).view(np.uint8)
    return out


def gather(pages, table, b, hk, n, page_size, d, blocks=None):
    """float64 keys and values of a sequence's first n positions (or of those in `blocks`), without those that have no page."""
    codes = orc.e4m3_decode_table()
    sub, Hk = page_size // BLOCK, pages.shape[2]
    flat = pages.reshape(-1, Hk, pages.shape[-1])
    K, V = [np.zeros((0, d))], [np.zeros((0, d))]
    for j in range(-(-n // BLOCK)) if blocks is None else blocks:
        if not 0 <= j < -(-n // BLOCK):
            continue
        page = table[b, j // sub]
        if not 0 <= page < pages.shape[0]:
            continue
        kc, vc, ks, vs = split(np.ascontiguousarray(flat[page * sub + j % sub, hk]), d)
        rows = min(BLOCK, n - j * BLOCK)
        K.append(codes[kc[:rows]] * ks[:rows, None].astype(np.float64))
        V.append(codes[vc[:, :rows].T] * vs[:rows, None].astype(np.float64))
    return np.concatenate(K), np.concatenate(V)


def select(q, bounds, table, lens, page_size, n_blocks, n_recent):
    """index int32 [B, Hk, n_blocks]."""
    B, H, d = q.shape
    num_pages, sub, Hk = bounds.shape[:3]
    flat = bounds.reshape(-1, Hk, bounds.shape[-1])
    out = np.full((B, Hk, n_blocks), -1, np.int32)
    for b in range(B):
        n = -(-int(lens[b]) // BLOCK)
        kept = min(n_blocks, n)
        recent = min(n_recent, kept)
        old = n - recent
        for k in range(Hk):
            rows = q[b, k * (H // Hk):(k + 1) * (H // Hk)].astype(F32)
            most = np.abs(rows).max()
            q8 = np.rint((rows * (F32(127) / most if most > 0 else F32(0))).astype(F32)).astype(np.int64)
            rating = []
            for j in range(old):
                page = table[b, j // sub]
                if not 0 <= page < num_pages:
                    rating.append(-np.inf)
                    continue
                r = flat[page * sub + j % sub, k]
                hi, lo = r[:d].view(np.int8).astype(np.int64), r[d:2 * d].view(np.int8).astype(np.int64)
                s = r[2 * d:2 * d + 4].view(F32)[0]
                best = np.maximum(q8 * hi, q8 * lo).sum(-1).max()
                rating.append(float(F32(best) * s) if s < np.inf else np.inf)
            kept_old = sorted(sorted(range(old), key=lambda j: (-rating[j], j))[:kept - recent])
            out[b, k, :kept] = kept_old + list(range(old, n))
    return out


def decode(q, pages, table, lens, depth, scale, page_size, index=None):
    """o, lse in 64 bits and, per element, how far 32-bit arithmetic with weights of f16 may be off."""
    B, H, d = q.shape
    Hk = pages.shape[2]
    G = H // Hk
    q = q.astype(np.float64)
    o, lse = np.zeros((B, H, d)), np.full((B, H), -np.inf)
    o_tol, lse_tol = np.zeros((B, H, d)), np.zeros((B, H))
    for b in range(B):
        for k in range(Hk):
            blocks = None
            if index is not None:
                blocks = index[b, k][:min(index.shape[2], -(-int(lens[b]) // BLOCK))]
            K, V = gather(pages, table, b, k, int(lens[b]), page_size, d, blocks)
            if depth is not None and len(depth):
                K = np.concatenate([K, depth[:, b, k, 0].astype(np.float64)])
                V = np.concatenate([V, depth[:, b, k, 1].astype(np.float64)])
            if len(K) == 0:
                continue
            for h in range(k * G, (k + 1) * G):
                s = K @ q[b, h] * scale
                m = s.max()
                lse[b, h] = m + np.log(np.exp(s - m).sum())
                p = np.exp(s - lse[b, h])
                o[b, h] = p @ V
                # scores: sums of d products in fp32 (at most d roundings of 2^-24 of the sum of magnitudes, and a few of their scaling)
                ds = (d + 8) * 2.0 ** -24 * (np.abs(K) @ np.abs(q[b, h])).max() * scale
                # exponentials and logarithms to 2^-21, sums of n terms in fp32 over partial sums of a few hundred
                e = 2 * ds + 2.0 ** -20 + 1024 * 2.0 ** -24
                lse_tol[b, h] = ds + e + 2.0 ** -23 * abs(lse[b, h])
                # weights half a step of f16 off, the result half a step of bf16
                o_tol[b, h] = (2.0 ** -11 + 2 * e) * (p @ np.abs(V)) + 2.0 ** -8 * np.abs(o[b, h]) * 1.01 + 1e-30
    return o, lse, o_tol, lse_tol


def make(B, T, Hk, d, page_size, lens, seed, device="cuda", spare=2, garbage=True):
    """Pages of sequences of the given lengths, made without the library: what lies behind a sequence's last position is garbage.  Returns numpy pages, bounds,
    block table (int32) and the device copies of the three."""
    rng = np.random.default_rng(seed)
    sub = page_size // BLOCK
    need = [-(-int(n) // page_size) for n in lens]
    num = sum(need) + spare
    order = rng.permutation(num).astype(np.int32)
    table = np.full((B, max(-(-T // page_size), 1)), -7 if garbage else 0, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    fill = lambda *s: rng.integers(0, 256, s, dtype=np.uint8) if garbage else np.zeros(s, np.uint8)
    pages, bounds = fill(num, sub, Hk, 128 * d + 512), fill(num, sub, Hk, 2 * d + 16)
    K, V = (bf16(rng.standard_normal((B, max(max(lens), 1), Hk, d))) for _ in range(2))
    pages, bounds = write(pages, bounds, K, V, table, [0] * B, lens, page_size)
    dev = [torch.from_numpy(x.copy()).to(device) for x in (pages, bounds, table)]
    return pages, bounds, table, dev


def bf16(x):
    """Rounded to bf16, as float32."""
    return torch.from_numpy(np.asarray(x, F32)).to(torch.bfloat16).float().numpy()


def put(x, dtype=torch.bfloat16, device="cuda"):
    return torch.from_numpy(np.ascontiguousarray(x)).to(device=device, dtype=dtype)
