"""Plain 64-bit forms of the 4-bit pages and of a step's page tables, and the
error bounds that the GPU results are held to.  CPU only; no code of the library."""
import math

import torch

from paged_ref import U

CODES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
NAN = 0x7f


def e4m3(byte):
    """The value of a scale's byte."""
    e, m = byte >> 3 & 15, byte & 7
    if byte & 0x7f == NAN:
        return math.nan
    return (-1.0 if byte >> 7 else 1.0) * (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))


SCALES = torch.tensor([e4m3(b) for b in range(256)], dtype=torch.float64)
VALUES = torch.tensor(CODES + [-c for c in CODES], dtype=torch.float64)


def nearest(x, values):
    """Index of the nearest of the ascending values; ties to the even index."""
    hi = torch.searchsorted(values, x.contiguous()).clamp(1, len(values) - 1)
    lo = hi - 1
    a, b = x - values[lo], values[hi] - x
    return torch.where((a < b) | ((a == b) & (lo % 2 == 0)), lo, hi)


def encode(x, factor=1.0):
    """x [..., 128] -> (codes uint8 [..., 64], scales uint8 [..., 8]); factor: a number or [..., 1]."""
    x = x.double().cpu()
    g = x.unflatten(-1, (8, 16)) / (factor if isinstance(factor, float) else factor.double().cpu()[..., None])
    odd = ~torch.isfinite(g).all(-1)
    g = torch.where(odd[..., None], torch.zeros_like(g), g)
    scale = nearest((g.abs().amax(-1) / 6).clamp(2.0 ** -9, 448.0), SCALES[:127])
    c = nearest((g.abs() / SCALES[scale][..., None]).clamp_max(6.0), VALUES[:8]) + 8 * (g.signbit() & ~odd[..., None])
    c = c.flatten(-2).to(torch.uint8)
    return c[..., 0::2] | c[..., 1::2] << 4, torch.where(odd, NAN, scale).to(torch.uint8)


def decode(codes, scales, factor=1.0):
    """The values in 64 bits."""
    codes, scales = codes.cpu().long(), scales.cpu().view(torch.uint8).long()
    v = VALUES[torch.stack([codes & 15, codes >> 4], -1).flatten(-2)].unflatten(-1, (8, 16))
    f = factor if isinstance(factor, float) else factor.double().cpu()[..., None]
    return (v * SCALES[scales][..., None] * f).flatten(-2)


def dense(pools, x):
    """Pool "k" or "v" in 64 bits as [n_pages][page_rows][Hkv][128], factors included."""
    f = getattr(pools, x + "_factor")
    return decode(getattr(pools, x), getattr(pools, x + "_scale"), 1.0 if f is None else f[:, None, None]).transpose(1, 2)


def attention(q, kd, vd, table, lens, cu, w=None, skip_pages=()):
    """q [T][Hq][128] over kd, vd of dense() -> (result, bound before rounding); tokens past the first w of a
    sequence and behind cu[-1] are NaN."""
    f32 = q.dtype == torch.float32
    q = q.double().cpu()
    T, hq, _ = q.shape
    page, hkv = kd.shape[1], kd.shape[2]
    out, bound = torch.full((T, hq, 128), math.nan, dtype=torch.float64), torch.zeros((T, hq, 128), dtype=torch.float64)
    table = table.cpu()
    for s in range(len(lens)):
        first, m, n = cu[s], cu[s + 1] - cu[s], max(0, int(lens[s]))
        ids = table[s, :-(-n // page)].tolist()
        keep = torch.tensor([p not in skip_pages and 0 <= p < kd.shape[0] for p in ids], dtype=torch.bool).repeat_interleave(page)[:n]
        ids = [p if 0 <= p < kd.shape[0] else 0 for p in ids]
        k, v = (x[ids].reshape(-1, hkv, 128)[:n] for x in (kd, vd))
        for i in range(m if w is None else min(m, w)):
            sees = max(0, n - (m - 1 - i))
            for g in range(hq):
                h = g * hkv // hq
                if not keep[:sees].any():
                    out[first + i, g] = 0
                    continue
                kk, vv, qq = k[:sees, h][keep[:sees]], v[:sees, h][keep[:sees]], q[first + i, g]
                p = torch.softmax(kk @ qq / math.sqrt(128), 0)
                out[first + i, g] = p @ vv
                mag = p @ vv.abs()
                size = kk.abs() @ qq.abs() / math.sqrt(128)
                # a query's elements as fp16 of a largest in [1, 2): 2^-25 of that; two parts of fp32 ones 2^-22 too
                part = 2.0 ** -25 * float(qq.abs().max()) * kk.abs().sum(-1) / math.sqrt(128)
                # a score: 128 products and sums, each cut off to fp32 at worst (2 U), its factors, the difference
                delta = float((264 * U * size + part + (2.0 ** -22 * size if f32 else 0)).max()) * 1.0001
                # weights to 2^-11, or 2^-22 in two parts, and 2^-25 where the largest is 2^10; 2^x 4 U.  Sums: at
                # least four warps share a session's blocks, then merges of up to 8 warps and 1,024 parts
                weight = 2.0 ** -22 if f32 else 2.0 ** -11
                chain = 2 * (len(kk) / 4 + 32 + 80) * U
                bound[first + i, g] = (mag * (2 * delta + 2 * chain + 12 * U + weight)
                                       + len(kk) * 2.0 ** -35 * vv.abs().amax(0))
    return out, bound


def step(table, lens, keep, fresh, free, n_free, n_pages, page, places):
    """stlite_pages_step on lists, in place; free has n_pages entries.  Returns (cu_new, n_free, slot)."""
    M = len(table[0])
    S = len(lens)
    have = [max(0, min(n, M * page)) for n in lens]
    stay = [h if keep is None else max(0, min(k, h)) for h, k in zip(have, keep or have)]
    new = [max(0, f) for f in fresh]
    top = max(0, min(n_free, n_pages))
    for s in range(S):
        for i in range(-(-stay[s] // page), -(-have[s] // page)):
            if top < n_pages:
                free[top] = table[s][i]
            top += 1
    top = min(top, n_pages)
    pages_asked = tokens_asked = 0
    cu, slot, at = [0], [], top
    for s in range(S):
        first, need = -(-stay[s] // page), -(-(stay[s] + new[s]) // page)
        ok = stay[s] + new[s] <= M * page
        if ok:
            pages_asked += need - first
            ok = need == first or pages_asked <= top
        if ok:
            tokens_asked += new[s]
            ok = new[s] == 0 or tokens_asked <= places
        f, need = (new[s], need) if ok else (0, first)
        for i in range(first, need):
            at -= 1
            table[s][i] = free[at]
        lens[s] = stay[s] + f
        for r in range(stay[s], stay[s] + f):
            p = table[s][r // page]
            slot.append(p * page + r % page if 0 <= p < n_pages else -1)
        cu.append(cu[-1] + f)
    return cu, at, slot + [-1] * (places - len(slot))
