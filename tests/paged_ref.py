"""Plain 64-bit forms of the paged-cache operators, row by row, and the error
bounds that the GPU results are held to.  CPU only; no code of the library."""
import math
from fractions import Fraction

import torch

U = 2.0 ** -24  # half a step of fp32


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def default_freq(base):
    return [base ** (-2.0 * i / 128) for i in range(64)]


TWO_PI = Fraction(2 * 314159265358979323846264338327950288419716939937510582097494459, 10 ** 62)


def angle(p, freq):
    """p * freq within a turn, the product and the reduction exact: a product in doubles is 2^-22 off at 2^31."""
    x = int(p) * Fraction(freq)
    return float(x - TWO_PI * round(x / TWO_PI))


def rotate(x, pos, inv_freq, section=(64, 0, 0), interleaved=False, norm=None, eps=1e-6):
    """x [T][H][128], pos [axes][T] -> (result, bound on a result's error before its rounding), 64 bits."""
    x = x.double().cpu()
    rel = 5.0
    if norm is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * norm.double().cpu()
        rel += 16.0
    pos = pos.cpu().view(-1, x.shape[0])
    y, bound = torch.empty_like(x), torch.empty_like(x)
    for i in range(64):
        axis = 0 if i < section[0] else (1 if i < section[0] + section[1] else 2)
        ang = torch.tensor([angle(p, inv_freq[i]) for p in pos[axis].tolist()], dtype=torch.float64)[:, None]
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + 64)
        xa, xb = x[..., a], x[..., b]
        y[..., a] = xa * ang.cos() - xb * ang.sin()
        y[..., b] = xb * ang.cos() + xa * ang.sin()
        # fp32: sine and cosine within 2.6 U (the angle's rounding, pi U / 2, and the function's), two
        # products and a sum 2 U, the upper 32 bits of the turn 2^-32 of pi; a norm 16 U more (19 additions halved by the root, 2 ulp of the root, two products)
        bound[..., a] = bound[..., b] = rel * U * (xa.abs() + xb.abs())
    return y, bound


def within(got, ref, bound, what=""):
    """|got - ref| <= bound plus the rounding to got's type."""
    g = got.detach().cpu().double()
    tol = bound + half_step(got.dtype) * (ref.abs() + bound) + torch.finfo(torch.float32).tiny
    bad = ~((g - ref).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), float((g - ref).abs().max()), bad.nonzero()[:3].tolist())


def rows_of(pool, table_row, n):
    """The first n rows of a sequence, [n][Hkv][128]."""
    page = pool.shape[1]
    ids = [int(p) for p in table_row[:-(-n // page)].tolist()]
    return pool[ids].reshape(-1, pool.shape[2], pool.shape[3])[:n]


def attention(q, k_pool, v_pool, table, lens, cu, w=None, skip_pages=()):
    """q [T][Hq][128] -> (result, bound before rounding); tokens of cu past the first w of a sequence and
    behind cu[-1] are NaN in the result.  skip_pages: pages whose rows are left out."""
    q = q.double().cpu()
    T, hq, _ = q.shape
    page, hkv = k_pool.shape[1], k_pool.shape[2]
    out = torch.full((T, hq, 128), math.nan, dtype=torch.float64)
    bound = torch.zeros_like(out)
    bf16 = k_pool.dtype == torch.bfloat16
    table = table.cpu()
    for s in range(len(lens)):
        first, m = cu[s], cu[s + 1] - cu[s]
        n = int(lens[s])
        if n > 0:
            safe = table[s].clone()
            keep = torch.ones(n, dtype=torch.bool)
            for i in range(-(-n // page)):
                if int(safe[i]) in skip_pages or int(safe[i]) < 0 or int(safe[i]) >= k_pool.shape[0]:
                    keep[i * page:(i + 1) * page] = False
                    safe[i] = 0
            k = rows_of(k_pool, safe.to(k_pool.device), n).cpu().double()
            v = rows_of(v_pool, safe.to(k_pool.device), n).cpu().double()
        for i in range(m if w is None else min(m, w)):
            sees = max(0, n - (m - 1 - i))
            for h in range(hkv):
                for g in range(h * hq // hkv, (h + 1) * hq // hkv):
                    if sees == 0 or not keep[:sees].any():
                        out[first + i, g] = 0
                        continue
                    kk, vv = k[:sees, h][keep[:sees]], v[:sees, h][keep[:sees]]
                    x = kk @ q[first + i, g] / math.sqrt(128)
                    p = torch.softmax(x, 0)
                    out[first + i, g] = p @ vv
                    mag = p @ vv.abs()
                    # a score: 128 products and sums, the factor and its product, in units of its magnitudes; its
                    # error moves p by e^delta - 1, numerator and denominator; exp2 2 U and the difference before it
                    size = float((kk.abs() @ q[first + i, g].abs()).max()) / math.sqrt(128)
                    delta = 132 * U * size
                    # sums: a warp adds at most every eighth row in turn, and then up to 16 warps and 1,024 splits
                    chain = (len(kk) / 8 + 16 + 64) * U
                    split = 2.0 ** -16 if bf16 else 0.0  # probabilities as two bf16 parts
                    bound[first + i, g] = mag * (2 * delta + 2 * chain + 8 * U + split)
    return out, bound
