"""Attention over 4-bit pages at the ends of what factors and scores may be:
against plain 64-bit forms (q4_ref.py), or against what scores that are all
equal, or far apart, leave of the softmax."""
import math

import pytest
import torch

import paged_ref
import q4_ref as ref
from test_paged_gpu import BF, F32, I32, _gen, _ints, _table, st  # noqa: F401  (fixture)
from test_q4_gpu import _pools

pytestmark = pytest.mark.gpu
U = paged_ref.U


def _mean_bound(v, f32):
    """Of rows v [n][128] whose weights are equal: a weight is 2^x of x within 14, in two halves (ex2 2 ulp, 4 U), then
    rounded to 11 bits, or 22; the sums' chain is q4_ref.attention's."""
    weight = 2.0 ** -22 if f32 else 2.0 ** -11
    return v.abs().mean(0) * (weight + 8 * U + 2 * 2 * (len(v) / 4 + 112) * U)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("factor", [2.0 ** -60, 2.0 ** -25, 2.0 ** -21, 1.0, 2.0 ** 60])
@pytest.mark.parametrize("hq,hkv,new", [(7, 1, 1), (4, 2, 3), (16, 1, 2)])
def test_small_queries_and_any_factor(st, dtype, factor, hq, hkv, new):
    """Queries of zeros and tiny ones, heads of any factor, lengths that no block ends at: a score of 0 is one, not
    what is left of 0 times a factor that is none."""
    g, page, rows = _gen(hq + new), 16, [37, 1, 300, 1000, 64]
    table, pages = _table(rows, page, 5)
    p = _pools(st, g, pages, page, hkv)
    p = st.Q4Pools(p.k, p.v, p.k_scale, p.v_scale, torch.full((hkv,), factor, device="cuda"))
    q = torch.randn((len(rows) * new, hq, 128), generator=g)
    q[:, ::3] = 0
    q[:, 1::3] *= 1e-30
    q[:, 2::3] *= min(1.0, 1 / factor)
    q = q.to(dtype).cuda()
    pt = st.make_pages(pages, page, table.cuda(), _ints(rows), max_new=new)
    got = st.paged_attention_q4(q, p, pt)
    want, bound = ref.attention(q, ref.dense(p, "k"), ref.dense(p, "v"), table, rows, [new * s for s in range(len(rows) + 1)])
    paged_ref.within(got, want, bound)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("factor", [1.0, 2.0 ** 60])
def test_largest_scores(st, dtype, factor):
    """Products beyond fp32: the row of the largest takes all, equal ones share, and a score of 0 stays one."""
    g, page, hkv, rows = _gen(3), 16, 2, [40, 333, 50]
    table, pages = _table(rows, page, 4)
    p = _pools(st, g, pages, page, hkv)
    q = torch.randn((3, 8, 128), generator=g)
    q = (q / q.abs().amax(-1, keepdim=True) * 3e38).to(dtype)
    top = [11, 200]
    for s, r in enumerate(top):  # for each head a row of its queries' signs
        for h in range(hkv):
            q[s, 4 * h:4 * h + 4] = q[s, 4 * h].clone()
            row = torch.where(q[s, 4 * h].float() < 0, -6.0 * 448, 6.0 * 448)
            at = (int(table[s, r // page]), h, r % page)
            c, x = ref.encode(row)
            p.k[at], p.k_scale.view(torch.uint8)[at] = c.cuda(), x.cuda()
    p.k[table[2, :4].long().cuda()] = 0  # keys of zeros
    p = st.Q4Pools(p.k, p.v, p.k_scale, p.v_scale, torch.full((hkv,), factor, device="cuda"))
    pt = st.make_pages(pages, page, table.cuda(), _ints(rows))
    got = st.paged_attention_q4(q.cuda(), p, pt).cpu()
    v = ref.dense(p, "v")
    for s, r in enumerate(top):
        want = v[int(table[s, r // page]), r % page].repeat_interleave(4, 0)
        # its weight is over itself: as a reciprocal, 2 U
        paged_ref.within(got[s], want, want.abs() * 4 * U, s)
    for h in range(hkv):
        kept = paged_ref.rows_of(v, table[2], 50)[:, h]
        paged_ref.within(got[2, 4 * h:4 * h + 4], kept.mean(0).expand(4, 128), _mean_bound(kept, dtype == F32).expand(4, 128))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("hq,hkv,new", [(7, 1, 1), (8, 1, 3), (16, 2, 4)])
def test_scores_of_any_magnitude(st, dtype, sign, hq, hkv, new):
    """Scores of 2^18 to 2^33 (as powers of two), where fp32's numbers are 2^-5 to 2^10 apart: those of the rows that
    have the largest are all equal, the others' half of them or twice, so that the result is a mean."""
    g, page, n, S = _gen(hq + new), 16, 93, 64
    table, pages = _table([n], page, 3)
    p = st.make_q4_pools(pages, page, hkv)
    v = torch.randn((pages, hkv, page, 128), generator=g)
    large = torch.rand(n, generator=g) < 0.5
    large[:40] = False  # the largest come later
    large[n - new:] = False  # every token sees the same ones of them
    large[0] = sign < 0
    key = torch.zeros((pages, hkv, page, 128))
    for r in range(n):  # the larger score is that of 6, or of -3
        key[int(table[0, r // page]), :, r % page, 5] = 6.0 if large[r] else 3.0
    for x, src in (("k", key), ("v", v)):
        c, s = ref.encode(src)
        getattr(p, x).copy_(c)
        getattr(p, x + "_scale").view(torch.uint8).copy_(s)
    vd = paged_ref.rows_of(ref.dense(p, "v"), table[0], n)
    assert torch.equal(paged_ref.rows_of(ref.dense(p, "k"), table[0], n)[:, 0, 5], torch.where(large, 6.0, 3.0).double())
    size = torch.exp2(18 + 15 * torch.arange(S) / (S - 1)) / 6  # of the query that makes such a score of a 6
    q = torch.zeros((S, new, hq, 128))
    q[..., 5] = (sign * size * math.sqrt(128) / math.log2(math.e))[:, None, None]
    pt = st.make_pages(pages, page, table.repeat(S, 1).cuda(), _ints([n] * S), max_new=new)
    got = st.paged_attention_q4(q.view(S * new, hq, 128).to(dtype).cuda(), p, pt).view(S, new, hq, 128)
    for i in range(new):
        for h in range(hkv):
            rows = large if sign > 0 else ~large
            kept = vd[:, h][rows & (torch.arange(n) < n - (new - 1 - i))]
            G = hq // hkv
            shape = (S, G, 128)
            paged_ref.within(got[:, i, G * h:G * h + G], kept.mean(0).expand(shape),
                             _mean_bound(kept, dtype == F32).expand(shape), (i, h))
