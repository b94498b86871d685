"""Attention over 4-bit pages at the ends of what factors and scores may be:
against plain 64-bit forms (q4_ref.py), or against what scores that are all
equal, or far apart, leave of the softmax."""
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
