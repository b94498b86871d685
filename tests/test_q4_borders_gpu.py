"""Rows into 4-bit pages of heads whose factor is any number: codes and scales
to the bit of the quotients' in 64 bits (q4_ref.encode), where fp32's nearest
to a quotient lies on the border between two."""
import math

import pytest
import torch

import q4_ref as ref
from test_paged_gpu import BF, F32, I32, _gen, _ints, _randn, _table, st  # noqa: F401  (fixture)
from test_q4_gpu import _equal

pytestmark = pytest.mark.gpu
BORDERS = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64)


def _beside(x, steps):
    """fp32 x, `steps` numbers further from 0."""
    return (x.view(I32) + steps).view(F32)


def _rows(g, n, hkv, dtype):
    """Rows [n][hkv][128] and the heads' factors: elements (and groups' largest) whose quotients are next to a border."""
    scale = ref.SCALES[torch.randint(1, 127, (n, hkv, 8), generator=g)]
    border = BORDERS[torch.randint(0, 7, (n, hkv, 8, 16), generator=g)]
    if dtype == F32:  # any factor: elements are within two steps of a border of theirs
        f = torch.exp2(torch.rand(hkv, generator=g) * 8 - 4)
        x = (border * (scale * f.double()[:, None])[..., None]).float()
        x = _beside(x, torch.randint(-2, 3, x.shape, generator=g).to(I32))
        # the largest: six times the scale, or next to six times a border to the next scale
        up = ref.SCALES[(torch.searchsorted(ref.SCALES[:127], scale) + 1).clamp_max(126)]
        top = torch.where(torch.rand(scale.shape, generator=g) < 0.5, scale, (scale + up) / 2)
        top = _beside((6 * top * f.double()[:, None]).float(), torch.randint(-2, 3, scale.shape, generator=g).to(I32))
    else:  # elements of 8 bits: the factor is the one that brings one of them to a border
        m = torch.randint(128, 256, (hkv,), generator=g).double() / 128
        steps, b0 = torch.randint(8, 16, (hkv,), generator=g).double(), BORDERS[torch.randint(0, 7, (hkv,), generator=g)]
        f = (m / (b0 * steps)).float()  # m / (step f) is b0, but for f's rounding
        f[::2] = (m / (6 * (2 * steps + 1))).float()[::2]  # and here a group's largest between two scales
        e = torch.exp2(torch.randint(-3, 4, (n, hkv, 8), generator=g).double())
        x = (m[:, None] * e)[..., None].expand(n, hkv, 8, 16).clone()
        x[torch.rand(x.shape, generator=g) < 0.3] *= 0.5
        top = (6 * (steps * f.double())[:, None] * e)
        top = torch.where(torch.arange(hkv)[:, None] % 2 == 0, m[:, None] * e, top)
    sign = torch.where(torch.rand(x.shape, generator=g) < 0.5, -1.0, 1.0)
    x = x.abs().minimum(top[..., None].to(x.dtype)) * sign
    at = torch.randint(0, 16, top.shape, generator=g)[..., None]
    x.scatter_(-1, at, top[..., None].to(x.dtype))
    return x.flatten(-2).to(dtype), f


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("hkv", [1, 64])
@pytest.mark.parametrize("which", ["kv", "k", "v"])
def test_rows_beside_borders(st, dtype, hkv, which):
    """Compaction of keys and values, and appended ones; heads with a factor for keys, for values or for both."""
    g, page, n = _gen(hkv), 16, 96
    x, f = _rows(g, n, hkv, dtype)
    want = {y: ref.encode(x, f[:, None] if y in which else 1.0) for y in "kv"}
    factors = [f.cuda() if y in which else None for y in "kv"]
    table, pages = _table([n], page, 7)
    r = torch.arange(n)
    at = (table[0].long()[r // page], slice(None), r % page)
    pt = st.make_pages(pages, page, table.cuda(), _ints([n]), max_new=n)
    p = st.make_q4_pools(pages, page, hkv, *factors)
    idx = torch.arange(n, dtype=I32).repeat(hkv, 1).cuda()
    st.stlite_compact_paged_q4([(x.cuda(), x.cuda(), p, idx)], n, pt, 0)
    for y in "kv":
        _equal(p, y, *want[y], at)
    p = st.make_q4_pools(pages, page, hkv, *factors)
    q, pos = _randn(g, n, hkv, 128, dtype=dtype), torch.zeros(n, dtype=I32, device="cuda")
    st.stlite_paged_append_q4(q, x.cuda(), x.cuda(), pos, st.make_rope(), pt, q.clone(), p)
    for y in "kv":  # at position 0 nothing turns: a row has one form, as a key and as a value
        _equal(p, y, *want[y], at, y == "k")


@pytest.mark.parametrize("factor", [0.35, 0.7, 1.4, 0.1, 3.3])
def test_factors_of_a_few_digits(st, factor):
    """Every bf16 element of two binades under every scale of one, in heads of such a factor."""
    page = 16
    m = torch.arange(128, 384).double() / 128
    f = torch.full((1,), factor)
    rows = []
    for scale in range(8, 16):
        group = torch.cat([m.view(-1, 8), -m.view(-1, 8)], -1) * 2.0 ** math.floor(math.log2(3 * factor))
        top = (6 * scale / 8 * f.double()).to(BF).double()
        rows.append(group.clamp(-top, top).index_fill(-1, torch.tensor([3]), float(top)).reshape(-1, 128))
    x = torch.cat(rows).to(BF)[:, None]
    n = len(x)
    table, pages = _table([n], page, 1)
    r = torch.arange(n)
    p = st.make_q4_pools(pages, page, 1, f.cuda(), f.cuda())
    pt = st.make_pages(pages, page, table.cuda(), _ints([n]), max_new=n)
    st.stlite_compact_paged_q4([(x.cuda(), x.cuda(), p, torch.arange(n, dtype=I32, device="cuda")[None])], n, pt, 0)
    for y in "kv":
        _equal(p, y, *ref.encode(x, f[:, None]), (table[0].long()[r // page], slice(None), r % page))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("exponent", [-60, -30, 30, 59])
def test_elements_far_from_their_factor(st, dtype, exponent):
    """Magnitudes from 2^-126 to 2^126 of either sign: quotients past fp32's ends become the largest code, or 0."""
    g, page, n, hkv = _gen(exponent + 99), 16, 40, 4
    f = 2.0 ** exponent * torch.tensor([1.0, 1.0 + 2 ** -23, 1.37, 1.99])
    x = torch.randn((n, hkv, 8, 16), generator=g).clamp(-1, 1) * torch.exp2(torch.randint(-126, 127, (n, hkv, 8, 1), generator=g).float())
    x[::3] *= torch.exp2(torch.randint(-40, 1, x[::3].shape, generator=g).float())
    x[:, :, :, 3] = torch.exp2(torch.randint(-126, 127, (n, hkv, 8), generator=g).float())  # few bits, as a border
    x[:, :, :, 4] = -x[:, :, :, 3]
    x = x.flatten(-2).to(dtype)
    want = ref.encode(x, f[:, None])
    table, pages = _table([n], page, 7)
    r = torch.arange(n)
    at = (table[0].long()[r // page], slice(None), r % page)
    pt = st.make_pages(pages, page, table.cuda(), _ints([n]), max_new=n)
    p = st.make_q4_pools(pages, page, hkv, f.cuda(), f.cuda())
    st.stlite_compact_paged_q4([(x.cuda(), x.cuda(), p, torch.arange(n, dtype=I32).repeat(hkv, 1).cuda())], n, pt, 0)
    for y in "kv":
        _equal(p, y, *want, at)
    p = st.make_q4_pools(pages, page, hkv, f.cuda(), f.cuda())
    q, pos = _randn(g, n, hkv, 128, dtype=dtype), torch.zeros(n, dtype=I32, device="cuda")
    st.stlite_paged_append_q4(q, x.cuda(), x.cuda(), pos, st.make_rope(), pt, q.clone(), p)
    for y in "kv":
        _equal(p, y, *want, at, y == "k")
