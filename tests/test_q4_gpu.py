"""Caches in 4 bits on the GPU: rows in (append, compaction, the fused pass) and
out, and attention over them, through the public entry points, against plain
64-bit forms (q4_ref.py)."""
import math

import pytest
import torch

import paged_ref
import q4_ref as ref
from test_paged_gpu import BF, F32, I32, _gen, _ints, _randn, _table, st  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


def _pools(st, g, pages, page, hkv, factors=False, noise=True):
    """Pools of random rows (whole pools: rows that nobody names hold other numbers)."""
    f = [torch.exp2(torch.randint(-3, 4, (hkv,), generator=g).float()) * (1 + 0.3 * torch.rand(hkv, generator=g))
         for _ in range(2)] if factors else [None, None]
    p = st.make_q4_pools(pages, page, hkv, *[x if x is None else x.cuda() for x in f])
    if noise:
        for x in "kv":
            c, s = ref.encode(torch.randn((pages, hkv, page, 128), generator=g))
            getattr(p, x).copy_(c)
            getattr(p, x + "_scale").view(torch.uint8).copy_(s)
    return p


def _special(g, *shape, dtype):
    """Rows with what quantising can go wrong on: zeros, borders between codes, groups of one size, tiny and huge."""
    x = torch.randn(shape, generator=g)
    flat = x.view(-1, 16)
    n = flat.shape[0]
    kinds = torch.randint(0, 10, (n,), generator=g)
    borders = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    for i in range(n):
        k = int(kinds[i])
        if k == 0:
            flat[i] = 0
        elif k == 1:  # elements at borders of a scale with four bits
            flat[i] = borders[torch.randint(0, 8, (16,), generator=g)] * (8 + i % 8) * 2.0 ** (i % 5 - 4)
            flat[i, i % 16] = -6.0 * (8 + i % 8) * 2.0 ** (i % 5 - 4)
        elif k == 2:
            flat[i] *= 1e-4
        elif k == 3:
            flat[i] *= 1e5
        elif k == 4:  # a scale at a border: 6 * 17/16
            flat[i] = flat[i].clamp(-1, 1)
            flat[i, 3] = 6.375 * 2.0 ** (i % 7 - 3)
        elif k == 5:
            flat[i] = -0.0
            flat[i, 5] = 1.0
    return x.to(dtype)


def _unsigned_zeros(c):
    """Codes with that of -0 (8) as that of 0: both stand for 0, and which of them a turned key of less than any code's
    half gets is a matter of its sign alone."""
    lo, hi = c & 15, c >> 4
    return torch.where(lo == 8, 0, lo) | torch.where(hi == 8, 0, hi) << 4


def _equal(p, x, codes, scales, at, turned=False):
    """Codes and scales of pool x at index `at` of [pages][hkv][page]."""
    c, s = getattr(p, x).cpu()[at], getattr(p, x + "_scale").view(torch.uint8).cpu()[at]
    if turned:
        c, codes = _unsigned_zeros(c), _unsigned_zeros(codes)
    assert torch.equal(s, scales), (x, (s != scales).sum(), (s != scales).nonzero()[:3])
    assert torch.equal(c, codes), (x, (c != codes).sum(), (c != codes).nonzero()[:3])


# ------------------------------------------------------------ rows in and out

@pytest.mark.parametrize("n,budget,hkv,page,layers,dtype,factors", [
    (300, 77, 4, 16, 3, BF, False), (300, 77, 1, 7, 2, F32, True), (64, 64, 2, 1, 1, BF, True), (1, 1, 3, 16, 1, F32, False),
    (500, 129, 8, 100, 34, BF, False)])
def test_compaction_bits(st, n, budget, hkv, page, layers, dtype, factors):
    """Codes and scales to the bit, rows of other sessions untouched."""
    g = _gen(n + hkv)
    table, pages = _table([40, budget], page, n)
    rows, pools, idx = [], [], []
    for _ in range(layers):
        k, v = (_special(g, n, hkv, 128, dtype=dtype) for _ in range(2))
        rows.append((k, v))
        pools.append(_pools(st, g, pages, page, hkv, factors))
        idx.append(torch.stack([torch.randperm(n, generator=g)[:budget].sort().values for _ in range(hkv)]).to(I32))
    before = [{x: (getattr(p, x).clone().cpu(), getattr(p, x + "_scale").view(torch.uint8).clone().cpu()) for x in "kv"} for p in pools]
    pt = st.make_pages(pages, page, table.cuda())
    st.stlite_compact_paged_q4([(k.cuda(), v.cuda(), p, i.cuda()) for (k, v), p, i in zip(rows, pools, idx)], budget, pt, 1)
    r = torch.arange(budget)
    at = (table[1].long()[r // page], slice(None), r % page)
    for l, p in enumerate(pools):
        for x, src in zip("kv", rows[l]):
            f = getattr(p, x + "_factor")
            kept = torch.stack([src[idx[l][h].long(), h] for h in range(hkv)], 1)
            c, s = ref.encode(kept, 1.0 if f is None else f[:, None])
            _equal(p, x, c, s, at)
            bc, bs = before[l][x]
            bc[at], bs[at] = c, s
            assert torch.equal(getattr(p, x).cpu(), bc) and torch.equal(getattr(p, x + "_scale").view(torch.uint8).cpu(), bs)


def test_compaction_leaves_bad_rows(st):
    """Indices outside the cache, pages outside the pool: those rows are left."""
    g = _gen(5)
    k, v = (_randn(g, 50, 2, 128) for _ in range(2))
    p = _pools(st, g, 4, 4, 2)
    was = {x: getattr(p, x).clone() for x in ("k", "v")}
    idx = torch.tensor([[0, 50, 7, -1, 9, 3], [1, 2, 3, 4, 5, 6]], dtype=I32)
    table = torch.tensor([[2, 9, 0]], dtype=I32)  # rows 4, 5 have no page
    st.stlite_compact_paged_q4([(k, v, p, idx.cuda())], 6, st.make_pages(4, 4, table.cuda()), 0)
    for x, src in (("k", k), ("v", v)):
        want = was[x].cpu()
        for h in range(2):
            for r in range(4):
                if 0 <= idx[h, r] < 50:
                    want[2, h, r] = ref.encode(src[int(idx[h, r]), h])[0]
        assert torch.equal(getattr(p, x).cpu(), want)


def test_groups_that_hold_no_number(st):
    """An infinity or a NaN makes its group NaN, and no other."""
    x = torch.randn((6, 1, 128), generator=_gen(1)).to(BF)
    for i, bad in enumerate((float("inf"), -float("inf"), float("nan"))):
        x[i, 0, 17 + 16 * i] = bad
    p = st.make_q4_pools(2, 4, 1)
    idx = torch.arange(6, dtype=I32, device="cuda")[None]
    pt = st.make_pages(2, 4, _ints([[1, 0]]), _ints([6]), max_new=6)
    st.stlite_compact_paged_q4([(x.cuda(), x.cuda(), p, idx)], 6, pt, 0)
    k, v = st.paged_fetch_q4(p, pt, 6)
    want = ref.decode(*ref.encode(x))
    for i in range(3):
        want[i, 0, 16 * (i + 1):16 * (i + 2)] = float("nan")
    for y in (k, v):
        assert torch.equal(y.cpu().double().nan_to_num(99), want.nan_to_num(99))


@pytest.mark.parametrize("page", [1, 7, 16, 64])
@pytest.mark.parametrize("hq,hkv,dtype,interleaved,axes,norm,fused,factors", [
    (28, 4, BF, False, 1, False, True, False), (12, 2, BF, True, 3, True, True, True), (7, 1, F32, False, 3, True, False, True),
    (3, 3, F32, True, 1, False, False, False)])
def test_append_bits(st, page, hq, hkv, dtype, interleaved, axes, norm, fused, factors):
    """q as stlite_rotate_qk leaves it; keys as the rotation in 64 bits put into 4; values as they are."""
    g = _gen(page + hq)
    new, old = [3, 0, 1, 9, 2], [0, 5, 16, 30, 1]
    rows, T, pad = [o + m for o, m in zip(old, new)], sum(new), 4
    x = _special(g, T + pad, hq + 2 * hkv, 128, dtype=dtype).cuda()
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    section = (16, 24, 24) if axes == 3 else (64, 0, 0)
    pos = torch.randint(0, 140000, (axes, T + pad), generator=g, dtype=I32).cuda()
    w = [(1 + 0.3 * torch.randn(128, generator=g)).to(dtype).cuda() if norm else None for _ in range(2)]
    rope = st.make_rope(1e6, section, interleaved)
    table, pages = _table(rows, page, page)
    cu = [sum(new[:i]) for i in range(len(new) + 1)]
    pt = st.make_pages(pages, page, table.cuda(), _ints(rows), _ints(cu), max_new=9)
    p = _pools(st, g, pages, page, hkv, factors)
    before = {y: getattr(p, y).clone().cpu() for y in "kv"}
    qo = torch.full((T + pad, hq, 128), 7, dtype=dtype, device="cuda")
    st.stlite_paged_append_q4(q, k, v, pos, rope, pt, qo, p, *w, 1e-5)
    want_q, _ = st.rotate_qk(q, k, pos, rope, *w, 1e-5)
    assert torch.equal(qo[:T], want_q[:T]) and (qo[T:] == 7).all()
    eps = torch.tensor(1e-5, dtype=F32).double().item()
    y, _ = paged_ref.rotate(k, pos, paged_ref.default_freq(1e6), section, interleaved, w[1], eps)
    seq = [s for s, m in enumerate(new) for _ in range(m)]
    row = [old[s] + i for s, m in enumerate(new) for i in range(m)]
    at = (torch.tensor([int(table[s, r // page]) for s, r in zip(seq, row)]), slice(None), torch.tensor([r % page for r in row]))
    for name, src in (("k", y), ("v", v)):
        f = getattr(p, name + "_factor")
        c, s = ref.encode(src[:T], 1.0 if f is None else f[:, None])
        _equal(p, name, c, s, at, name == "k")
        before[name][at] = c
        assert torch.equal(_unsigned_zeros(getattr(p, name).cpu()), _unsigned_zeros(before[name]))
    # and out again
    ko, vo = st.paged_fetch_q4(p, pt, T + pad, dtype)
    for name, got in (("k", ko), ("v", vo)):
        f = getattr(p, name + "_factor")
        want = ref.decode(getattr(p, name).cpu()[at], getattr(p, name + "_scale").view(torch.uint8).cpu()[at],
                          1.0 if f is None else f[:, None])
        paged_ref.within(got[:T], want, want.abs() * paged_ref.U)
        assert not got[T:].any()


def _turned_equal(p, y, interleaved, at, factor=1.0):
    """Keys of pool p have the codes and scales of y, but within 2^-50 of its pair's magnitude of a border an element
    may have the code of either side: angles are held to 2^-65 of a turn a position (1,000 of them 2^-52.4), and the
    reference, rounded four times, may be off by 2^-51 itself."""
    pairs = y.unflatten(-1, (64, 2) if interleaved else (2, 64))
    off = pairs.norm(dim=-1 if interleaved else -2, keepdim=True).expand_as(pairs).flatten(-2) * 2.0 ** -50
    ends = [(y.abs() - off).clamp_min(0), y.abs() + off]
    scale = p.k_scale.view(torch.uint8).cpu()[at]
    low, high = (ref.encode(e, factor)[1] for e in ends)
    assert ((low <= scale) & (scale <= high)).all() and (low != high).sum() < 10
    step = ref.SCALES[scale.long()].repeat_interleave(16, -1) * factor
    low, high = (ref.nearest((e / step).clamp_max(6.0), ref.VALUES[:8]) for e in ends)
    code = torch.stack([p.k.cpu()[at] & 15, p.k.cpu()[at] >> 4], -1).flatten(-2)
    assert ((low <= code % 8) & (code % 8 <= high)).all() and (low != high).sum() < 100
    assert ((code % 8 == 0) | ((code >= 8) == y.signbit())).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_keys_at_borders(st, interleaved):
    """Keys turned by tiny angles, elements at borders between codes and scales: each has the code of 64 bits."""
    g, T, hkv, page = _gen(31), 200, 4, 16
    k = _special(g, T, hkv, 128, dtype=BF)
    q = _randn(g, T, hkv, 128)
    pos = torch.randint(1, 1000, (T,), generator=g, dtype=I32)
    freq = [2.0 ** -(20 + i % 12) for i in range(64)]  # an element moves by some of its half steps in fp32
    rope = st.make_rope(interleaved=interleaved, inv_freq=freq)
    table, pages = _table([T], page, 3)
    pt = st.make_pages(pages, page, table.cuda(), _ints([T]), max_new=T)
    p, w = st.make_q4_pools(pages, page, hkv), (1 + 0.2 * torch.randn(128, generator=g)).to(BF)
    r = torch.arange(T)
    at = (table[0].long()[r // page], slice(None), r % page)
    eps = torch.tensor(1e-6, dtype=F32).double().item()
    for norm in (None, w.cuda()):
        st.stlite_paged_append_q4(q, k.cuda(), k.cuda(), pos.cuda(), rope, pt, q.clone(), p, None, norm, 1e-6)
        y, _ = paged_ref.rotate(k, pos[None], freq, (64, 0, 0), interleaved, norm, eps)
        _turned_equal(p, y, interleaved, at)
        _equal(p, "v", *ref.encode(k), at)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_keys_that_cancel(st, dtype, interleaved):
    """Pairs of one size turned by almost an eighth of a turn: one half of each, of either sign, is 2^-17 of what it is
    the difference of, all of it below the fp32 rotation's error, and the factor makes codes of it."""
    g, T, hkv, page = _gen(41), 40, 4, 16
    size = (0.5 + torch.rand((T, hkv, 64), generator=g)).to(dtype)
    sign = torch.tensor([1.0, -1.0])[torch.randint(0, 2, (2, T, hkv, 64), generator=g)]
    sign[1, :, 0], sign[1, :, 1] = sign[0, :, 0], -sign[0, :, 1]  # heads whose first halves, or second ones, cancel
    pair = (size * sign[0], size * sign[1])
    k = torch.stack(pair, -1).flatten(-2).to(dtype) if interleaved else torch.cat(pair, -1).to(dtype)
    freq = [2 * math.pi * (0.125 + (-1) ** i * (1 + i / 64) * 2.0 ** -20) for i in range(64)]
    factor = torch.tensor([1.0, 1.25, 1.5, 0.7]) * 2.0 ** -25
    table, pages = _table([T], page, 3)
    pt = st.make_pages(pages, page, table.cuda(), _ints([T]), max_new=T)
    p, q, pos = st.make_q4_pools(pages, page, hkv, factor.cuda()), _randn(g, T, 4, 128, dtype=dtype), torch.ones(T, dtype=I32)
    rope = st.make_rope(interleaved=interleaved, inv_freq=freq)
    st.stlite_paged_append_q4(q, k.cuda(), k.cuda(), pos.cuda(), rope, pt, q.clone(), p)
    y, _ = paged_ref.rotate(k, pos[None], freq, (64, 0, 0), interleaved)
    r = torch.arange(T)
    _turned_equal(p, y, interleaved, (table[0].long()[r // page], slice(None), r % page), factor.double()[:, None])


@pytest.mark.parametrize("tokens,hq,hkv,dtype", [(5003, 12, 2, BF), (2433, 3, 1, F32), (4868, 28, 4, BF)])
def test_long_prompts_as_short_ones(st, tokens, hq, hkv, dtype):
    """A call's tokens as calls of at most 1,000 of them leave them, padding unwritten."""
    g, page, pad = _gen(tokens), 64, 5
    q, k, v = (_randn(g, tokens + pad, h, 128, dtype=dtype) for h in (hq, hkv, hkv))
    pos, rope = torch.randint(0, 30000, (tokens + pad,), generator=g, dtype=I32).cuda(), st.make_rope(1e6)
    cut = tokens // 3
    table, pages = _table([cut, tokens - cut], page, tokens)
    out, pools = [torch.full_like(q, 7) for _ in range(2)], [st.make_q4_pools(pages, page, hkv) for _ in range(2)]
    pt = st.make_pages(pages, page, table.cuda(), _ints([cut, tokens - cut]), _ints([0, cut, tokens]), max_new=tokens)
    st.stlite_paged_append_q4(q, k, v, pos, rope, pt, out[0], pools[0])
    assert (out[0][tokens:] == 7).all()
    for s, (first, end) in enumerate(((0, cut), (cut, tokens))):
        for t in range(first, end, 1000):
            u = min(end, t + 1000)
            pt = st.make_pages(pages, page, table[s:s + 1].cuda(), _ints([u - first]), max_new=u - t)
            st.stlite_paged_append_q4(q[t:u], k[t:u], v[t:u], pos[t:u], rope, pt, out[1][t:u], pools[1])
    assert torch.equal(*out)
    for x in ("k", "v", "k_scale", "v_scale"):
        assert torch.equal(*(getattr(p, x).view(torch.uint8) for p in pools)), x


@pytest.mark.parametrize("layers", [1, 5, 33])
def test_fetch_whole_sessions(st, layers):
    """Every row of every session, an idle one and pages outside the pool among them: those rows are left."""
    g, page, hkv, rows = _gen(layers), 16, 2, [37, 0, 1, 64]
    table, pages = _table(rows, page, 3)
    table[3, 1] = pages + 5
    pools = [_pools(st, g, pages, page, hkv, True) for _ in range(layers)]
    cu = [0, 37, 37, 38, 102]
    pt = st.make_pages(pages, page, table.cuda(), _ints(rows), _ints(cu), max_new=64)
    for dtype in (BF, F32):
        out = [tuple(torch.full((110, hkv, 128), 5, dtype=dtype, device="cuda") for _ in range(2)) for _ in range(layers)]
        st.stlite_paged_fetch_q4([(p, *o) for p, o in zip(pools, out)], pt)
        for p, o in zip(pools, out):
            for x, got in zip("kv", o):
                d = ref.dense(p, x)
                for s, n in enumerate(rows):
                    for r in range(n):
                        y, t = got[cu[s] + r].cpu(), int(table[s, r // page])
                        if t >= pages:
                            assert (y == 5).all()
                        else:
                            paged_ref.within(y, d[t, r % page], d[t, r % page].abs() * paged_ref.U)
                assert (got[102:] == 5).all()


# ------------------------------------------------------------------ attention

def _attend(st, g, rows, new, page, hq, hkv, dtype, factors=False, w=None, pad=0, spare=2, scale=1.0):
    table, pages = _table(rows, page, len(rows) + page, spare)
    p = _pools(st, g, pages, page, hkv, factors)
    ragged = pad or len(set(new)) > 1
    cu = [sum(new[:i]) for i in range(len(new) + 1)]
    q = _randn(g, cu[-1] + pad, hq, 128, dtype=F32)
    q = (q * scale).to(dtype)
    pt = st.make_pages(pages, page, table.cuda(), _ints(rows), _ints(cu) if ragged else None, max_new=w or max(max(new), 1))
    return q, p, pt, table, cu


def _check(got, p, q, table, rows, cu, w=None, skip=()):
    want, bound = ref.attention(q, ref.dense(p, "k"), ref.dense(p, "v"), table, rows, cu, w, skip)
    live = ~want.isnan().any(-1).any(-1)
    paged_ref.within(got[live.to(got.device)], want[live], bound[live])
    return live


@pytest.mark.parametrize("page", [1, 7, 16, 24, 100])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("hq,hkv,rows,new", [
    (28, 4, [1, 15, 16, 17, 200, 33], [1] * 6), (7, 1, [700], [1]), (2, 2, [0, 40, 0, 3], [1] * 4),
    (16, 1, [50, 129], [3, 3]), (12, 2, [3, 70, 0, 18, 250], [5, 2, 0, 1, 5]), (32, 8, [90], [16]), (3, 1, [5, 20], [16, 16])])
def test_attention_matches(st, page, dtype, hq, hkv, rows, new):
    g = _gen(page + hq + len(rows))
    q, p, pt, table, cu = _attend(st, g, rows, new, page, hq, hkv, dtype, factors=page % 2 == 0)
    _check(st.paged_attention_q4(q, p, pt), p, q, table, rows, cu)


@pytest.mark.parametrize("hq,hkv,new", [(7, 1, 1), (14, 2, 3), (28, 4, 4), (16, 1, 2), (8, 8, 1)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_long(st, hq, hkv, new, dtype):
    """Sessions that many CTAs share beside short ones, scores that spread over a hundred powers of two."""
    g = _gen(hq + new)
    rows = [5000, 40, 1031, 0, 2]
    q, p, pt, table, cu = _attend(st, g, rows, [new] * 5, 16, hq, hkv, dtype, True, scale=6.0)
    ws = st.paged_q4_workspace(q, p, pt)
    out = torch.empty_like(q)
    st.stlite_paged_attention_q4(q, p, pt, out, ws)
    _check(out, p, q, table, rows, cu)
    assert st.stlite_device_status(ws) == st.STLITE_OK
    first = out.clone()
    for _ in range(3):  # the same bits on every repeat, whatever the workspace holds
        ws[16:].random_(0, 255)
        st.stlite_paged_attention_q4(q, p, pt, out, ws)
        assert torch.equal(out, first)


def test_attention_padding_and_idle(st):
    """Tokens behind the last sequence, tokens that see no row, and a session with fewer rows than tokens."""
    g = _gen(9)
    rows, new = [20, 0, 2, 64], [2, 3, 4, 0]
    q, p, pt, table, cu = _attend(st, g, rows, new, 16, 8, 2, BF, pad=5, w=4)
    ws, out = st.paged_q4_workspace(q, p, pt), torch.full_like(q, 3)
    q[7] = float("nan")  # a token that sees a row
    q[5] = float("nan")  # one that sees none
    st.stlite_paged_attention_q4(q, p, pt, out, ws)
    assert not out[2:7].any() and (out[9:] == 3).all() and out[7].isnan().all()
    q[7] = q[5] = 0
    st.stlite_paged_attention_q4(q, p, pt, out, ws)
    _check(out[:9], p, q[:9], table, rows, cu)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_extremes(st, dtype):
    """Queries of zeros, of very different elements, huge and tiny; caches of zeros and of one row repeated."""
    g = _gen(2)
    rows, new = [300, 64, 17], [4, 4, 4]
    q, p, pt, table, cu = _attend(st, g, rows, new, 16, 4, 1, dtype)
    q[0] = 0
    q[1] *= 1e-30
    q[2, 0] = 0
    q[2, 0, 5] = 3e38
    q[3, :, ::2] *= 1e-6
    q[4] *= 1e-38 if dtype == F32 else 1e-36
    p.k[int(table[1, 0])] = 0
    p.v_scale.view(torch.uint8)[int(table[2, 0])] = 0x7e  # the largest
    got = st.paged_attention_q4(q, p, pt)
    want, bound = ref.attention(q, ref.dense(p, "k"), ref.dense(p, "v"), table, rows, cu)
    for i in (0, 1, 3, 4, 5, 6, 7, 8, 9, 10, 11):
        paged_ref.within(got[i], want[i], bound[i])
    # scores of some 1e38: the row of the largest one takes all
    paged_ref.within(got[2, 1:], want[2, 1:], bound[2, 1:])
    assert ((got[2, 0].cpu().double() - want[2, 0]).abs() <= 2.0 ** -8 * 6).all()


def test_no_number_reaches_only_who_sees_it(st):
    """A key's NaN scale makes the seeing tokens' heads NaN, a value's its 16 elements; rows past a length and rows
    that only newer tokens see reach nobody else."""
    g = _gen(4)
    rows, new = [70, 33, 300], [4, 4, 4]
    for dtype in (BF, F32):
        for hq, hkv in ((8, 2), (28, 2)):
            q, p, pt, table, cu = _attend(st, g, rows, new, 16, hq, hkv, dtype)

            def place(s, r):
                return int(table[s, r // 16]), r % 16

            clean = st.paged_attention_q4(q, p, pt)
            ks, vs = (z.view(torch.uint8) for z in (p.k_scale, p.v_scale))
            for z in (ks, vs):  # past the lengths
                z[place(0, 70)[0], :, 70 % 16:] = 0x7f
                z[place(1, 33)[0], :, 33 % 16:] = 0xff
            assert torch.equal(st.paged_attention_q4(q, p, pt), clean)
            a, b = place(0, 68)
            vs[a, 1, b, 3] = 0xff      # seen by the last two tokens of session 0
            a, b = place(1, 32)
            ks[a, 0, b, 7] = 0x7f      # by the last one of session 1
            a, b = place(2, 7)
            vs[a, 0, b, 0] = 0x7f      # by all of session 2
            got, G = st.paged_attention_q4(q, p, pt), hq // hkv
            odd = torch.zeros(got.shape, dtype=torch.bool)
            odd[2:4, G:2 * G, 48:64] = True
            odd[7, :G] = True
            odd[8:12, :G, :16] = True
            assert torch.equal(got.isnan().cpu(), odd)
            assert torch.equal(got.cpu()[~odd], clean.cpu()[~odd])


def test_bad_pages_and_lengths(st):
    """Rows of pages outside the pool, and past the table, are left out and reported."""
    g = _gen(6)
    for rows in ([130, 90], [2100, 90]):
        q, p, pt, table, cu = _attend(st, g, rows, [2, 2], 16, 14, 2, BF)
        ws, out = st.paged_q4_workspace(q, p, pt), torch.empty_like(q)
        table[0, 3], table[1, 0] = p.k.shape[0], -1
        pt.table.copy_(table)
        st.stlite_paged_attention_q4(q, p, pt, out, ws)
        _check(out, p, q, table, rows, cu)
        assert st.stlite_device_status(ws) == st.STLITE_EINVAL
        table[0, 3] = table[1, 0] = 0
        pt.table.copy_(table)
        pt.length[0] = table.shape[1] * 16 + 5
        st.stlite_paged_attention_q4(q, p, pt, out, ws)
        _check(out, p, q, table, [table.shape[1] * 16, 90], cu)
        assert st.stlite_device_status(ws) == st.STLITE_EINVAL and st.stlite_device_status(ws) == st.STLITE_OK


def test_pools_past_32_bits(st):
    """Codes further than 2^32 bytes into the pool."""
    hkv, page = 8, 64
    pages = (1 << 32) // (hkv * page * 64) + 40
    p = st.make_q4_pools(pages, page, hkv)
    rows = [200, 70]
    table = torch.tensor([[pages - 1, 3, pages - 7, pages - 2], [pages - 3, pages - 30, 0, 0]], dtype=I32)
    g = _gen(8)
    k, v = (_randn(g, 300, hkv, 128) for _ in range(2))
    idx = torch.arange(200, dtype=I32).repeat(hkv, 1).cuda()
    pt = st.make_pages(pages, page, table.cuda(), _ints(rows), max_new=2)
    st.stlite_compact_paged_q4([(k, v, p, idx)], 200, pt, 0)
    st.stlite_compact_paged_q4([(k, v, p, (idx[:, :70] + 90).contiguous())], 70, pt, 1)
    q = _randn(g, 4, 16, 128)
    out = st.paged_attention_q4(q, p, pt)
    used = sorted(set(table.flatten().tolist()))
    small = st.Q4Pools(*[z[used].contiguous() for z in (p.k, p.v)], *[z.view(torch.uint8)[used].contiguous() for z in (p.k_scale, p.v_scale)])
    moved = torch.tensor([[used.index(x) for x in r] for r in table.tolist()], dtype=I32)
    _check(out, small, q, moved, rows, [0, 2, 4])
    ko, _ = st.paged_fetch_q4(p, pt, 4)
    assert torch.equal(ko[:2].double().cpu(), ref.decode(*ref.encode(k[198:200])))


def test_captured_and_grown(st):
    """Append and attention captured once, replayed as the sessions grow; two graphs share a workspace."""
    g, hq, hkv, page, S = _gen(12), 8, 2, 16, 3
    rows = [30, 1, 64]
    table, pages = _table([n + 8 for n in rows], page, 1)
    p = _pools(st, g, pages, page, hkv)
    length, pos, rope = _ints(rows), _ints([5, 6, 7]), st.make_rope()
    pt = st.make_pages(pages, page, table.cuda(), length)
    q, k, v = _randn(g, S, hq, 128), _randn(g, S, hkv, 128), _randn(g, S, hkv, 128)
    qo, out, out2, ws = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q), st.paged_q4_workspace(q, p, pt)

    def step(o):
        st.stlite_paged_append_q4(q, k, v, pos, rope, pt, qo, p)
        st.stlite_paged_attention_q4(qo, p, pt, o, ws)

    step(out)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph, o in zip(graphs, (out, out2)):
        with torch.cuda.graph(graph):
            step(o)
    for i in range(6):
        length += 1
        q.copy_(_randn(g, S, hq, 128))
        k.copy_(_randn(g, S, hkv, 128))
        graphs[0].replay()
        graphs[1].replay()
        rows = length.tolist()
        _check(out, p, qo, table, rows, [0, 1, 2, 3])
        assert torch.equal(out, out2)


def test_other_stream(st):
    """The helpers on a stream of the caller's."""
    g = _gen(3)
    rows = [100, 7]
    q, p, pt, table, cu = _attend(st, g, rows, [1, 1], 16, 8, 2, BF)
    s = torch.cuda.Stream()
    out = st.paged_attention_q4(q, p, pt, stream=s)
    k, _ = st.paged_fetch_q4(p, pt, 2, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    _check(out, p, q, table, rows, cu)
    d = ref.dense(p, "k")
    assert torch.equal(k[1].cpu().double(), d[int(table[1, 0]), 6])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_fused_pass_and_a_serving_step(st, dtype):
    """The pass into 4-bit pages keeps what the dense one keeps; tokens are appended and attended from; the session
    comes out again."""
    from paper_2603_00188_gb300 import synth
    from parity import to_device
    wl = synth.scaled("traj50", 3, beta=0.2)
    q, k, v = (x.to(dtype) for x in to_device(wl))
    hq, hkv, layers, page = q.shape[1], k.shape[1], 3, 16
    ks = [k, k.flip(0).contiguous(), (k * 0.5).contiguous()]
    b, prm = st.stlite_budget(k.shape[0], wl.beta), st.make_params(wl.beta)
    want = [st.compress_layer(q, x, v, wl.frames, beta=wl.beta) for x in ks]
    n_pages = -(-(b + 5) // page) + 9
    table = torch.full((2, -(-(b + 5) // page)), -1, dtype=I32, device="cuda")
    length, cu = _ints([0, 0]), _ints([0, 0, 0])
    free, n_free = torch.randperm(n_pages, generator=_gen(1)).to(I32).cuda(), _ints([n_pages])
    pt = st.make_pages(n_pages, page, table, length, cu, max_new=5)
    pools = [st.make_q4_pools(n_pages, page, hkv) for _ in range(layers)]
    st.stlite_pages_step(pt, None, _ints([0, b]), free, n_free, b)  # the second session begins
    idx = [torch.empty((hkv, b), dtype=I32, device="cuda") for _ in range(layers)]
    ws = st.workspace(st.make_shape(q, k), wl.frames, prm).repeat(layers)
    assert st.stlite_compress_layers_paged_q4([(q, x, v, p, i) for x, p, i in zip(ks, pools, idx)], wl.frames, prm, pt, 1, ws) == b
    for (ko, vo, ix), p, i in zip(want, pools, idx):
        assert torch.equal(ix, i)
        kf, vf = st.paged_fetch_q4(p, pt, b, F32)
        assert torch.equal(kf.cpu().double(), ref.decode(*ref.encode(ko)))
        assert torch.equal(vf.cpu().double(), ref.decode(*ref.encode(vo)))
    slot = torch.empty(5, dtype=I32, device="cuda")
    st.stlite_pages_step(pt, None, _ints([0, 3]), free, n_free, slot)
    assert cu.tolist() == [0, 0, 3] and length.tolist() == [0, b + 3] and slot[3:].tolist() == [-1, -1]
    g = _gen(2)
    nq, nk, nv = _randn(g, 5, hq, 128, dtype=dtype), _randn(g, 5, hkv, 128, dtype=dtype), _randn(g, 5, hkv, 128, dtype=dtype)
    pos, rope, qo = torch.arange(5, dtype=I32, device="cuda"), st.make_rope(), torch.zeros_like(nq)
    for p in pools:
        st.stlite_paged_append_q4(nq, nk, nv, pos, rope, pt, qo, p)
        out = st.paged_attention_q4(qo, p, pt)
        _check(out[:3], p, qo[:3], table, [0, b + 3], [0, 0, 3])
        _, vf = st.paged_fetch_q4(p, pt, 5, F32)
        assert torch.equal(vf[:3].cpu().double(), ref.decode(*ref.encode(nv[:3])))
        pool = p.v.transpose(1, 2).reshape(-1, hkv, 64)[slot[:3].long()]  # where the step said they go
        assert torch.equal(pool.cpu(), ref.encode(nv[:3])[0])
