"""Paged caches on the GPU: rotation, append, attention and compaction through
the public entry points, against plain 64-bit forms (paged_ref.py)."""
import random

import pytest
import torch

import paged_ref as ref
from paper_2603_00188_gb300 import synth
from parity import to_device

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
I32 = torch.int32


@pytest.fixture(scope="module")
def st():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2603_00188_gb300 import build
    build.build()
    from paper_2603_00188_gb300 import stlite
    return stlite


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _randn(g, *shape, dtype=BF):
    return torch.randn(shape, generator=g).to(dtype).cuda()


def _table(rows, page, seed, spare=2, garbage=-7):
    """Every sequence's pages in random places; entries past them hold garbage."""
    count = [-(-n // page) for n in rows]
    pages = sum(count) + spare
    order = torch.randperm(pages, generator=_gen(seed)).tolist()
    most = max(1, max(count))
    table = torch.full((len(rows), most), garbage, dtype=I32)
    at = 0
    for s, c in enumerate(count):
        table[s, :c] = torch.tensor(order[at:at + c], dtype=I32)
        at += c
    return table, pages


def _ints(x):
    return torch.tensor(x, dtype=I32, device="cuda")


# ------------------------------------------------------------------ rotation

@pytest.mark.parametrize("n,hq,hkv,dtype,interleaved,axes,norm,fused", [
    (1, 28, 4, BF, False, 1, False, False), (1, 1, 1, F32, True, 3, True, False), (5, 12, 2, BF, False, 3, True, True),
    (33, 3, 3, BF, True, 1, True, True), (300, 28, 4, BF, False, 3, False, True), (77, 16, 8, F32, False, 1, True, True),
    (2, 7, 1, F32, True, 1, False, False), (1000, 5, 1, BF, True, 3, True, False), (4100, 2, 1, BF, False, 1, False, True)])
def test_rotate_matches(st, n, hq, hkv, dtype, interleaved, axes, norm, fused):
    g = _gen(n + hq)
    x = _randn(g, n, hq + 2 * hkv, 128, dtype=dtype)
    q, k = x[:, :hq], x[:, hq:hq + hkv]
    if not fused:
        q, k = q.contiguous(), k.contiguous()
    section = (16, 24, 24) if axes == 3 else (64, 0, 0)
    pos = torch.randint(0, 140000, (axes, n), generator=g, dtype=I32)
    wq, wk = ((1 + 0.3 * torch.randn(128, generator=g)).to(dtype).cuda() for _ in range(2)) if norm else (None, None)
    rope = st.make_rope(1e6, section, interleaved)
    qo, ko = torch.full_like(q.contiguous(), 9), torch.full_like(k.contiguous(), 9)
    st.stlite_rotate_qk(q, k, pos.cuda(), rope, qo, ko, wq, wk, 1e-5)
    freq = ref.default_freq(1e6)
    for got, src, w in ((qo, q, wq), (ko, k, wk)):
        r, b = ref.rotate(src, pos, freq, section, interleaved, w, 1e-5)
        ref.within(got, r, b)
    if norm:  # one of the two norms alone
        st.stlite_rotate_qk(q, k, pos.cuda(), rope, qo, ko, None, wk, 1e-5)
        r, b = ref.rotate(q, pos, freq, section, interleaved)
        ref.within(qo, r, b + 16 / 5 * b)


def test_rotate_at_far_positions(st):
    """Angles keep their precision to the ends of the positions' range."""
    pos = torch.tensor([0, 1, -1, 132800, 1 << 24, (1 << 24) + 1, 2 ** 31 - 1, -2 ** 31, 123456789], dtype=I32)
    g = _gen(3)
    q, k = _randn(g, len(pos), 2, 128, dtype=F32), _randn(g, len(pos), 1, 128, dtype=F32)
    for inv in (None, [2.5, -0.3, 1.0, 6.2831853, 40.0, 0.0] + [10.0 ** (-i / 8) for i in range(58)]):
        qo, ko = st.rotate_qk(q, k, pos.cuda(), st.make_rope(1e4, inv_freq=inv))
        freq = inv or ref.default_freq(1e4)
        for got, src in ((qo, q), (ko, k)):
            r, b = ref.rotate(src, pos, freq)
            ref.within(got, r, b)


@pytest.mark.parametrize("section", [(0, 64, 0), (0, 0, 64), (1, 62, 1), (63, 0, 1), (32, 32, 0)])
def test_rotate_sections(st, section):
    """Any division of the pairs among the axes, empty ones too."""
    g = _gen(11)
    q, k = _randn(g, 9, 3, 128), _randn(g, 9, 1, 128)
    pos = torch.randint(-50, 5000, (3, 9), generator=g, dtype=I32)
    for interleaved in (False, True):
        qo, ko = st.rotate_qk(q, k, pos.cuda(), st.make_rope(1e4, section, interleaved))
        for got, src in ((qo, q), (ko, k)):
            r, b = ref.rotate(src, pos, ref.default_freq(1e4), section, interleaved)
            ref.within(got, r, b)


def test_rotate_very_many_heads(st):
    """One token of more heads than the square of a 16-bit number's groups: the same as as many tokens of one head."""
    hq, hkv = 100 * 4096, 4096
    q, k = (torch.randn((1, h, 128), generator=torch.Generator("cuda").manual_seed(h), device="cuda").to(BF) for h in (hq, hkv))
    pos = _ints([4321])
    qo, ko = st.rotate_qk(q, k, pos, st.make_rope())
    for src, got in ((q, qo), (k, ko)):
        x = src[0, ::1024, None].contiguous()
        want, _ = st.rotate_qk(x, x, pos.repeat(x.shape[0]), st.make_rope())
        assert torch.equal(got[0, ::1024, None], want)
    part = slice(hq - 3000, hq)  # whole, at the far end
    x = q[0, part, None].contiguous()
    assert torch.equal(qo[0, part, None], st.rotate_qk(x, x, pos.repeat(3000), st.make_rope())[0])


def test_rotate_in_place_and_extremes(st):
    g = _gen(8)
    q, k = _randn(g, 50, 12, 128), _randn(g, 50, 2, 128)
    q[3, 5] = 0
    k[7, 0, 64:] = 1e30
    w = _randn(g, 128)
    pos = torch.arange(50, dtype=I32, device="cuda")
    want = st.rotate_qk(q, k, pos, st.make_rope(), w)
    assert not want[0][3, 5].any()  # a zero head stays zero under its norm
    q2, k2 = q.clone(), k.clone()
    st.stlite_rotate_qk(q2, k2, pos, st.make_rope(), q2, k2, w)
    assert torch.equal(q2, want[0]) and torch.equal(k2, want[1])
    assert torch.isfinite(want[1]).all()


# -------------------------------------------------------------------- append

@pytest.mark.parametrize("page", [1, 7, 16, 64])
@pytest.mark.parametrize("dtype,hq,hkv,norm,fused", [(BF, 28, 4, False, True), (F32, 6, 3, True, False),
                                                     (BF, 16, 1, True, True)])
def test_append_matches(st, page, dtype, hq, hkv, norm, fused):
    """Ragged new tokens (none for some sequences), padding behind them; only the new rows change."""
    g = _gen(page * 7 + hq)
    new = [3, 0, 1, 40, 2]
    rows = [3, 9, 65, 101, 2]
    cu = [0, 3, 3, 4, 44, 46]
    n = cu[-1] + 5
    table, pages = _table(rows, page, page)
    x = _randn(g, n, hq + 2 * hkv, 128, dtype=dtype)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    pos = torch.randint(0, 100000, (3, n), generator=g, dtype=I32)
    section = (16, 24, 24)
    wq, wk = (_randn(g, 128, dtype=dtype) for _ in range(2)) if norm else (None, None)
    kp, vp = (torch.full((pages, page, hkv, 128), 7, dtype=dtype, device="cuda") for _ in range(2))
    qo = torch.full((n, hq, 128), 5, dtype=dtype, device="cuda")
    pg = st.make_pages(pages, page, table.cuda(), _ints(rows), _ints(cu))
    st.stlite_paged_append(q, k, v, pos.cuda(), st.make_rope(1e6, section), pg, qo, kp, vp, wq, wk)
    freq = ref.default_freq(1e6)
    rq, bq = ref.rotate(q, pos, freq, section, norm=wq)
    rk, bk = ref.rotate(k, pos, freq, section, norm=wk)
    ref.within(qo[:cu[-1]], rq[:cu[-1]], bq[:cu[-1]], "q")
    assert (qo[cu[-1]:] == 5).all()
    want_k, bound = torch.full(kp.shape, 7, dtype=torch.float64), torch.zeros(kp.shape, dtype=torch.float64)
    want_v = torch.full(vp.shape, 7, dtype=dtype)
    for s in range(5):
        for i in range(new[s]):
            r = rows[s] - new[s] + i
            at = int(table[s, r // page]), r % page
            want_k[at], bound[at], want_v[at] = rk[cu[s] + i], bk[cu[s] + i], v[cu[s] + i].cpu()
    ref.within(kp, want_k, bound, "k")
    assert torch.equal(vp.cpu(), want_v)


@pytest.mark.parametrize("seqs", [32, 33, 200, 1100])
def test_append_finds_every_sequence(st, seqs):
    """Each token's sequence among many, several of them without new tokens, the last ones too."""
    r = random.Random(seqs)
    new = [r.choice([0, 0, 1, 2, 5]) for _ in range(seqs - 2)] + [0, 0]
    rows = [m + r.randint(0, 20) for m in new]
    cu = [sum(new[:i]) for i in range(seqs + 1)]
    g = _gen(seqs)
    q, k, v = _randn(g, cu[-1] + 2, 1, 128), _randn(g, cu[-1] + 2, 1, 128), _randn(g, cu[-1] + 2, 1, 128)
    table, pages = _table(rows, 4, seqs)
    kp, vp = (torch.full((pages, 4, 1, 128), 7, dtype=BF, device="cuda") for _ in range(2))
    pg = st.make_pages(pages, 4, table.cuda(), _ints(rows), _ints(cu))
    pos = torch.arange(cu[-1] + 2, dtype=I32, device="cuda")
    qo = torch.full_like(q, 5)
    st.stlite_paged_append(q, k, v, pos, st.make_rope(), pg, qo, kp, vp)
    wq, wk = st.rotate_qk(q, k, pos, st.make_rope())
    want_k, want_v = torch.full_like(kp, 7), torch.full_like(vp, 7)
    at = [(int(table[s, (rows[s] - m + i) // 4]), (rows[s] - m + i) % 4, cu[s] + i)
          for s, m in enumerate(new) for i in range(m)]
    p, o, t = (torch.tensor(x, device="cuda") for x in zip(*at))
    want_k[p, o], want_v[p, o] = wk[t], v[t]
    assert torch.equal(kp, want_k) and torch.equal(vp, want_v)
    assert torch.equal(qo[:cu[-1]], wq[:cu[-1]]) and (qo[cu[-1]:] == 5).all()


def test_append_one_each_and_in_place(st):
    """Without cu_new: `max_new` tokens of each sequence, q rotated in place."""
    g = _gen(4)
    rows = [17, 4, 260]
    table, pages = _table(rows, 16, 1)
    q, k, v = _randn(g, 6, 4, 128), _randn(g, 6, 2, 128), _randn(g, 6, 2, 128)
    pos = torch.arange(6, dtype=I32, device="cuda")
    kp, vp = (torch.zeros((pages, 16, 2, 128), dtype=BF, device="cuda") for _ in range(2))
    pg = st.make_pages(pages, 16, table.cuda(), _ints(rows), max_new=2)
    want, wk = st.rotate_qk(q, k, pos, st.make_rope())
    st.stlite_paged_append(q, k, v, pos, st.make_rope(), pg, q, kp, vp)
    assert torch.equal(q, want)
    for s in range(3):
        got = ref.rows_of(kp, table[s], rows[s])[-2:], ref.rows_of(vp, table[s], rows[s])[-2:]
        assert torch.equal(got[0], wk[2 * s:2 * s + 2]) and torch.equal(got[1], v[2 * s:2 * s + 2])
    assert int(kp.ne(0).any(-1).any(-1).sum()) == 6


def test_append_many_each(st):
    """A long chunk of every prompt without cu_new, more tokens each than an observation window may have."""
    g = _gen(6)
    rows, w = [700, 601, 999], 600
    table, pages = _table(rows, 24, 2)
    q, k, v = _randn(g, 3 * w, 3, 128), _randn(g, 3 * w, 1, 128), _randn(g, 3 * w, 1, 128)
    pos = torch.arange(3 * w, dtype=I32, device="cuda")
    kp, vp = (torch.zeros((pages, 24, 1, 128), dtype=BF, device="cuda") for _ in range(2))
    qo = torch.empty_like(q)
    pg = st.make_pages(pages, 24, table.cuda(), _ints(rows), max_new=w)
    st.stlite_paged_append(q, k, v, pos, st.make_rope(), pg, qo, kp, vp)
    wq, wk = st.rotate_qk(q, k, pos, st.make_rope())
    assert torch.equal(qo, wq)
    for s, n in enumerate(rows):
        assert torch.equal(ref.rows_of(kp, table[s], n)[-w:], wk[s * w:s * w + w])
        assert torch.equal(ref.rows_of(vp, table[s], n)[-w:], v[s * w:s * w + w])
        assert not ref.rows_of(vp, table[s], n)[:-w].any()


def test_append_leaves_bad_rows(st):
    """Rows outside a sequence's pages, and pages outside the pool, are not written; q is rotated all the same."""
    g = _gen(5)
    table = torch.tensor([[0, 3], [1, -1], [5, 2], [2, 1]], dtype=I32)  # a pool of 4 pages of 8 rows
    rows = [18, 10, 3, 0]  # row 17 past the table; page -1; page 5; row -1
    q, k, v = _randn(g, 4, 4, 128), _randn(g, 4, 2, 128), _randn(g, 4, 2, 128)
    pos = torch.arange(4, dtype=I32, device="cuda")
    kp, vp = (torch.full((6, 8, 2, 128), 3, dtype=BF, device="cuda") for _ in range(2))
    pg = st.make_pages(4, 8, table.cuda(), _ints(rows))
    qo = torch.zeros_like(q)
    st.stlite_paged_append(q, k, v, pos, st.make_rope(), pg, qo, kp[:4], vp[:4])
    assert (kp == 3).all() and (vp == 3).all()
    assert torch.equal(qo, st.rotate_qk(q, k, pos, st.make_rope())[0])


# ---------------------------------------------------------------- compaction

@pytest.mark.parametrize("n,budget,hkv,page,dtype,layers", [(50, 1, 1, 16, BF, 1), (300, 77, 4, 16, BF, 3),
                                                            (300, 300, 3, 7, F32, 2), (2000, 513, 2, 64, BF, 34),
                                                            (129, 64, 8, 1, F32, 1), (90, 33, 1, 16, BF, 5)])
def test_compact_paged_matches_dense(st, n, budget, hkv, page, dtype, layers):
    g = _gen(n)
    rows = [20, budget, 5]
    table, pages = _table(rows, page, 2)
    io, dense = [], []
    all_idx = torch.empty((layers, hkv, budget), dtype=I32, device="cuda")  # a layer's part on any 4-byte boundary
    for l in range(layers):
        k, v = _randn(g, n, hkv, 128, dtype=dtype), _randn(g, n, hkv, 128, dtype=dtype)
        idx = torch.stack([torch.randperm(n, generator=g)[:budget].sort().values for _ in range(hkv)]).to(I32).cuda()
        kp, vp = (torch.full((pages, page, hkv, 128), 2, dtype=dtype, device="cuda") for _ in range(2))
        all_idx[l] = idx
        io.append((k, v, kp, vp, all_idx[l]))
        ko, vo = torch.empty((budget, hkv, 128), dtype=dtype, device="cuda"), torch.empty((budget, hkv, 128), dtype=dtype, device="cuda")
        q = torch.zeros((1, hkv, 128), dtype=dtype, device="cuda")
        st.stlite_compact(q, k, v, budget, idx, ko, vo)
        dense.append((ko, vo))
    pg = st.make_pages(pages, page, table.cuda())
    st.stlite_compact_paged(io, budget, pg, 1)
    for (_, _, kp, vp, _), (ko, vo) in zip(io, dense):
        for pool, want in ((kp, ko), (vp, vo)):
            assert torch.equal(ref.rows_of(pool, table[1], budget), want)
            # nothing else: the other pages and the end of the last one
            written = torch.full_like(pool, 2)
            flat = written.view(-1, hkv, 128)
            slots = [int(table[1, r // page]) * page + r % page for r in range(budget)]
            flat[slots] = want
            assert torch.equal(pool, written)


def test_compact_paged_refuses_unlike_layers(st):
    def layer(n=20, hkv=2, pages=4, dtype=BF, budget=5):
        k = torch.zeros((n, hkv, 128), dtype=dtype, device="cuda")
        kp = torch.zeros((pages, 8, hkv, 128), dtype=dtype, device="cuda")
        return k, k.clone(), kp, kp.clone(), torch.zeros((hkv, budget), dtype=I32, device="cuda")

    pg = st.make_pages(4, 8, torch.zeros((1, 2), dtype=I32, device="cuda"))
    st.stlite_compact_paged([layer(), layer()], 5, pg, 0)
    good = layer()
    bad = [layer(n=19), layer(pages=3), layer(budget=4), layer(hkv=1), (good[0].cpu(), *good[1:]),
           (good[0], good[1].cpu(), *good[2:]), (*good[:4], good[4].cpu()),
           (good[0].transpose(0, 1).contiguous().transpose(0, 1), *good[1:])]
    for other in bad:
        for io in ([layer(), other], [other, layer()]):
            with pytest.raises((ValueError, st.StliteError)):
                st.stlite_compact_paged(io, 5, pg, 0)
    with pytest.raises(st.StliteError):
        st.stlite_compact_paged([layer(n=20, budget=17)], 17, pg, 0)  # the sequence's table has 16 rows


def test_compact_paged_leaves_bad_rows_and_reads_host_values(st):
    g = _gen(1)
    k = _randn(g, 40, 2, 128)
    v = torch.randn((40, 2, 128), generator=g).to(BF).pin_memory()
    idx = torch.tensor([[0, -1, 5, 39], [3, 40, 7, 8]], dtype=I32, device="cuda")
    table = torch.tensor([[2, 9]], dtype=I32)  # rows 2, 3 on a page outside the pool
    kp, vp = (torch.full((5, 2, 2, 128), 4, dtype=BF, device="cuda") for _ in range(2))
    st.stlite_compact_paged([(k, v, kp, vp, idx)], 4, st.make_pages(5, 2, table.cuda()), 0)
    torch.cuda.synchronize()
    want_k, want_v = torch.full_like(kp, 4), torch.full_like(vp, 4)
    for pool, src in ((want_k, k), (want_v, v.cuda())):
        pool[2, 0, 0], pool[2, 0, 1] = src[0, 0], src[3, 1]
    assert torch.equal(kp, want_k) and torch.equal(vp, want_v)


@pytest.mark.parametrize("make", [lambda: synth.scaled("traj50", 3, beta=0.2), lambda: synth.tiny_ref()],
                         ids=["bf16", "fp32"])
def test_compress_into_pages_equals_dense(st, make):
    wl = make()
    q, k, v = to_device(wl)
    prm = st.make_params(wl.beta)
    ko, vo, idx = st.compress_layer(q, k, v, wl.frames, beta=wl.beta)
    b, hkv = ko.shape[0], k.shape[1]
    table, pages = _table([5, b], 16, 3)
    kp, vp = (torch.zeros((pages, 16, hkv, 128), dtype=k.dtype, device="cuda") for _ in range(2))
    idx2 = torch.empty_like(idx)
    ws = st.workspace(st.make_shape(q, k), wl.frames, prm)
    got = st.stlite_compress_layers_paged([(q, k, v, kp, vp, idx2)], wl.frames, prm,
                                          st.make_pages(pages, 16, table.cuda()), 1, ws)
    assert got == b and torch.equal(idx, idx2)
    assert torch.equal(ref.rows_of(kp, table[1], b), ko) and torch.equal(ref.rows_of(vp, table[1], b), vo)
    assert st.stlite_device_status(ws) == st.STLITE_OK


def test_compress_into_pages_captured(st):
    """The fused pass into two sequences' pages, 34 layers, captured and replayed on new contents."""
    wl = synth.scaled("traj50", 2, beta=0.2)
    q, k, v = to_device(wl)
    prm, b, hkv = st.make_params(wl.beta), st.stlite_budget(k.shape[0], wl.beta), k.shape[1]
    table, pages = _table([b, b], 16, 4)
    pg = st.make_pages(pages, 16, table.cuda())
    layers = 34
    ks, vs = (torch.stack([x] * layers) for x in (k, v))
    kp, vp = (torch.zeros((layers, pages, 16, hkv, 128), dtype=BF, device="cuda") for _ in range(2))
    idx = torch.empty((layers, hkv, (b + 3) // 4 * 4), dtype=I32, device="cuda")  # every layer's on 16 bytes
    io = [(q, ks[l], vs[l], kp[l], vp[l], idx[l]) for l in range(layers)]
    ws = torch.zeros(layers * st.stlite_workspace_size(st.make_shape(q, k), wl.frames, prm), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def both(stream):
        for seq in (0, 1):
            st.stlite_compress_layers_paged(io, wl.frames, prm, pg, seq, ws, stream)

    both(side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both(side)
    for l in range(layers):
        ks[l].copy_(k.roll(l, 0))
        vs[l].copy_(v.roll(l, 0))
    kp.zero_()
    vp.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for l in (0, 1, 31, 32, 33):
        ko, vo, _ = st.compress_layer(q, ks[l], vs[l], wl.frames, beta=wl.beta)
        for seq in (0, 1):
            assert torch.equal(ref.rows_of(kp[l], table[seq], b), ko)
            assert torch.equal(ref.rows_of(vp[l], table[seq], b), vo)
    assert st.stlite_device_status(ws) == st.STLITE_OK


# ----------------------------------------------------------------- attention

def _attention_case(st, rows, cu, page, hq, hkv, dtype, seed, w=None, scale=1.0, garbage=float("nan")):
    """Pools whose unused rows are garbage, and the call's arguments."""
    g = _gen(seed)
    table, pages = _table(rows, page, seed)
    kp, vp = (torch.full((pages, page, hkv, 128), garbage, dtype=dtype, device="cuda") for _ in range(2))
    for s, n in enumerate(rows):
        for pool in (kp, vp):
            fill = _randn(g, n, hkv, 128, dtype=dtype)
            for i in range(0, n, page):
                part = fill[i:i + page]
                pool[int(table[s, i // page]), :len(part)] = part
    n = cu[-1]
    q = (torch.randn((n, hq, 128), generator=g) * scale).to(dtype).cuda()
    uniform = [b - a for a, b in zip(cu, cu[1:])]
    same = len(set(uniform)) == 1
    pg = st.make_pages(pages, page, table.cuda(), _ints(rows), None if same and w is None else _ints(cu),
                       w or max(uniform))
    return q, kp, vp, pg, table


def _attend(st, q, kp, vp, pg):
    ws = st.paged_workspace(q, kp, pg)
    out = torch.full_like(q, 11)
    st.stlite_paged_attention(q, kp, vp, pg, out, ws)
    torch.cuda.synchronize()
    return out, ws


def _check(out, q, kp, vp, table, rows, cu, w=None, **kw):
    r, b = ref.attention(q, kp, vp, table, rows, cu, w, **kw)
    done = ~r[:, 0, 0].isnan()
    ref.within(out[done.cuda()], r[done], b[done])
    assert (out[~done.cuda()] == 11).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("hq,hkv,page", [(28, 4, 16), (12, 2, 64), (16, 1, 7), (3, 3, 1), (40, 8, 24), (9, 1, 100)])
@pytest.mark.parametrize("rows,new", [([1], 1), ([257], 1), ([1000, 3, 0, 64, 65, 15, 16, 17], 1),
                                      ([5, 2, 300], 4), ([129, 40], 8), ([33, 300], 16)])
def test_attention_matches(st, dtype, hq, hkv, page, rows, new):
    cu = [new * i for i in range(len(rows) + 1)]
    q, kp, vp, pg, table = _attention_case(st, rows, cu, page, hq, hkv, dtype, sum(rows) + page)
    out, ws = _attend(st, q, kp, vp, pg)
    _check(out, q, kp, vp, table, rows, cu)
    assert st.stlite_device_status(ws) == st.STLITE_OK


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,new,w", [([300, 12, 0, 5000, 31], [2, 0, 3, 5, 1], 5), ([40, 700], [0, 16], 16),
                                        ([64, 64, 64], [4, 1, 6], 3), ([200], [0], 2), ([9] * 300, [1] * 300, 1), ([5, 20] * 600, [0, 1] * 600, 2)])
def test_attention_ragged(st, dtype, rows, new, w):
    """cu_new: any number of new tokens; those past w of a sequence are left alone."""
    cu = [sum(new[:i]) for i in range(len(new) + 1)]
    q, kp, vp, pg, table = _attention_case(st, rows, cu + [], 16, 14, 2, dtype, len(rows) + w, w) if cu[-1] else \
        _attention_case(st, rows, [0, 1], 16, 14, 2, dtype, 5, w)
    if not cu[-1]:  # a batch with no new token at all, padding only
        pg = st.make_pages(pg.c.n_pages, 16, pg.table, pg.length, _ints(cu), w)
        out, _ = _attend(st, q, kp, vp, pg)
        assert (out == 11).all()
        return
    pad = torch.zeros((3, 14, 128), dtype=dtype, device="cuda")
    q = torch.cat([q, pad])
    out, ws = _attend(st, q, kp, vp, pg)
    _check(out, q, kp, vp, table, rows, cu, w)
    assert st.stlite_device_status(ws) == st.STLITE_OK


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("seqs,most,hq,hkv,w,page", [(330, 60, 4, 4, 1, 16), (700, 35, 2, 2, 2, 7), (250, 300, 8, 8, 1, 64),
                                                     (1300, 16, 14, 1, 1, 16), (64, 900, 8, 4, 1, 32)])
def test_attention_many_short(st, dtype, seqs, most, hq, hkv, w, page):
    """So many sessions that items are not split, or are a warp's each; idle ones and ones without a token among them."""
    r = random.Random(seqs)
    rows = [r.choice([0, 1, r.randint(1, most), r.randint(1, most), most]) for _ in range(seqs)]
    new = [r.randint(0, w) if w > 1 else 1 for _ in range(seqs)]
    cu = [sum(new[:i]) for i in range(seqs + 1)]
    q, kp, vp, pg, table = _attention_case(st, rows, cu, page, hq, hkv, dtype, seqs, w)
    out, ws = _attend(st, q, kp, vp, pg)
    _check(out, q, kp, vp, table, rows, cu, w)
    assert st.stlite_device_status(ws) == st.STLITE_OK


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_long_and_last_rows_count(st, dtype):
    """Long caches of several sequences; large values in the first and the last row alone."""
    rows, hq, hkv = [20011, 7003, 1], 8, 2
    cu = [0, 2, 4, 6]
    q, kp, vp, pg, table = _attention_case(st, rows, cu, 16, hq, hkv, dtype, 77)
    for s, n in enumerate(rows):
        for r in {0, n - 1}:
            vp[int(table[s, r // 16]), r % 16] *= n
    out, _ = _attend(st, q, kp, vp, pg)
    _check(out, q, kp, vp, table, rows, cu)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_extreme_scores(st, dtype):
    """Scores of thousands (one row takes all the weight), and keys of -inf."""
    rows, cu = [500, 90], [0, 1, 2]
    q, kp, vp, pg, table = _attention_case(st, rows, cu, 16, 8, 2, dtype, 5, scale=300.0)
    out, _ = _attend(st, q, kp, vp, pg)
    _check(out, q, kp, vp, table, rows, cu)
    assert torch.isfinite(out).all()
    q[:] = q.abs() + 0.1
    kp[int(table[1, 0]), 2:5] = -torch.inf  # rows 2, 3, 4 of sequence 1 score -inf: weight 0
    q[1] = q[1] / 300
    out, _ = _attend(st, q, kp, vp, pg)
    keep = [i for i in range(90) if i not in (2, 3, 4)]
    kk, vv = (ref.rows_of(p, table[1], 90).cpu().double()[keep] for p in (kp, vp))
    for g in range(8):
        p = torch.softmax(kk[:, g // 4] @ q[1, g].cpu().double() / 128 ** 0.5, 0)
        want = p @ vv[:, g // 4]
        assert ((out[1, g].cpu().double() - want).abs() <= 0.01 * (p @ vv[:, g // 4].abs())).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("hq,hkv,new", [(4, 2, 3), (6, 2, 5), (7, 1, 3), (12, 2, 5), (16, 1, 8)])
@pytest.mark.parametrize("length", [5, 18, 400, 2003])
def test_attention_no_numbers_in_masked_rows(st, dtype, hq, hkv, new, length):
    """A newer token's key and value may hold anything: the older tokens do not see them.  The newest does."""
    rows, cu = [length, 40], [0, new, 2 * new]
    q, kp, vp, pg, table = _attention_case(st, rows, cu, 16, hq, hkv, dtype, length + new)
    clean, _ = _attend(st, q, kp, vp, pg)
    for j, x in ((length - 1, float("nan")), (length - 2, float("inf"))):
        at = int(table[0, j // 16]), j % 16
        vp[at][0, 5] = x
        kp[at][hkv - 1, 7] = x
    out, _ = _attend(st, q, kp, vp, pg)
    older, spoilt = [i for i in range(2 * new) if i not in (new - 1, new - 2)], out[new - 1]
    r, b = ref.attention(q, kp, vp, table, rows, cu)
    assert not r[older].isnan().any()
    ref.within(out[older], r[older], b[older])
    assert (out[older].float() - clean[older].float()).abs().max() <= 2 ** -6 * clean.float().abs().max()
    assert spoilt[:, 5].float().isnan()[: hq // hkv].all()  # the newest token sees the NaN of its own value
    assert out[new - 2, 0, 5].float().isinf() or out[new - 2, 0, 5].float().isnan()


def test_attention_bad_pages_and_lengths(st):
    """A page outside the pool: its rows are left out and the workspace says so; a length past the table too."""
    rows, cu = [100, 50], [0, 1, 2]
    q, kp, vp, pg, table = _attention_case(st, rows, cu, 16, 8, 2, BF, 21)
    for bad in (-1, pg.c.n_pages, 2 ** 31 - 1, -2 ** 31):
        t2 = table.clone()
        t2[0, 2] = bad
        p2 = st.make_pages(pg.c.n_pages, 16, t2.cuda(), pg.length)
        out, ws = _attend(st, q, kp, vp, p2)
        _check(out, q, kp, vp, t2, rows, cu)
        assert st.stlite_device_status(ws) == st.STLITE_EINVAL
        assert st.stlite_device_status(ws) == st.STLITE_OK  # cleared
    t2 = table.clone()
    t2[1] = -3  # no page of sequence 1 exists: zeros
    out, ws = _attend(st, q, kp, vp, st.make_pages(pg.c.n_pages, 16, t2.cuda(), pg.length))
    assert not out[1].any() and st.stlite_device_status(ws) == st.STLITE_EINVAL
    for lens in ([100, 113], [2 ** 31 - 1, 50], [-5, 50]):
        short = st.make_pages(pg.c.n_pages, 16, table.cuda(), _ints(lens))
        eff = [max(0, min(n, 112)) for n in lens]
        if eff[0] == 112 or eff[1] == 112:
            kp, vp = kp.nan_to_num(0.5), vp.nan_to_num(0.25)
            t2 = table.clone()
            t2[1, 4:] = t2[0, :3]
            short = st.make_pages(pg.c.n_pages, 16, t2.cuda(), _ints(lens))
        out, ws = _attend(st, q, kp, vp, short)
        _check(out, q, kp, vp, short.table, eff, cu)
        assert st.stlite_device_status(ws) == st.STLITE_EINVAL


def test_attention_shared_pages(st):
    """Two sequences may read the same pages (a shared prefix): equal queries, equal bits."""
    rows, cu = [200, 200], [0, 1, 2]
    q, kp, vp, pg, table = _attention_case(st, rows, cu, 16, 8, 2, BF, 22)
    t2 = table.clone()
    t2[1] = t2[0]
    q[1] = q[0]
    out, _ = _attend(st, q, kp, vp, st.make_pages(pg.c.n_pages, 16, t2.cuda(), pg.length))
    _check(out, q, kp, vp, t2, rows, cu)


def test_attention_past_32_bit_offsets(st):
    """Pages whose elements lie beyond 2^31 and bytes beyond 2^32 of the pool; append and compaction too."""
    page, hkv = 64, 8
    pages = (2 ** 31 // (page * hkv * 128)) + 40
    kp, vp = (torch.empty((pages, page, hkv, 128), dtype=BF, device="cuda") for _ in range(2))
    g = _gen(9)
    rows = [130]
    table = torch.tensor([[pages - 1, 0, pages - 20]], dtype=I32)
    for p in table[0].tolist():
        kp[p], vp[p] = _randn(g, page, hkv, 128), _randn(g, page, hkv, 128)
    q, k, v = _randn(g, 1, 8, 128), _randn(g, 1, hkv, 128), _randn(g, 1, hkv, 128)
    pg = st.make_pages(pages, page, table.cuda(), _ints(rows))
    pos = _ints([129])
    st.stlite_paged_append(q, k, v, pos, st.make_rope(), pg, q, kp, vp)
    assert torch.equal(vp[pages - 20, 1], v[0])
    out, _ = _attend(st, q, kp, vp, pg)
    _check(out, q, kp, vp, table, rows, [0, 1])
    kd, idx = _randn(g, 130, hkv, 128), torch.arange(130, dtype=I32, device="cuda").repeat(hkv, 1)
    st.stlite_compact_paged([(kd, kd, kp, vp, idx)], 130, pg, 0)
    assert torch.equal(ref.rows_of(kp, table[0], 130), kd) and torch.equal(ref.rows_of(vp, table[0], 130), kd)


def test_attention_repeats_its_bits(st):
    rows = [3000, 17, 900, 12000]
    q, kp, vp, pg, _ = _attention_case(st, rows, [0, 1, 2, 3, 4], 16, 28, 4, BF, 31)
    first, ws = _attend(st, q, kp, vp, pg)
    for _ in range(5):
        out = torch.full_like(q, 11)
        st.stlite_paged_attention(q, kp, vp, pg, out, ws)
        assert torch.equal(out, first)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,hkv,new", [([9000, 40], 2, 1), ([300] * 200, 2, 1), ([700, 0, 5000], 1, 5)])
def test_attention_workspace_of_others(st, dtype, rows, hkv, new):
    """Behind the error word a workspace may hold anything: other calls on the stream share it."""
    cu = [new * i for i in range(len(rows) + 1)]
    q, kp, vp, pg, _ = _attention_case(st, rows, cu, 16, 7 * hkv, hkv, dtype, hkv + new)
    want, ws = _attend(st, q, kp, vp, pg)
    for fill in (0xff, 0x01, 0x7f):
        ws[256:] = fill
        out = torch.full_like(q, 11)
        st.stlite_paged_attention(q, kp, vp, pg, out, ws)
        assert torch.equal(out, want)
    assert st.stlite_device_status(ws) == st.STLITE_OK


def test_attention_on_a_side_stream_and_in_graphs(st):
    """A call on a stream of its own; one capture replayed as the cache grows; two captures sharing a workspace."""
    rows = [40, 700]
    q, kp, vp, pg, table = _attention_case(st, [60, 720], [0, 1, 2], 16, 8, 2, BF, 41)
    pg.length.copy_(_ints(rows))
    ws = st.paged_workspace(q, kp, pg)
    q2 = q.flip(0).contiguous()
    outs = [torch.empty_like(q) for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        st.stlite_paged_attention(q, kp, vp, pg, outs[0], ws)
    side.synchronize()
    _check(outs[0], q, kp, vp, table, rows, [0, 1, 2])
    graphs = []
    for x, o in ((q, outs[0]), (q2, outs[1])):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=side):
            st.stlite_paged_attention(x, kp, vp, pg, o, ws, stream=side)
        graphs.append(gr)
    for step in range(4):
        now = [r + 5 * step for r in rows]
        pg.length.copy_(_ints(now))
        graphs[0].replay()
        graphs[1].replay()
        graphs[0].replay()
        torch.cuda.synchronize()
        _check(outs[0], q, kp, vp, table, now, [0, 1, 2])
        _check(outs[1], q2, kp, vp, table, now, [0, 1, 2])
    assert st.stlite_device_status(ws) == st.STLITE_OK


# ------------------------------------------------------------------ together

def test_serving_steps(st):
    """Two sessions as a server runs them: the prompt's q and k rotated, the cache compressed into pages, then
    tokens appended and attended to, drafts among them; against the same in 64 bits."""
    hq, hkv, page = 28, 4, 16
    frames = ([0, 140], [10, 10], [12, 12])
    g = _gen(51)
    rope, freq = st.make_rope(1e6, (16, 24, 24)), ref.default_freq(1e6)
    n, beta = 280, 0.3
    b = st.stlite_budget(n, beta)
    table, pages = _table([b + 12, b + 12], page, 6)
    kp, vp = (torch.full((pages, page, hkv, 128), float("nan"), dtype=BF, device="cuda") for _ in range(2))
    lens = _ints([b, b])
    plain = []  # each session's (keys, values) in 64 bits, as cached
    for s in range(2):
        x = _randn(g, n, hq + 2 * hkv, 128)
        pos = torch.arange(n, dtype=I32).repeat(3, 1).cuda()
        q, k = st.rotate_qk(x[:, :hq], x[:, hq:hq + hkv], pos, rope)
        v = x[:, hq + hkv:].contiguous()
        win = q[-32:].contiguous()
        idx = torch.empty((hkv, b), dtype=I32, device="cuda")
        prm = st.make_params(beta)
        ws = st.workspace(st.make_shape(win, k), frames, prm)
        st.stlite_compress_layers_paged([(win, k, v, kp, vp, idx)], frames, prm,
                                        st.make_pages(pages, page, table.cuda()), s, ws)
        at = idx.long().t()[..., None].expand(-1, -1, 128)
        plain.append([k.gather(0, at).cpu().double(), v.gather(0, at).cpu().double()])
    ws = None
    t = n
    for new in ([1, 1], [1, 1], [3, 3], [2, 2]):
        total, w = sum(new), new[0]
        x = _randn(g, total, hq + 2 * hkv, 128)
        q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
        pos = torch.tensor([t + i for m in new for i in range(m)], dtype=I32).repeat(3, 1)
        lens += w
        pg = st.make_pages(pages, page, table.cuda(), lens, max_new=w)
        qo = torch.empty((total, hq, 128), dtype=BF, device="cuda")
        st.stlite_paged_append(q, k, v, pos.cuda(), rope, pg, qo, kp, vp)
        out = torch.empty_like(qo)
        ws = st.paged_workspace(qo, kp, pg)
        st.stlite_paged_attention(qo, kp, vp, pg, out, ws)
        rk, bk = ref.rotate(k, pos, freq, (16, 24, 24))
        rq, bq = ref.rotate(q, pos, freq, (16, 24, 24))
        ref.within(qo, rq, bq)
        for s in range(2):
            mine = slice(s * w, s * w + w)
            plain[s][0] = torch.cat([plain[s][0], rk[mine].to(BF).double()])
            plain[s][1] = torch.cat([plain[s][1], v[mine].cpu().double()])
            for i in range(w):
                sees = plain[s][0].shape[0] - (w - 1 - i)
                for h in range(hq):
                    kk, vv = plain[s][0][:sees, h // 7], plain[s][1][:sees, h // 7]
                    p = torch.softmax(kk @ qo[s * w + i, h].cpu().double() / 128 ** 0.5, 0)
                    # a key rounded to the other neighbour (where 64 bits and fp32 fall apart) moves a score by
                    # 2^-8 of one product, far below the rounding of the result
                    tol = 2 ** -8 * (p @ vv).abs() + 2 ** -8 * (p @ vv.abs())
                    assert ((out[s * w + i, h].cpu().double() - p @ vv).abs() <= tol).all()
        t += w
    assert st.stlite_device_status(ws) == st.STLITE_OK
