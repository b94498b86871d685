"""4-bit pages and a step's page tables, on the host: what the entry points
refuse before anything is enqueued, what the binding refuses before the library
sees a pointer, and the plain forms of the GPU tests, by hand."""
import ctypes
import math

import pytest
import torch

import q4_ref as ref
from test_paged_abi import BIG, PAGES, ROPES, TOKENS, _code, _pages, _shape, _tokens, good, st  # noqa: F401  (fixtures)
from test_paged_binding import DEVICE, _refused

BF, F32, I32, U8, E4M3 = torch.bfloat16, torch.float32, torch.int32, torch.uint8, torch.float8_e4m3fn
POOLS = [dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(k=8), dict(v=24), dict(k_scale=4),
         dict(v_scale=12), dict(k_factor=2), dict(v_factor=1)]


def _pools(st, good, **kw):
    f = dict(k=good, v=good, k_scale=good, v_scale=good, k_factor=None, v_factor=None)
    f.update({n: good + v if v else v for n, v in kw.items()})
    return st.Q4PoolsC(*[f[n] for n, _ in st.Q4PoolsC._fields_])


def _layers(st, good, n=1, pools=None, **kw):
    f = dict(q=good, k=good, v=good, idx=good, pools=pools or _pools(st, good))
    f.update(kw)
    return (st.Q4Layer * n)(*[st.Q4Layer(*[f[x] for x, _ in st.Q4Layer._fields_]) for _ in range(n)])


def _calls(st, good, pages, pools=None, layers=None, shape=None):
    """Every call over 4-bit pages, with everything else as it should be."""
    lib, sh, x = st._lib, shape or _shape(st), _tokens(st, good)
    p, io = bytes(pools or _pools(st, good)), layers or _layers(st, good, pools=pools)
    return dict(append=lambda: lib.stlite_paged_append_q4(sh, st.make_rope(), x, pages, good, p, None),
                attend=lambda: lib.stlite_paged_attention_q4(sh, pages, good, p, good, good, 1 << 26, None),
                fetch=lambda: lib.stlite_paged_fetch_q4(sh, pages, 1, io, None),
                compact=lambda: lib.stlite_compact_paged_q4(_shape(st, n=100), 10, pages, 0, 1, io, None))


@pytest.mark.parametrize("kw", PAGES + BIG, ids=str)
def test_pages_refused(st, good, kw):
    pg = _pages(st, good, **kw)
    for name, call in _calls(st, good, pg).items():
        if name != "compact" or not ("len" in kw or "cu_new" in kw):
            assert call() == _code(st, kw), name
    size = ctypes.c_size_t(7)
    assert st._lib.stlite_paged_q4_workspace_size(_shape(st), pg, size) == _code(st, kw) and size.value == 7
    step = st._lib.stlite_pages_step(pg if "cu_new" in kw else _pages(st, good, **{"cu_new": good, **kw}), good, good, good,
                                     good, 5, good, None)
    assert step == _code(st, kw)


@pytest.mark.parametrize("kw", POOLS, ids=str)
def test_pools_refused(st, good, kw):
    for name, call in _calls(st, good, _pages(st, good), _pools(st, good, **kw)).items():
        assert call() == st.STLITE_EINVAL, name


@pytest.mark.parametrize("kw,code", [(dict(n=5), 1), (dict(hq=7), 1), (dict(d=64), 2), (dict(dt=2), 1), (dict(n=0), 1),
                                     (dict(w=0), 1), (dict(n=-1), 1)], ids=str)
def test_shapes_refused(st, good, kw, code):
    for name, call in _calls(st, good, _pages(st, good), shape=_shape(st, **kw)).items():
        if name != "compact":
            assert call() == code, name


def test_attention_refused(st, good):
    sh, pg, lib, p, size = _shape(st), _pages(st, good), st._lib, bytes(_pools(st, good)), ctypes.c_size_t()
    assert lib.stlite_paged_q4_workspace_size(sh, pg, size) == st.STLITE_OK and size.value >= 256
    assert lib.stlite_paged_q4_workspace_size(sh, pg, None) == st.STLITE_EINVAL
    for i in (0, 2, 3):
        for bad in (None, good + 8):
            a = [good, p, good, good]
            a[i] = bad
            assert lib.stlite_paged_attention_q4(sh, pg, *a, size.value, None) == st.STLITE_EINVAL
    assert lib.stlite_paged_attention_q4(sh, pg, good, None, good, good, size.value, None) == st.STLITE_EINVAL
    assert lib.stlite_paged_attention_q4(sh, pg, good, p, good, good, size.value - 1, None) == st.STLITE_EWORKSPACE
    for kw, code in ((dict(w=17, n=68), 2), (dict(hq=34), 2)):
        assert lib.stlite_paged_attention_q4(_shape(st, **kw), pg, good, p, good, good, 1 << 26, None) == code
    # a step without a token looks at nothing else
    none = _pages(st, good, cu_new=good)
    assert lib.stlite_paged_attention_q4(_shape(st, n=0), none, None, None, None, None, 0, None) == st.STLITE_OK


def test_append_refused(st, good):
    lib, sh, pg, p, inv = st._lib, _shape(st), _pages(st, good), bytes(_pools(st, good)), st.STLITE_EINVAL

    def append(rope, x, q_out=good, pools=p, shape=sh, pages=pg):
        return lib.stlite_paged_append_q4(shape, rope, x, pages, q_out, pools, None)

    for change in ROPES:
        rope = st.make_rope()
        change(rope)
        assert append(rope, _tokens(st, good)) == inv
    for kw in TOKENS + [dict(v=None), dict(v=8), dict(v_stride=8)]:
        x = _tokens(st, good, **{n: good + v if n in ("q", "k", "v", "pos", "q_norm", "k_norm") and v else v for n, v in kw.items()})
        assert append(st.make_rope(), x) == inv, kw
    x = _tokens(st, good)
    assert append(None, x) == append(st.make_rope(), None) == append(st.make_rope(), x, None) == inv
    assert append(st.make_rope(), x, good + 8) == append(st.make_rope(), x, pools=None) == inv
    assert append(st.make_rope(), _tokens(st, good, q_stride=8 * 128 + 8)) == inv  # in place, not packed
    assert append(st.make_rope(), None, None, None, _shape(st, n=0), _pages(st, good, cu_new=good)) == st.STLITE_OK


def test_layers_refused(st, good):
    lib, pg = st._lib, _pages(st, good)
    fr, prm = st.FrameSpec([0], [5], [5]), st.make_params(0.5)
    need = st.stlite_workspace_size(st.Shape(100, 8, 2, 128, 1, 0), fr, prm)

    def fused(layers, n=1, pages=pg, seq=0, params=prm, ws=good, size=need):
        return lib.stlite_compress_layers_paged_q4(st.Shape(100, 8, 2, 128, 1, 0), fr.c, params, pages, seq, n, layers, None, ws,
                                                   size, None)

    def compact(layers, n=1, budget=10, seq=0):
        return lib.stlite_compact_paged_q4(_shape(st, n=100), budget, pg, seq, n, layers, None)

    def fetch(layers, n=1):
        return lib.stlite_paged_fetch_q4(_shape(st), pg, n, layers, None)

    ok = _layers(st, good)
    for call in (fused, compact, fetch):
        assert call(ok, 0) == call(ok, -3) == call(None) == st.STLITE_EINVAL
        for field in ("k", "v"):
            for bad in (None, good + 8):
                assert call(_layers(st, good, **{field: bad})) == st.STLITE_EINVAL
        for kw in POOLS:
            assert call(_layers(st, good, pools=_pools(st, good, **kw))) == st.STLITE_EINVAL
    for bad in (None, good + 2):
        assert fused(_layers(st, good, idx=bad)) == compact(_layers(st, good, idx=bad)) == st.STLITE_EINVAL
    assert fused(_layers(st, good, q=None)) == fused(_layers(st, good, idx=good + 4)) == st.STLITE_EINVAL
    for budget, seq in ((0, 0), (101, 0), (81, 0), (10, -1), (10, 4)):
        assert compact(ok, budget=budget, seq=seq) == st.STLITE_EINVAL
    assert fused(ok, seq=4) == fused(ok, params=st.make_params(0.9)) == fused(ok, params=st.make_params(0.0)) == st.STLITE_EINVAL
    assert fused(ok, size=need - 1) == st.STLITE_EWORKSPACE
    assert fetch(None) == st.STLITE_EINVAL
    none = _pages(st, good, cu_new=good)
    assert lib.stlite_paged_fetch_q4(_shape(st, n=0), none, 1, None, None) == st.STLITE_OK
    assert lib.stlite_paged_fetch_q4(_shape(st, n=0), none, 0, None, None) == st.STLITE_EINVAL
    big = _shape(st, n=1 << 20, hq=4096, hkv=4096)
    assert lib.stlite_paged_fetch_q4(big, _pages(st, good, cu_new=good), 1, ok, None) == st.STLITE_EUNSUPPORTED


def test_step_refused(st, good):
    pg, call = _pages(st, good, cu_new=good), st._lib.stlite_pages_step
    assert call(_pages(st, good), good, good, good, good, 5, good, None) == st.STLITE_EINVAL  # nowhere for the sums
    for i in range(5):
        a = [good, good, good, good, good]
        a[i] = good + 2
        assert call(pg, *a[:4], 5, a[4], None) == st.STLITE_EINVAL
    for i in (1, 2, 3):
        a = [good, good, good, good]
        a[i] = None
        assert call(pg, *a, 5, good, None) == st.STLITE_EINVAL
    assert call(pg, good, good, good, good, -1, good, None) == st.STLITE_EINVAL


def test_structs_have_the_headers_layout(st):
    assert ctypes.sizeof(st.Q4PoolsC) == 48 and ctypes.sizeof(st.Q4Layer) == 80 and st.Q4Layer.pools.offset == 32


# ---------------------------------------------------------------- the binding

@pytest.fixture
def anywhere(st, monkeypatch):
    for name in ("stlite_paged_append_q4", "stlite_paged_attention_q4", "stlite_paged_fetch_q4", "stlite_compact_paged_q4",
                 "stlite_compress_layers_paged_q4", "stlite_pages_step"):
        monkeypatch.setattr(st._lib, name, None)


def _tensors(p=6, hkv=2, r=4, scale=E4M3):
    codes, scales = torch.zeros((p, hkv, r, 64), dtype=U8), torch.zeros((p, hkv, r, 8), dtype=U8).view(scale)
    return dict(k=codes, v=codes.clone(), k_scale=scales, v_scale=scales.clone())


def test_pools_are_alike(st):
    t = _tensors()
    f = torch.ones(2)
    for kw in (t, _tensors(scale=U8), {**t, "k_factor": f}, {**t, "v_factor": f, "k_factor": f}):
        st.Q4Pools(**kw)
    for name, bad in (("k", t["k"][:5]), ("v", t["v"].view(6, 4, 2, 64)), ("v", t["v"].view(torch.int8)), ("k", t["k"][..., :32]),
                      ("k", t["k"].transpose(1, 2).contiguous().transpose(1, 2)), ("k_scale", t["v_scale"][..., :4]),
                      ("v_scale", t["v_scale"].view(torch.int8)), ("v_scale", t["v_scale"][:, :1]),
                      ("k_scale", t["v_scale"].view(U8).float()), ("k_factor", torch.ones(3)), ("v_factor", torch.ones(2, dtype=BF)),
                      ("k_factor", torch.ones(4)[::2]), ("k", t["k"].view(6, 2, 256))):
        with pytest.raises(ValueError):
            st.Q4Pools(**{**t, name: bad})
    p = st.make_q4_pools(3, 5, 2, device="cpu")
    assert p.k.shape == (3, 2, 5, 64) and p.v_scale.shape == (3, 2, 5, 8) and p.v_scale.dtype == E4M3


def test_calls_compare_tensors(st, anywhere):
    pages = st.make_pages(6, 4, torch.zeros((2, 3), dtype=I32), torch.zeros(2, dtype=I32))
    pools, other = st.Q4Pools(**_tensors()), [st.Q4Pools(**_tensors(5)), st.Q4Pools(**_tensors(r=8)), st.Q4Pools(**_tensors(hkv=1))]
    q, kv = torch.zeros((2, 4, 128), dtype=BF), torch.zeros((2, 2, 128), dtype=BF)
    pos, rope, ws = torch.zeros(2, dtype=I32), st.make_rope(), torch.zeros(64, dtype=U8)

    def append(match, **kw):
        a = dict(q=q, k=kv, v=kv, pos=pos, rope=rope, pages=pages, q_out=q.clone(), pools=pools)
        _refused(st.stlite_paged_append_q4, match=match, **{**a, **kw})

    append(DEVICE)
    for x in other:
        append("pools", pools=x)
    append("output", q_out=q[:1])
    append("output", q_out=q.float())
    append("v is as k", v=kv.float())
    append("q and k", k=kv.float(), v=kv.float())
    append("pos is", pos=pos.long())

    def attend(match, **kw):
        _refused(st.stlite_paged_attention_q4, match=match, **{**dict(q=q, pools=pools, pages=pages, out=q.clone(), ws=ws), **kw})

    attend(DEVICE)
    for x in other[:2]:
        attend("pools", pools=x)
    attend("q is", q=q.transpose(0, 1))
    attend("output", out=q.float())
    attend("output", out=q[:1])

    def fetch(match, *layers):
        _refused(st.stlite_paged_fetch_q4, list(layers), pages, match=match)

    ok = (pools, kv, kv.clone())
    fetch(DEVICE, ok)
    for x in other:
        fetch("pools", ok, (x, kv, kv))
    for bad in (kv[:1], kv.float(), torch.zeros((2, 4, 64), dtype=BF), kv.transpose(0, 1)):
        fetch("every layer", ok, (pools, kv, bad))
        fetch("every layer", ok, (pools, bad, kv))
    k, idx = torch.zeros((20, 2, 128), dtype=BF), torch.zeros((2, 6), dtype=I32)

    def compact(match, *layers):
        _refused(st.stlite_compact_paged_q4, list(layers), 6, pages, 0, match=match)

    ok = (k, k.clone(), pools, idx)
    compact(DEVICE, ok)
    for x in other:
        compact("pools", ok, (k, k, x, idx))
    for bad in ((k[:10], k, pools, idx), (k, k.float(), pools, idx), (k, k, pools, idx[:, :5]), (k, k, pools, idx.long()),
                (k, k.transpose(0, 1), pools, idx)):
        compact("every layer", ok, bad)
    frames, prm = ([0], [4], [4]), st.make_params(0.25)

    def fused(match, *layers):
        _refused(st.stlite_compress_layers_paged_q4, list(layers), frames, prm, pages, 0, ws, match=match)

    ok = (q, k, k.clone(), pools, idx)
    fused(DEVICE, ok)
    for x in other:
        fused("pools", ok, (q, k, k, x, idx))
    for bad in ((q[:1], k, k, pools, idx), (q, k, k[:10], pools, idx), (q.float(), k, k, pools, idx), (q, k, k, pools, idx[:, :4])):
        fused("every layer", ok, bad)


def test_step_compares_tensors(st, anywhere):
    z = lambda *s: torch.zeros(s, dtype=I32)  # noqa: E731
    pages = st.make_pages(6, 4, z(2, 3), z(2), z(3))

    def step(match, **kw):
        a = dict(pages=pages, keep=z(2), fresh=z(2), free_pages=z(6), n_free=z(1), slot=z(9))
        _refused(st.stlite_pages_step, match=match, **{**a, **kw})

    step(DEVICE)
    step(DEVICE, keep=None, slot=7)
    step("length and cu_new", pages=st.make_pages(6, 4, z(2, 3), z(2)))
    step("length and cu_new", pages=st.make_pages(6, 4, z(2, 3), None, z(3)))
    for bad in (dict(keep=z(3)), dict(keep=z(2).long()), dict(fresh=z(1)), dict(fresh=z(2).float()), dict(fresh=z(4)[::2]),
                dict(free_pages=z(5)), dict(free_pages=z(6).long()), dict(n_free=z(2)), dict(n_free=z(1).long()), dict(slot=z(3, 3)),
                dict(slot=z(9).long()), dict(slot=z(18)[::2]), dict(slot=-1)):
        step("contiguous int32", **bad)


# ----------------------------------------------------- the plain forms by hand

def test_codes_by_hand():
    assert [ref.e4m3(b) for b in (0, 1, 7, 8, 0x38, 0x7e, 0xb8)] == [0.0, 2.0 ** -9, 7 * 2.0 ** -9, 2.0 ** -6, 1.0, 448.0, -1.0]
    assert math.isnan(ref.e4m3(0x7f)) and torch.equal(ref.SCALES.float().nan_to_num(9), torch.arange(256).to(U8).view(E4M3).float().nan_to_num(9))
    x = torch.zeros(128)
    x[:16] = torch.tensor([6.0, -4, 3, 2, 1.5, 1, 0.5, 0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.26])
    x[16:18] = torch.tensor([448 * 6.0 * 3, -448 * 6.0])
    x[32] = 2.0 ** -9 * 5  # below the smallest scale's six
    x[48] = 17 / 16 * 6  # between the scales 1 and 9/8, and 1 is even
    x[49] = 1.0
    c, s = ref.encode(x)
    assert s.tolist() == [0x38, 0x7e, 1, 0x38, 1, 1, 1, 1]
    codes = torch.stack([c & 15, c >> 4], -1).flatten().tolist()
    assert codes[:16] == [7, 14, 5, 4, 3, 2, 1, 0, 0, 2, 2, 4, 4, 6, 6, 9]
    assert codes[16:18] == [7, 15] and codes[32] == 6 and codes[48:50] == [7, 2] and not any(codes[50:])
    d = ref.decode(c, s)
    assert d[:8].tolist() == [6.0, -4, 3, 2, 1.5, 1, 0.5, 0] and d[32] == 2.0 ** -7 and d[16] == 448 * 6.0
    c, s = ref.encode(x, 4.0)
    assert s[0] == 0x28 and ref.decode(c, s, 4.0)[:4].tolist() == [6.0, -4, 3, 2]


def test_step_by_hand():
    """Two sessions of pages of four rows: the first ends and begins anew, the second grows; then too little is left."""
    table, lens, free = [[5, 1, -1], [2, -1, -1]], [7, 3], [0, 3, 4, -9, -9, -9]
    cu, n, slot = ref.step(table, lens, [0, 3], [1, 4], free, 3, 6, 4, 9)
    # free: 0 3 4 5 1; the first takes 1, the second 5
    assert (table, lens, cu, n) == ([[1, 1, -1], [2, 5, -1]], [1, 7], [0, 1, 5], 3)
    assert slot == [4, 11, 20, 21, 22, -1, -1, -1, -1] and free[:3] == [0, 3, 4]
    cu, n, slot = ref.step(table, lens, None, [20, 5], free, 0, 6, 4, 9)  # past the table; a third page, and none is left
    assert cu == [0, 0, 0] and lens == [1, 7] and n == 0 and slot == [-1] * 9
    cu, n, _ = ref.step(table, lens, None, [3, 1], free, 1, 6, 4, 3)  # both fit their pages; places for one
    assert cu == [0, 3, 3] and n == 1
