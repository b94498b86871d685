"""Paged caches, on the host: what the entry points refuse before anything is
enqueued, and the plain forms that the GPU tests compare with, by hand."""
import ctypes
import math

import pytest
import torch

import paged_ref
from paper_2603_00188_gb300 import build as pkg_build


@pytest.fixture(scope="module")
def st():
    pkg_build.build()
    from paper_2603_00188_gb300 import stlite
    return stlite


@pytest.fixture(scope="module")
def good():
    """A 16-byte-aligned address that stands for a tensor: device memory larger than anything
    these shapes describe where there is a device (zeros: a valid table, length and cu_new too)."""
    if torch.cuda.is_available():
        buf = torch.zeros(32 << 20, dtype=torch.uint8, device="cuda")
        yield buf.data_ptr()
        del buf
    else:
        yield 0x10000


def _pages(st, good, **kw):
    f = dict(n_seqs=4, n_pages=20, page_rows=16, max_pages=5, table=good, len=good, cu_new=None)
    f.update(kw)
    return bytes(st.Pages(*[f[n] for n, _ in st.Pages._fields_]))


def _tokens(st, good, **kw):
    f = dict(q=good, k=good, v=good, q_stride=0, k_stride=0, v_stride=0, q_norm=None, k_norm=None, eps=1e-6, pos=good)
    f.update(kw)
    return bytes(st.Tokens(*[f[n] for n, _ in st.Tokens._fields_]))


def _shape(st, n=4, hq=8, hkv=2, d=128, w=1, dt=0):
    """As packed bytes, which a pointer argument takes as it takes an address."""
    return bytes(st.Shape(n, hq, hkv, d, w, dt))


PAGES = [dict(n_seqs=0), dict(n_pages=0), dict(page_rows=0), dict(max_pages=-1), dict(table=None), dict(table=2),
         dict(len=None), dict(len=6), dict(cu_new=9)]
BIG = [dict(n_pages=1 << 20, page_rows=1 << 12), dict(n_pages=1, page_rows=1 << 16, max_pages=1 << 16)]


def _code(st, kw):
    return st.STLITE_EUNSUPPORTED if kw in BIG else st.STLITE_EINVAL


@pytest.mark.parametrize("kw", PAGES + BIG, ids=str)
def test_pages_refused(st, good, kw):
    pg, sh = _pages(st, good, **kw), _shape(st)
    size = ctypes.c_size_t(7)
    assert st._lib.stlite_paged_workspace_size(sh, pg, size) == _code(st, kw)
    assert size.value == 7
    assert st._lib.stlite_paged_attention(sh, pg, good, good, good, good, good, 1 << 24, None) == _code(st, kw)
    assert st._lib.stlite_paged_append(sh, st.make_rope(), _tokens(st, good), pg, good, good, good,
                                       None) == _code(st, kw)
    if "len" not in kw and "cu_new" not in kw:
        io = (st.LayerIO * 1)(st.LayerIO(*[good] * 6))
        assert st._lib.stlite_compact_paged(_shape(st, n=100), 10, pg, 0, 1, io, None) == _code(st, kw)


def test_lengths_optional_for_compaction_only(st, good):
    """stlite_compact_paged does not look at len or cu_new: with everything else refused it says so for that."""
    io = (st.LayerIO * 1)(st.LayerIO(*[good] * 6))
    pg = _pages(st, good, len=None)
    for budget, seq, layers, table in ((0, 0, 1, io), (101, 0, 1, io), (81, 0, 1, io), (10, -1, 1, io), (10, 4, 1, io),
                                       (10, 0, 0, io), (10, 0, 1, None)):
        assert st._lib.stlite_compact_paged(_shape(st, n=100), budget, pg, seq, layers, table, None) == st.STLITE_EINVAL
    for field in ("k", "v", "k_out", "v_out", "idx_out"):
        for bad in (None, good + (2 if field == "idx_out" else 8)):
            io = (st.LayerIO * 1)(st.LayerIO(*[good] * 6))
            setattr(io[0], field, bad)
            assert st._lib.stlite_compact_paged(_shape(st, n=100), 10, pg, 0, 1, io, None) == st.STLITE_EINVAL
    fr, prm = st.FrameSpec([0], [5], [5]), st.make_params(0.9)
    need = st.stlite_workspace_size(st.Shape(100, 8, 2, 128, 1, 0), fr, prm)
    io = (st.LayerIO * 1)(st.LayerIO(*[good] * 6))

    def fused(pages, seq, params, layers, ws_bytes):
        return st._lib.stlite_compress_layers_paged(st.Shape(100, 8, 2, 128, 1, 0), fr.c, params, pages, seq, 1, layers, None, good,
                                                    ws_bytes, None)

    assert fused(pg, 0, prm, io, need) == st.STLITE_EINVAL  # 90 rows, 80 in the table
    small = st.make_params(0.5)
    assert fused(pg, 4, small, io, need) == st.STLITE_EINVAL
    assert fused(pg, 0, st.make_params(0.0), io, need) == st.STLITE_EINVAL
    assert fused(pg, 0, small, None, need) == st.STLITE_EINVAL
    assert fused(_pages(st, good, table=None), 0, small, io, need) == st.STLITE_EINVAL
    assert fused(pg, 0, small, io, need - 1) == st.STLITE_EWORKSPACE
    io[0].k_out = None
    assert fused(pg, 0, small, io, need) == st.STLITE_EINVAL


@pytest.mark.parametrize("kw,code", [(dict(n=5), 1), (dict(w=2), 1), (dict(w=17, n=68), 2), (dict(hq=34), 2),
                                     (dict(hq=7), 1), (dict(d=64), 2), (dict(dt=2), 1), (dict(n=0), 1)], ids=str)
def test_attention_shapes_refused(st, good, kw, code):
    size = ctypes.c_size_t()
    assert st._lib.stlite_paged_workspace_size(_shape(st, **kw), _pages(st, good), size) == code
    assert st._lib.stlite_paged_attention(_shape(st, **kw), _pages(st, good), good, good, good, good, good, 1 << 24,
                                          None) == code


def test_attention_sizes_refused(st, good):
    """Block and item numbers that would pass 32 bits."""
    size = ctypes.c_size_t()
    for kw, hkv in ((dict(n_seqs=1 << 10, cu_new=good, max_pages=1 << 12, page_rows=1 << 12, n_pages=100), 8),
                    (dict(n_pages=1 << 24), 8), (dict(n_seqs=1 << 25, cu_new=good), 8),
                    (dict(n_seqs=1 << 29, max_pages=1, cu_new=good), 8)):
        sh = _shape(st, hkv=hkv)
        assert st._lib.stlite_paged_workspace_size(sh, _pages(st, good, **kw), size) == st.STLITE_EUNSUPPORTED
        assert st._lib.stlite_paged_attention(sh, _pages(st, good, **kw), good, good, good, good, good, 1 << 24,
                                              None) == st.STLITE_EUNSUPPORTED


def test_attention_pointers_refused(st, good):
    sh, pg, size = _shape(st), _pages(st, good), ctypes.c_size_t()
    assert st._lib.stlite_paged_workspace_size(sh, pg, size) == st.STLITE_OK and size.value >= 256
    assert st._lib.stlite_paged_workspace_size(sh, pg, None) == st.STLITE_EINVAL
    args = [good] * 5
    for i in range(5):
        for bad in (None, good + 8):
            a = list(args)
            a[i] = bad
            assert st._lib.stlite_paged_attention(sh, pg, *a, size.value, None) == st.STLITE_EINVAL
    assert st._lib.stlite_paged_attention(sh, pg, *args, size.value - 1, None) == st.STLITE_EWORKSPACE


ROPES = [lambda r: setattr(r, "interleaved", 2), lambda r: r.section.__setitem__(0, 63),
         lambda r: r.section.__setitem__(slice(0, 3), [65, -1, 0]), lambda r: r.inv_freq.__setitem__(5, math.nan),
         lambda r: r.inv_freq.__setitem__(63, math.inf),
         lambda r: r.inv_freq.__setitem__(0, -5e9)]
TOKENS = [dict(q=None), dict(k=None), dict(pos=None), dict(q=8), dict(k=24), dict(pos=2), dict(q_norm=8),
          dict(k_norm=4), dict(q_stride=8 * 128 - 8), dict(q_stride=8 * 128 + 4), dict(k_stride=2 * 128 + 1),
          dict(k_stride=-256), dict(q_stride=1 << 41), dict(q_norm=16, eps=math.nan), dict(k_norm=16, eps=-1.0),
          dict(k_norm=16, eps=math.inf)]


def test_rotation_refused(st, good):
    lib, sh, pg = st._lib, _shape(st), _pages(st, good)

    def both(rope, x, code, q_out=good, k_out=good + 4096, shape=sh):
        assert lib.stlite_rotate_qk(shape, rope, x, q_out, k_out, None) == code
        assert lib.stlite_paged_append(shape, rope, x, pg, q_out, k_out, good, None) == code

    inv = st.STLITE_EINVAL
    for change in ROPES:
        rope = st.make_rope()
        change(rope)
        both(rope, _tokens(st, good), inv)
    both(None, _tokens(st, good), inv)
    both(st.make_rope(), None, inv)
    for kw in TOKENS:
        x = _tokens(st, good, **{n: good + v if n in ("q", "k", "pos", "q_norm", "k_norm") and v else v
                                 for n, v in kw.items()})
        both(st.make_rope(), x, inv)
    both(st.make_rope(), _tokens(st, good), inv, q_out=None)
    both(st.make_rope(), _tokens(st, good), inv, q_out=good + 8)
    both(st.make_rope(), _tokens(st, good), inv, k_out=None)
    both(st.make_rope(), _tokens(st, good), inv, shape=_shape(st, n=0))
    both(st.make_rope(), _tokens(st, good), inv, shape=_shape(st, w=0))
    both(st.make_rope(), _tokens(st, good), st.STLITE_EUNSUPPORTED, shape=_shape(st, d=64))
    # more heads of tokens than fit an int32
    both(st.make_rope(), _tokens(st, good), st.STLITE_EUNSUPPORTED, shape=_shape(st, n=200000, hq=40000, hkv=2000,
                                                                                  w=50000))
    # an output that is its input has the output's packing
    both(st.make_rope(), _tokens(st, good, q_stride=8 * 128 + 8), inv, q_out=good)
    assert lib.stlite_rotate_qk(sh, st.make_rope(), _tokens(st, good, k=good + 4096, k_stride=264), good, good + 4096,
                                None) == inv
    for bad in (dict(v=None), dict(v=good + 8), dict(v_stride=8)):
        assert lib.stlite_paged_append(sh, st.make_rope(), _tokens(st, good, **bad), pg, good, good, good, None) == inv
    assert lib.stlite_paged_append(sh, st.make_rope(), _tokens(st, good), pg, good, good, None, None) == inv
    assert lib.stlite_paged_append(_shape(st, n=5), st.make_rope(), _tokens(st, good), pg, good, good, good,
                                   None) == inv
    for base in (0.0, -1.0, math.nan, math.inf):
        assert lib.stlite_rope_init(base, st.Rope()) == inv
    assert lib.stlite_rope_init(1e4, None) == inv


def test_packed_arguments_have_the_structs_layout(st):
    """The binding passes shapes and tokens as packed bytes."""
    assert st._SHAPE.pack(1, 2, 3, 4, 5, 6) == bytes(st.Shape(1, 2, 3, 4, 5, 6))
    x = [1 << 40, 2 << 40, 3 << 40, -4, 5, 6, 7 << 40, 8 << 40, 0.25, 9 << 40]
    assert st._TOKENS.pack(*x) == bytes(st.Tokens(*x))


def test_rope_frequencies(st):
    rope = st.make_rope(1e6, section=(16, 24, 24), interleaved=True)
    for i, f in enumerate(paged_ref.default_freq(1e6)):
        assert abs(rope.inv_freq[i] - f) <= 2 ** -50 * f
    assert list(rope.section) == [16, 24, 24] and rope.interleaved == 1
    assert list(st.make_rope(inv_freq=[0.5 ** i for i in range(64)]).inv_freq)[:3] == [1.0, 0.5, 0.25]
    with pytest.raises(ValueError):
        st.make_rope(inv_freq=[1.0] * 63)


def test_binding_checks_tensors(st):
    """What the binding refuses before the library sees a pointer (CPU tensors: nothing could run)."""
    i32 = torch.int32
    table = torch.zeros((2, 3), dtype=i32)
    ln = torch.zeros(2, dtype=i32)
    for bad in (dict(table=table.long()), dict(table=table.t()), dict(table=table[0]), dict(length=ln[:1]),
                dict(length=torch.zeros(4, dtype=i32)[::2]), dict(cu_new=ln)):
        with pytest.raises(ValueError):
            st.make_pages(6, 4, **{**dict(table=table, length=ln), **bad})
    pages = st.make_pages(6, 4, table, ln)
    x = torch.zeros((2, 4, 128), dtype=torch.bfloat16)
    kv = torch.zeros((2, 2, 128), dtype=torch.bfloat16)
    pool = torch.zeros((6, 4, 2, 128), dtype=torch.bfloat16)
    pos, rope = torch.zeros(2, dtype=i32), st.make_rope()

    def append(**kw):
        a = dict(q=x, k=kv, v=kv, pos=pos, rope=rope, pages=pages, q_out=x.clone(), k_pages=pool, v_pages=pool.clone())
        a.update(kw)
        with pytest.raises(ValueError):
            st.stlite_paged_append(**a)

    append()  # everything fits, but the tensors are on the host
    with pytest.raises(ValueError):
        st.stlite_rotate_qk(x, kv, pos, rope, x.clone(), kv.clone())
    with pytest.raises(ValueError):
        st.stlite_paged_attention(x, pool, pool, pages, x.clone(), ln)
    with pytest.raises(ValueError):
        st.stlite_compact_paged([(kv, kv, pool, pool, torch.zeros((2, 2), dtype=i32))], 2, pages, 0)
    append(k_pages=pool[:5])
    append(v_pages=pool.float())
    append(k_pages=pool.transpose(0, 1).contiguous().transpose(0, 1))
    append(q_out=x[:1])
    append(q_out=x.float())
    append(pos=pos.long())
    append(pos=torch.zeros(3, dtype=i32))
    append(rope=st.make_rope(section=(16, 24, 24)))
    append(v=kv[:, :1])
    append(k=kv.float(), v=kv.float())
    append(q=x.transpose(0, 1))
    append(q_norm=torch.ones(64, dtype=torch.bfloat16))
    append(q_norm=torch.ones(128))
    with pytest.raises(ValueError):
        st.stlite_paged_attention(x, pool, pool, pages, x[:, :2], ln)
    with pytest.raises(ValueError):
        st.stlite_paged_attention(x.transpose(0, 1), pool, pool, pages, x, ln)
    with pytest.raises(ValueError):
        st.stlite_rotate_qk(x, kv, pos, rope, x.clone(), kv[:1])
    idx = torch.zeros((2, 2), dtype=i32)
    for layer in ((kv, kv, pool[:3], pool, idx), (kv, kv, pool, pool, idx[:, :1])):
        with pytest.raises(ValueError):
            st.stlite_compact_paged([layer], 2, pages, 0)


# ----------------------------------------------------- the plain forms by hand

def test_rotation_by_hand():
    """A quarter turn moves (1, 0) to (0, 1); the norm of a constant head is its weights."""
    x = torch.zeros((1, 1, 128))
    x[0, 0, 3] = 1.0
    freq = [0.0] * 64
    freq[3] = math.pi / 2
    y, _ = paged_ref.rotate(x, torch.tensor([1]), freq)
    assert abs(float(y[0, 0, 3 + 64]) - 1) < 1e-15 and abs(float(y[0, 0, 3])) < 1e-15
    y, _ = paged_ref.rotate(x, torch.tensor([[0], [0], [1]]), freq, section=(2, 1, 61))
    assert abs(float(y[0, 0, 67]) - 1) < 1e-15  # pair 3 is on the last axis
    freq[1] = math.pi / 2
    y, _ = paged_ref.rotate(x, torch.tensor([1]), freq, interleaved=True)
    assert abs(float(y[0, 0, 2]) + 1) < 1e-15 and abs(float(y[0, 0, 3])) < 1e-15  # (0, 1) -> (-1, 0)
    w = torch.linspace(0.5, 2, 128)
    y, _ = paged_ref.rotate(torch.full((1, 1, 128), -3.0), torch.tensor([0]), freq, norm=w, eps=0.0)
    assert torch.allclose(y[0, 0], -w.double(), rtol=1e-14)


def test_attention_by_hand():
    """Equal keys give the mean of the visible values; a sequence of none gives zeros."""
    kp, vp = torch.zeros((3, 2, 1, 128)), torch.arange(6.0).view(3, 2, 1, 1).expand(3, 2, 1, 128).contiguous()
    table = torch.tensor([[2, 0], [1, 1]], dtype=torch.int32)
    out, _ = paged_ref.attention(torch.ones((3, 2, 128)), kp, vp, table, [3, 0], [0, 2, 3])
    assert float(out[1, 0, 0]) == (4 + 5 + 0) / 3 and float(out[0, 1, 5]) == 4.5
    assert not out[2].any()
    out, _ = paged_ref.attention(torch.ones((1, 2, 128)), kp, vp, table[:1], [3], [0, 1], skip_pages=(2,))
    assert float(out[0, 0, 0]) == 0.0
