"""Tensors of the right size and the wrong shape, type or device, which the
binding of the paged calls refuses before the library sees an address."""
import pytest
import torch

from test_paged_abi import st  # noqa: F401  (fixture)

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32
DEVICE = "on the current CUDA device"


@pytest.fixture
def anywhere(st, monkeypatch):
    """The library's calls, which never come; a CPU tensor gets as far as the check of the devices."""
    for name in ("stlite_paged_append", "stlite_rotate_qk", "stlite_paged_attention", "stlite_compact_paged",
                 "stlite_compress_layers_paged"):
        monkeypatch.setattr(st._lib, name, None)


def _refused(call, *args, match=None, **kw):
    with pytest.raises(ValueError, match=match):
        call(*args, **kw)


def test_positions_by_axis(st, anywhere):
    """Positions of three axes are [3][T] (or as many numbers in one row), not [T][3]."""
    q, k = torch.zeros((5, 4, 128), dtype=BF), torch.zeros((5, 2, 128), dtype=BF)
    three, one = st.make_rope(section=(16, 24, 24)), st.make_rope()

    def rotate(pos, rope, match):
        _refused(st.stlite_rotate_qk, q, k, pos, rope, q.clone(), k.clone(), match=match)

    for shape in ((5, 3), (5, 1, 3), (15, 1), (1, 15), (1, 5, 3)):
        rotate(torch.zeros(shape, dtype=I32), three, "pos is")
    for shape in ((3, 5), (15,), (3, 5, 1), (3, 1, 5)):
        rotate(torch.zeros(shape, dtype=I32), three, DEVICE)
    for shape in ((5,), (1, 5), (5, 1)):  # one order of five numbers
        rotate(torch.zeros(shape, dtype=I32), one, DEVICE)
    for pos in (torch.zeros((3, 5), dtype=I32), torch.zeros(4, dtype=I32)):
        rotate(pos, one, "pos is")
    table = torch.zeros((1, 3), dtype=I32)
    pool = torch.zeros((6, 4, 2, 128), dtype=BF)
    pages = st.make_pages(6, 4, table, torch.zeros(1, dtype=I32), max_new=5)
    for shape, match in (((5, 3), "pos is"), ((3, 5), DEVICE)):
        _refused(st.stlite_paged_append, q, k, k.clone(), torch.zeros(shape, dtype=I32), three, pages, q.clone(), pool,
                 pool.clone(), match=match)


def test_value_pool_has_the_key_pools_shape(st, anywhere):
    q = torch.zeros((2, 4, 128), dtype=BF)
    k = torch.zeros((6, 4, 2, 128), dtype=BF)
    pages = st.make_pages(6, 4, torch.zeros((2, 3), dtype=I32), torch.zeros(2, dtype=I32))
    ws = torch.zeros(64, dtype=torch.uint8)

    def attend(v, match):
        _refused(st.stlite_paged_attention, q, k, v, pages, q.clone(), ws, match=match)

    attend(k.clone(), DEVICE)
    for shape in ((6, 2, 4, 128), (4, 6, 2, 128), (6, 4, 1, 256), (48, 128), (6, 4, 2, 64)):
        attend(torch.zeros(shape, dtype=BF), "page pool")
    for dtype in (torch.float16, torch.int16, F32):
        attend(torch.zeros(k.shape, dtype=dtype), "page pool")


def _compaction_layer(n=20, hkv=2, budget=6):
    k, pool = torch.zeros((n, hkv, 128), dtype=BF), torch.zeros((5, 4, hkv, 128), dtype=BF)
    return dict(k=k, v=k.clone(), k_pages=pool, v_pages=pool.clone(), idx=torch.zeros((hkv, budget), dtype=I32))


# as many bytes as the first layer's, and something else
UNLIKE = [("k", torch.zeros((40, 1, 128), dtype=BF)), ("k", torch.zeros((2, 20, 128), dtype=BF)),
          ("v", torch.zeros((10, 2, 128), dtype=F32)), ("v", torch.zeros((20, 2, 128), dtype=torch.float16)),
          ("k", torch.zeros((20, 2, 128), dtype=torch.int16)), ("k_pages", torch.zeros((5, 2, 4, 128), dtype=BF)),
          ("v_pages", torch.zeros((4, 5, 2, 128), dtype=BF)), ("v_pages", torch.zeros((5, 4, 2, 64), dtype=F32)),
          ("idx", torch.zeros((2, 3), dtype=torch.int64)), ("idx", torch.zeros((2, 6), dtype=F32)),
          ("idx", torch.zeros((6, 2), dtype=I32)), ("idx", torch.zeros(12, dtype=I32))]


@pytest.mark.parametrize("name,other", UNLIKE, ids=lambda x: x if isinstance(x, str) else "%s %s" % (tuple(x.shape), x.dtype))
def test_compaction_layers_are_alike(st, anywhere, name, other):
    pages = st.make_pages(5, 4, torch.zeros((1, 3), dtype=I32))
    good = _compaction_layer()
    _refused(st.stlite_compact_paged, [tuple(good.values())] * 2, 6, pages, 0, match=DEVICE)
    bad = tuple({**good, name: other}.values())
    for layers in ([tuple(good.values()), bad], [bad, tuple(good.values())], [tuple(good.values())] * 3 + [bad]):
        _refused(st.stlite_compact_paged, layers, 6, pages, 0, match="every layer|idx")


FRAMES = ([0], [4], [4])
FUSED = [("q", torch.zeros((1, 8, 128), dtype=BF)), ("q", torch.zeros((2, 2, 128), dtype=F32)),
         ("k", torch.zeros((40, 1, 128), dtype=BF)), ("v", torch.zeros((19, 2, 128), dtype=BF)),
         ("v", torch.zeros((40, 1, 128), dtype=BF)), ("v", torch.zeros((20, 2, 128), dtype=torch.float16)),
         ("v", torch.zeros((20, 2, 64), dtype=F32)), ("k", torch.zeros((2, 20, 128), dtype=BF).transpose(0, 1)),
         ("idx", torch.zeros((2, 4), dtype=I32)), ("idx", torch.zeros((2, 5), dtype=torch.int64)),
         ("idx", torch.zeros((5, 2), dtype=I32).t()), ("k_pages", torch.zeros((5, 2, 4, 128), dtype=BF))]


@pytest.mark.parametrize("name,other", FUSED, ids=lambda x: x if isinstance(x, str) else "%s %s" % (tuple(x.shape), x.dtype))
def test_fused_pass_into_pages_checks_every_layer(st, anywhere, name, other):
    """Five rows of 20 are kept: idx_out has room for [2][5]."""
    pages, prm = st.make_pages(5, 4, torch.zeros((1, 3), dtype=I32)), st.make_params(0.25)
    good = dict(q=torch.zeros((2, 4, 128), dtype=BF), **_compaction_layer(budget=5))
    ws = torch.zeros(64, dtype=torch.uint8)

    def fused(layers, match):
        _refused(st.stlite_compress_layers_paged, layers, FRAMES, prm, pages, 0, ws, match=match)

    fused([tuple(good.values())] * 2, DEVICE)
    fused([tuple({**good, "idx": torch.zeros((2, 8), dtype=I32)}.values())], DEVICE)  # room to spare
    bad = tuple({**good, name: other}.values())
    for layers in ([tuple(good.values()), bad], [tuple(good.values())] * 3 + [bad]):
        fused(layers, "every layer|page pool")


@pytest.mark.gpu
def test_fused_pass_into_pages_wants_one_device(st):
    """A tensor on the host among the others on the device (values may be page-locked there)."""
    prm, b = st.make_params(0.25), 5
    good = {n: t.cuda() for n, t in dict(q=torch.zeros((2, 4, 128), dtype=BF), **_compaction_layer(budget=8)).items()}
    table = torch.tensor([[0, 3, 1]], dtype=I32)
    pages = st.make_pages(5, 4, table.cuda())
    ws = st.workspace(st.make_shape(good["q"], good["k"]), FRAMES, prm)
    call = st.stlite_compress_layers_paged
    assert call([tuple(good.values())], FRAMES, prm, pages, 0, ws) == b
    assert call([tuple({**good, "v": good["v"].cpu().pin_memory()}.values())], FRAMES, prm, pages, 0, ws) == b
    for name in good:
        bad = tuple({**good, name: good[name].cpu()}.values())
        _refused(call, [bad], FRAMES, prm, pages, 0, ws, match=DEVICE)
    _refused(call, [tuple(good.values())], FRAMES, prm, st.make_pages(5, 4, table), 0, ws, match=DEVICE)
    _refused(call, [tuple(good.values())], FRAMES, prm, pages, 0, ws.cpu(), match=DEVICE)
    assert st.stlite_device_status(ws) == st.STLITE_OK
