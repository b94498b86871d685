"""Serving steps without a token: every sequence may have none, and then the
packed tensors are empty (no address) and the calls do nothing."""
import ctypes
import math

import pytest
import torch

import test_paged_abi as abi
from test_paged_abi import good, st  # noqa: F401  (fixtures)

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def test_no_token_is_no_error(st, good):
    sh, pg, size = abi._shape(st, n=0, w=3), abi._pages(st, good, cu_new=good), ctypes.c_size_t()
    assert st._lib.stlite_paged_workspace_size(sh, pg, size) == st.STLITE_OK and size.value >= 256
    assert st._lib.stlite_paged_attention(sh, pg, None, None, None, None, None, 0, None) == st.STLITE_OK
    assert st._lib.stlite_paged_append(sh, st.make_rope(), None, pg, None, None, None, None) == st.STLITE_OK
    assert st._lib.stlite_paged_append(abi._shape(st, n=0, w=5000), st.make_rope(), None, pg, None, None, None,
                                       None) == st.STLITE_OK


def test_no_token_keeps_the_other_checks(st, good):
    sh, pg = abi._shape(st, n=0), abi._pages(st, good, cu_new=good)
    bad = st.make_rope()
    bad.inv_freq[3] = math.nan

    def both(code, shape=sh, pages=pg, rope=None):
        assert st._lib.stlite_paged_append(shape, rope or st.make_rope(), None, pages, None, None, None, None) == code
        if rope is None:
            assert st._lib.stlite_paged_attention(shape, pages, None, None, None, None, None, 0, None) == code

    both(st.STLITE_EINVAL, pages=abi._pages(st, good, cu_new=good, table=None))
    both(st.STLITE_EINVAL, pages=abi._pages(st, good))  # a token of each sequence, and none given
    both(st.STLITE_EINVAL, rope=bad)
    both(st.STLITE_EINVAL, shape=abi._shape(st, n=0, hq=7))
    both(st.STLITE_EUNSUPPORTED, shape=abi._shape(st, n=0, d=64))
    both(st.STLITE_EINVAL, shape=abi._shape(st, n=-1))
    assert st._lib.stlite_rotate_qk(abi._shape(st, n=-1), st.make_rope(), None, None, None, None) == st.STLITE_EINVAL


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("axes", [1, 3])
def test_no_token_through_the_binding(st, dtype, axes):
    hq, hkv = 4, 2
    q, k = (torch.empty((0, h, 128), dtype=dtype, device="cuda") for h in (hq, hkv))
    pos = torch.empty((axes, 0) if axes == 3 else (0,), dtype=I32, device="cuda")
    rope = st.make_rope(section=(16, 24, 24) if axes == 3 else (64, 0, 0))
    table = torch.zeros((2, 3), dtype=I32, device="cuda")
    lens, cu = torch.tensor([9, 0], dtype=I32, device="cuda"), torch.zeros(3, dtype=I32, device="cuda")
    kp, vp = (torch.full((5, 4, hkv, 128), 3, dtype=dtype, device="cuda") for _ in range(2))
    pages = st.make_pages(5, 4, table, lens, cu, max_new=2)
    norm = torch.ones(128, dtype=dtype, device="cuda")
    qo, ko = st.rotate_qk(q, k, pos, rope, norm)
    assert qo.shape == q.shape and ko.shape == k.shape
    st.stlite_paged_append(q, k, k.clone(), pos, rope, pages, qo, kp, vp, norm, norm)
    ws = st.paged_workspace(qo, kp, pages)
    out = torch.empty_like(qo)
    st.stlite_paged_attention(qo, kp, vp, pages, out, ws)
    assert st.paged_attention(qo, kp, vp, pages).shape == q.shape
    assert (kp == 3).all() and (vp == 3).all() and st.stlite_device_status(ws) == st.STLITE_OK
    side = torch.cuda.Stream()
    assert st.rotate_qk(q, k, pos, rope, stream=side)[1].shape == k.shape
    assert st.paged_attention(qo, kp, vp, pages, stream=side).shape == q.shape
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):  # an empty step among others
        kp.add_(1)
        st.stlite_paged_append(q, k, k, pos, rope, pages, qo, kp, vp)
        st.stlite_paged_attention(qo, kp, vp, pages, out, ws)
    graph.replay()
    torch.cuda.synchronize()
    assert (kp == 4).all() and (vp == 3).all()
