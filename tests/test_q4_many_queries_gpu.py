"""Attention over 4-bit pages where a head's queries take several reads of a
cache that many CTAs share, so that parts of every chunk are merged."""
import pytest
import torch

import q4_ref as ref
from test_paged_gpu import BF, F32, _gen, st  # noqa: F401  (fixture)
from test_q4_gpu import _attend, _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("hq,hkv,rows,new", [
    (14, 2, [4100, 30, 900], [5, 5, 5]), (8, 2, [3001, 0, 700, 5], [16, 16, 16, 16]), (16, 1, [6000], [16]),
    (12, 2, [2500, 17, 1, 3000], [11, 0, 16, 6]), (16, 1, [300] * 9, [3, 1, 16, 2, 0, 4, 7, 1, 1])])
def test_chunks_of_long_sessions(st, dtype, hq, hkv, rows, new):
    g = _gen(hq + len(rows))
    q, p, pt, table, cu = _attend(st, g, rows, new, 16, hq, hkv, dtype, True, scale=3.0)
    ws, out = st.paged_q4_workspace(q, p, pt), torch.empty_like(q)
    st.stlite_paged_attention_q4(q, p, pt, out, ws)
    assert _check(out, p, q, table, rows, cu).all()
    first = out.clone()
    ws[16:].random_(0, 255)
    st.stlite_paged_attention_q4(q, p, pt, out, ws)
    assert torch.equal(out, first) and st.stlite_device_status(ws) == st.STLITE_OK


@pytest.mark.parametrize("dtype", [BF, F32])
def test_one_chunk_without_a_number(st, dtype):
    """A value without a number in the last row of a long session, which the last token alone sees: its chunk's other
    tokens and the other chunks' have what they had."""
    hq, hkv, n, new = 8, 1, 3000, 16
    q, p, pt, table, cu = _attend(st, _gen(1), [n], [new], 16, hq, hkv, dtype)
    clean = st.paged_attention_q4(q, p, pt)
    at = (int(table[0, (n - 1) // 16]), 0, (n - 1) % 16, 2)
    p.v_scale.view(torch.uint8)[at] = ref.NAN
    got = st.paged_attention_q4(q, p, pt)
    odd = torch.zeros(got.shape, dtype=torch.bool)
    odd[-1, :, 32:48] = True
    assert torch.equal(got.isnan().cpu(), odd) and torch.equal(got.cpu()[~odd], clean.cpu()[~odd])
