"""Infinite values in rows that a token sees: its result is that infinity, as
the formula says, and the other dimensions are as without it."""
import pytest
import torch

import paged_ref as ref
from test_paged_gpu import BF, F32, _attend, _attention_case, st  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("hq,hkv,new", [(4, 2, 1), (7, 1, 2), (14, 2, 3), (7, 1, 4), (7, 1, 5)])
@pytest.mark.parametrize("length", [9, 17, 400, 6003])
def test_attention_infinite_values(st, dtype, hq, hkv, new, length):
    rows, cu = [length, 30, length], [0, new, 2 * new, 3 * new]
    q, kp, vp, pg, table = _attention_case(st, rows, cu, 16, hq, hkv, dtype, length + new)
    seen = [(0, 0, 5, 1.0), (length - new, 0, 9, -1.0), (3, hkv - 1, 70, 1.0), (2, hkv - 1, 70, 1.0), (1, 0, 127, -1.0)]
    for s in (0, 2):
        for j, h, dim, sign in seen:
            vp[int(table[s, j // 16]), j % 16, h, dim] = 0
    r, b = ref.attention(q, kp, vp, table, rows, cu)
    for s in (0, 2):
        for j, h, dim, sign in seen:
            vp[int(table[s, j // 16]), j % 16, h, dim] = sign * torch.inf
    out, ws = _attend(st, q, kp, vp, pg)
    finite = torch.ones(out.shape, dtype=torch.bool)
    for s in (0, 2):
        for j, h, dim, sign in seen:
            at = slice(s * new, s * new + new), slice(h * hq // hkv, (h + 1) * hq // hkv), dim
            assert (out[at] == sign * torch.inf).all(), (s, j, h, dim)
            finite[at] = False
    ref.within(out.cpu()[finite], r[finite], b[finite])
    assert st.stlite_device_status(ws) == st.STLITE_OK


def test_attention_one_row_of_infinities(st):
    """One row has all the weight, exactly one."""
    for dtype in (BF, F32):
        q, kp, vp, pg, table = _attention_case(st, [1], [0, 1], 16, 7, 1, dtype, 3)
        row = vp[int(table[0, 0]), 0, 0]
        row[::2], row[1::4] = torch.inf, -torch.inf
        out, _ = _attend(st, q, kp, vp, pg)
        assert torch.equal(out[0], row.expand(7, 128))
