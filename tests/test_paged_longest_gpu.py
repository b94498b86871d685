"""Sessions of as many rows as a table may have, a few short of 2^31, over pages that
the table names again and again."""
import math

import pytest
import torch

import paged_ref
import q4_ref as ref
from test_paged_gpu import BF, I32, _gen, _ints, _randn, st  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu
PAGE, ENTRIES = 42966, 49981  # 2^31 - 2 rows


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("short", [0, 29, 30])
def test_longest_session(st, q4, short):
    """short: rows that the length is below the table's.  The second session, of three rows, has the tokens after."""
    g, n = _gen(5), PAGE * ENTRIES - short
    table = (torch.arange(ENTRIES, dtype=I32) % 2).repeat(2, 1)
    table[1] = 2
    length = torch.tensor([n, 3], dtype=I32)
    pt = st.make_pages(3, PAGE, table.cuda(), length.cuda())
    k, v = (torch.randn((3 * PAGE, 1, 128), generator=g) for _ in range(2))
    v += torch.tensor([3.0, -1.0, 0.0]).repeat_interleave(PAGE)[:, None, None]
    q = _randn(g, 2, 7, 128)
    if q4:
        p = st.make_q4_pools(3, PAGE, 1)
        idx = torch.arange(3 * PAGE, dtype=I32)[None].cuda()
        rows = st.make_pages(3, PAGE, _ints([[0, 1, 2]]))
        st.stlite_compact_paged_q4([(k.to(BF).cuda(), v.to(BF).cuda(), p, idx)], 3 * PAGE, rows, 0)
        kd, vd = (x.reshape(-1, 128) for x in (ref.dense(p, "k"), ref.dense(p, "v")))
        ws, out = st.paged_q4_workspace(q, p, pt), torch.empty_like(q)
        st.stlite_paged_attention_q4(q, p, pt, out, ws)
    else:
        kp, vp = (x.view(3, PAGE, 1, 128).to(BF).cuda() for x in (k, v))
        kd, vd = (x.cpu().double().view(-1, 128) for x in (kp, vp))
        ws = st.paged_workspace(q, kp, pt)
        out = torch.empty_like(q)
        st.stlite_paged_attention(q, kp, vp, pt, out, ws)
    assert st.stlite_device_status(ws) == st.STLITE_OK
    # how often the first session has each row of the two pages: the last page's end `short` times less
    times = torch.tensor([ENTRIES - ENTRIES // 2, ENTRIES // 2]).repeat_interleave(PAGE).double()
    times[PAGE - short:PAGE] -= 1
    assert int(times.sum()) == n
    s = q.cpu().double() @ kd.t() / math.sqrt(128)
    w = torch.zeros_like(s[0])
    w[:, :2 * PAGE] = times * torch.exp(s[0, :, :2 * PAGE] - s[0, :, :2 * PAGE].amax(-1, keepdim=True))
    few = torch.softmax(s[1, :, 2 * PAGE:2 * PAGE + 3], -1)
    want = torch.stack([(w / w.sum(-1, keepdim=True)) @ vd, few @ vd[2 * PAGE:2 * PAGE + 3]])
    mag = torch.stack([(w / w.sum(-1, keepdim=True)) @ vd.abs(), few @ vd[2 * PAGE:2 * PAGE + 3].abs()])
    # scores and weights as in q4_ref.attention; sums: at least the warps of two CTAs an SM share the session's rows, a
    # product adds 16 of them, cut off to fp32 at worst (2 U), a lane's weights are those of every fourth or eighth (U)
    warps = 4 * 2 * torch.cuda.get_device_properties(0).multi_processor_count
    U, size = paged_ref.U, (q.cpu().double().abs() @ kd.abs().t() / math.sqrt(128)).amax()
    bound = mag * (2 * 264 * U * size + 2 ** -11 + (n / warps * (2 / 16 + 1 / 4) + 400) * U)
    paged_ref.within(out, want, bound)
