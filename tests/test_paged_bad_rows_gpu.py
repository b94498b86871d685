"""Rows that a table names wrongly, in every way the attention divides its
work: parts of items that have no row left, whole long sessions, batches of
fewer and of more items than there are thread blocks; and equal bits on every
repeat."""
import pytest
import torch

from test_paged_gpu import BF, F32, _attend, _attention_case, _check, _ints, st  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

LONG_AND_SHORT = [12000, 9000] + [30 + 7 * i % 571 for i in range(198)]
# (rows, new tokens each, Hq, Hkv): items whole, divided and described by item, divided and described by block
BATCHES = [([230, 97, 16], 1, 8, 2), ([9000, 40, 5000], 1, 14, 2), ([7000, 700], 5, 6, 2), (LONG_AND_SHORT, 1, 4, 2),
           (LONG_AND_SHORT, 2, 8, 2)]
IDS = ["whole", "by item", "by item, drafts", "by block", "by block, drafts"]


def _call(st, batch, dtype, seed=3):
    rows, new, hq, hkv = batch
    cu = [new * i for i in range(len(rows) + 1)]
    return (rows, cu) + _attention_case(st, rows, cu, 16, hq, hkv, dtype, seed)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("batch", BATCHES, ids=IDS)
def test_attention_bad_pages_everywhere(st, dtype, batch):
    rows, cu, q, kp, vp, pg, table = _call(st, batch, dtype)
    count = [-(-n // 16) for n in rows]

    def attend(change, bad=True):
        t = table.clone()
        change(t)
        out, ws = _attend(st, q, kp, vp, st.make_pages(pg.c.n_pages, 16, t.cuda(), pg.length, max_new=pg.max_new))
        _check(out, q, kp, vp, t, rows, cu)
        assert st.stlite_device_status(ws) == (st.STLITE_EINVAL if bad else st.STLITE_OK)
        return out

    def run_of_pages(t):  # the middle of the longest: more than a block's share of the work
        t[0, count[0] // 4:3 * count[0] // 4] = pg.c.n_pages

    def ends(t):
        for s in range(len(rows)):
            t[s, 0] = -1
            t[s, count[s] - 1] = 2 ** 31 - 1

    def longest(t):
        t[0] = -2 ** 31

    def everything(t):
        t[:] = pg.c.n_pages + 5

    attend(lambda t: None, bad=False)
    attend(run_of_pages)
    attend(ends)
    gone = attend(longest)
    assert not gone[:cu[1]].any()
    assert not attend(everything).any()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("batch", BATCHES, ids=IDS)
def test_attention_repeats_its_bits_in_every_form(st, dtype, batch):
    _, _, q, kp, vp, pg, _ = _call(st, batch, dtype, seed=8)
    first, ws = _attend(st, q, kp, vp, pg)
    for _ in range(5):
        out = torch.full_like(q, 11)
        st.stlite_paged_attention(q, kp, vp, pg, out, ws)
        assert torch.equal(out, first)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
def test_attention_lengths_past_the_table(st, dtype):
    """A length beyond the table among divided items: as many rows as the table has, and an error."""
    rows, cu, q, kp, vp, pg, table = _call(st, ([9008, 40, 5000], 1, 14, 2), dtype)
    assert table.shape[1] * 16 == 9008
    lens = _ints([9008 + 7, -3, 5000])
    out, ws = _attend(st, q, kp, vp, st.make_pages(pg.c.n_pages, 16, table.cuda(), lens))
    _check(out, q, kp, vp, table, [9008, 0, 5000], cu)
    assert st.stlite_device_status(ws) == st.STLITE_EINVAL
