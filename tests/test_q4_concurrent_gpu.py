"""Calls over 4-bit pages made at once: on streams and threads, on values that
stay on the host, on shared pools, and a whole step captured in one graph."""
import threading

import pytest
import torch

import paged_ref
import q4_ref as ref
from test_paged_gpu import BF, F32, I32, _gen, _ints, _randn, _table, st  # noqa: F401  (fixture)
from test_q4_gpu import _attend, _check, _pools, _unsigned_zeros

pytestmark = pytest.mark.gpu


def test_attention_on_streams_and_threads(st):
    """Eight threads, each with its stream and workspace, over the same pools: every one gets what one alone gets."""
    g = _gen(3)
    rows, new = [900, 33, 2500, 1], [2, 2, 2, 2]
    q, p, pt, table, cu = _attend(st, g, rows, new, 16, 14, 2, BF, True)
    want = st.paged_attention_q4(q, p, pt)
    _check(want, p, q, table, rows, cu)
    torch.cuda.synchronize()
    got, failed = [None] * 8, []

    def work(i):
        try:
            torch.cuda.set_device(0)
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                ws, out = st.paged_q4_workspace(q, p, pt), torch.empty_like(q)
                for _ in range(20):
                    st.stlite_paged_attention_q4(q, p, pt, out, ws)
                s.synchronize()
                assert st.stlite_device_status(ws) == st.STLITE_OK
            got[i] = out
        except Exception as e:  # told to the test's own thread
            failed.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(8)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
    assert all(torch.equal(x, want) for x in got)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_values_on_the_host(st, dtype):
    """Page-locked values: only the kept rows are read."""
    g = _gen(7)
    n, b, hkv, page = 400, 90, 2, 16
    k, v = (torch.randn((n, hkv, 128), generator=g).to(dtype) for _ in range(2))
    table, pages = _table([b], page, 5)
    idx = torch.stack([torch.randperm(n, generator=g)[:b].sort().values for _ in range(hkv)]).to(I32).cuda()
    pt = st.make_pages(pages, page, table.cuda(), _ints([b]), max_new=b)
    p, host = st.make_q4_pools(pages, page, hkv), v.pin_memory()
    st.stlite_compact_paged_q4([(k.cuda(), host, p, idx)], b, pt, 0)
    ko, vo = st.paged_fetch_q4(p, pt, b, F32)
    for got, src in ((ko, k), (vo, v)):
        kept = torch.stack([src[idx[h].cpu().long(), h] for h in range(hkv)], 1)
        assert torch.equal(got.cpu().double(), ref.decode(*ref.encode(kept)))


def test_step_on_two_streams(st):
    """Two servers' tables at once."""
    servers = []
    for i in range(2):
        S, page, M, n = 40, 16, 12, 300
        r = torch.Generator().manual_seed(i)
        free = torch.randperm(n, generator=r).to(I32)
        state = dict(table=torch.full((S, M), -1, dtype=I32), len=torch.zeros(S, dtype=I32), cu=torch.zeros(S + 1, dtype=I32),
                     free=free, n_free=torch.tensor([n], dtype=I32), slot=torch.zeros(2000, dtype=I32))
        asks = [(torch.randint(0, 100, (S,), generator=r).to(I32), torch.randint(0, 70, (S,), generator=r).to(I32)) for _ in range(6)]
        servers.append((state, asks))
    streams, device = [torch.cuda.Stream() for _ in range(2)], []
    for (state, asks), s in zip(servers, streams):
        d = {k: v.cuda() for k, v in state.items()}
        device.append((d, st.make_pages(300, 16, d["table"], d["len"], d["cu"]), [(a.cuda(), b.cuda()) for a, b in asks]))
        s.wait_stream(torch.cuda.current_stream())
    for i in range(6):
        for (d, pt, asks), s in zip(device, streams):
            st.stlite_pages_step(pt, asks[i][0], asks[i][1], d["free"], d["n_free"], d["slot"], stream=s)
    torch.cuda.synchronize()
    for (state, asks), (d, _, _) in zip(servers, device):
        table, lens, free, n = state["table"].tolist(), state["len"].tolist(), state["free"].tolist(), 300
        for keep, fresh in asks:
            cu, n, slot = ref.step(table, lens, keep.tolist(), fresh.tolist(), free, n, 300, 16, 2000)
        for name, want in (("table", table), ("len", lens), ("cu", cu), ("free", free), ("n_free", [n]), ("slot", slot)):
            assert d[name].tolist() == want, name


def test_a_step_in_one_graph(st):
    """Tables, append of two layers and attention over them captured once: each replay takes two drafts' place with two
    more, of which the last step's first one stays."""
    g, S, hq, hkv, page = _gen(12), 3, 8, 2, 16
    rows = [30, 15, 64]
    table, pages = _table(rows, page, 1, spare=9)
    width = torch.full((S, 8), -1, dtype=I32)
    width[:, :table.shape[1]] = table
    free = torch.tensor([p for p in range(pages) if p not in {int(table[s, i]) for s in range(S) for i in range(-(-rows[s] // page))}],
                        dtype=I32)
    free_d = torch.cat([free, torch.zeros(pages - len(free), dtype=I32)]).cuda()
    n_free, slot, keep, fresh = _ints([len(free)]), torch.zeros(2 * S, dtype=I32, device="cuda"), _ints(rows), _ints([2] * S)
    length, cu, pos, rope = _ints(rows), _ints([0] * (S + 1)), _ints(range(2 * S)), st.make_rope()
    pt = st.make_pages(pages, page, width.cuda(), length, cu, max_new=2)
    pools = [_pools(st, g, pages, page, hkv) for _ in range(2)]
    q, k, v = _randn(g, 2 * S, hq, 128), _randn(g, 2 * S, hkv, 128), _randn(g, 2 * S, hkv, 128)
    qo, outs = torch.empty_like(q), [torch.empty_like(q) for _ in range(2)]
    ws = st.paged_q4_workspace(q, pools[0], pt)

    def step():
        st.stlite_pages_step(pt, keep, fresh, free_d, n_free, slot)
        for p, out in zip(pools, outs):
            st.stlite_paged_append_q4(q, k, v, pos, rope, pt, qo, p)
            st.stlite_paged_attention_q4(qo, p, pt, out, ws)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(5):
        keep.copy_(length - 1)
        q.copy_(_randn(g, 2 * S, hq, 128))
        k.copy_(_randn(g, 2 * S, hkv, 128))
        graph.replay()
        want = [n + 2 + i + 1 for n in rows]
        assert length.tolist() == want and cu.tolist() == [0, 2, 4, 6]
        for p, out in zip(pools, outs):
            _check(out, p, qo, pt.table.cpu(), want, [0, 2, 4, 6])
        y, _ = paged_ref.rotate(k, pos[None], paged_ref.default_freq(1e4))
        at = slot.long().cpu()
        c, s = ref.encode(y)
        assert torch.equal(_unsigned_zeros(pools[1].k.cpu()[at // page, :, at % page]), _unsigned_zeros(c))
    paged_ref.within(qo, st.rotate_qk(q, k, pos, rope)[0].double().cpu(), torch.zeros(qo.shape, dtype=torch.float64))
