"""Paged calls on several streams and host threads at once, each with its own
workspace: the bits of one call after the other."""
import threading

import pytest
import torch

from test_paged_gpu import BF, F32, _attend, _attention_case, st  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


def _cases(st):
    out = []
    for i, (rows, new, hq, hkv, dtype) in enumerate([([9000, 40], 1, 14, 2, BF), ([300] * 200, 1, 4, 2, BF),
                                                     ([2000, 0, 700], 5, 7, 1, BF), ([1500, 800], 1, 8, 2, F32)]):
        cu = [new * j for j in range(len(rows) + 1)]
        q, kp, vp, pg, _ = _attention_case(st, rows, cu, 16, hq, hkv, dtype, 60 + i)
        want, ws = _attend(st, q, kp, vp, pg)
        out.append((q, kp, vp, pg, ws, want, torch.empty_like(q)))
    return out


def test_attention_on_streams_at_once(st):
    cases = _cases(st)
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, (q, kp, vp, pg, ws, _, out) in zip(streams, cases):
            st.stlite_paged_attention(q, kp, vp, pg, out, ws, stream=s)
    torch.cuda.synchronize()
    for q, kp, vp, pg, ws, want, out in cases:
        assert torch.equal(out, want)
        assert st.stlite_device_status(ws) == st.STLITE_OK


def test_attention_from_threads_at_once(st):
    cases, failed = _cases(st), []

    def work(case):
        q, kp, vp, pg, _, want, _ = case
        try:
            stream = torch.cuda.Stream()
            for _ in range(20):
                got = st.paged_attention(q, kp, vp, pg, stream=stream)
                stream.synchronize()
                if not torch.equal(got, want):
                    failed.append("bits")
        except Exception as e:  # noqa: BLE001  (reported by the main thread)
            failed.append(repr(e))

    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(c,)) for c in cases]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed


def test_helpers_captured(st):
    """A helper in a capture, its outputs and workspace from the graph's memory, on the capture's own stream."""
    q, kp, vp, pg, _, want, _ = _cases(st)[0]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    x = torch.zeros_like(q)
    with torch.cuda.graph(graph, stream=side):
        out = st.paged_attention(x, kp, vp, pg, stream=side)
        again = st.paged_attention(x, kp, vp, pg)
    x.copy_(q)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(again, want)
