"""The helpers that allocate their outputs and workspaces, given a stream that
is not the current one: the stream waits for what the current one holds, and
the tensors' memory is not given out again before the stream has used it."""
import pytest
import torch

from paper_2603_00188_gb300 import build as pkg_build

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32
HQ, HKV, N = 8, 2, 320
FRAMES = ([0, 160], [10, 10], [12, 12])


@pytest.fixture(scope="module")
def st():
    pkg_build.build()
    from paper_2603_00188_gb300 import stlite
    return stlite


def _inputs(device, seed=1):
    g = torch.Generator().manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=g).to(BF).to(device)

    return dict(q=randn(N, HQ, 128), k=randn(N, HKV, 128), v=randn(N, HKV, 128), kp=randn(20, 16, HKV, 128),
                vp=randn(20, 16, HKV, 128), norm=randn(128), pos=torch.arange(N, dtype=I32).to(device),
                table=torch.arange(20, dtype=I32).view(2, 10).to(device), lens=torch.tensor([150, 97], dtype=I32).to(device))


def _pages(st, x):
    return st.make_pages(20, 16, x["table"], x["lens"], max_new=2)


# helper -> (its entry point, a call of it, as a tuple of tensors)
HELPERS = {
    "rotate_qk": ("stlite_rotate_qk", lambda st, x, s: st.rotate_qk(
        x["q"], x["k"], x["pos"], st.make_rope(), x["norm"], x["norm"], stream=s)),
    "paged_attention": ("stlite_paged_attention", lambda st, x, s: (
        st.paged_attention(x["q"][:4], x["kp"], x["vp"], _pages(st, x), stream=s),)),
    "decode_attention": ("stlite_decode_attention", lambda st, x, s: (
        st.decode_attention(x["q"][:3], x["k"], x["v"], stream=s),)),
    "decode_attention_layers": ("stlite_decode_attention_layers", lambda st, x, s: tuple(
        st.decode_attention_layers([x["q"][:3], x["q"][3:6]], [x["k"], x["v"]], [x["v"], x["k"]], stream=s)[0])),
    "prompt_score": ("stlite_prompt_score", lambda st, x, s: st.prompt_score(x["q"], x["k"], stream=s)[:1]),
    "compress_layer": ("stlite_compress_layer", lambda st, x, s: st.compress_layer(
        x["q"][-8:], x["k"], x["v"], FRAMES, stream=s)),
}


def _tensors(x):
    if isinstance(x, torch.Tensor):
        return [x]
    if isinstance(x, (list, tuple)):
        return [t for y in x for t in _tensors(y)]
    return [t for t in (getattr(x, n, None) for n in ("table", "length", "cu_new")) if t is not None]


@pytest.mark.parametrize("given", ["other", "current", None])
@pytest.mark.parametrize("helper", HELPERS)
def test_helpers_order_streams(st, monkeypatch, helper, given):
    """On the host: the wait, and every tensor of the call recorded, before the entry point is called."""
    class Stream:
        cuda_stream = 7

        def wait_stream(self, other):
            log.append(("wait", self, other))

    log, current, other = [], Stream(), Stream()
    entry, call = HELPERS[helper]
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current)
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: log.append(("record", s, t.data_ptr())))
    monkeypatch.setattr(st, entry, lambda *a: log.append(("call", a)))
    stream = dict(other=other, current=current).get(given)
    call(st, _inputs("cpu"), stream)
    args = log.pop()[1]
    assert args[-1] is stream or args[-4] is stream
    if given != "other":
        assert not log
        return
    assert log[0] == ("wait", other, current)
    assert all(e[:2] == ("record", other) for e in log[1:])
    recorded = {e[2] for e in log[1:]}
    assert {t.data_ptr() for a in args for t in _tensors(a)} <= recorded


@pytest.mark.gpu
@pytest.mark.parametrize("helper", HELPERS)
def test_helpers_wait_for_the_current_stream(st, helper):
    """Inputs that the current stream writes late, and memory that it uses late, are ready on the other stream."""
    call, good = HELPERS[helper][1], _inputs("cuda")
    want = [t.clone() for t in call(st, good, None)]
    late, side = {n: torch.zeros_like(t) for n, t in good.items()}, torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(40_000_000)  # some 20 ms
    for n, t in late.items():
        t.copy_(good[n])
    got = call(st, late, side)
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("helper", HELPERS)
def test_helpers_keep_their_memory(st, helper):
    """Everything dropped while the other stream has not begun: nobody else gets the memory."""
    call, side = HELPERS[helper][1], torch.cuda.Stream()
    call(st, _inputs("cuda"), None)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(40_000_000)
    x = _inputs("cuda")
    want = [t.clone() for t in call(st, x, None)]
    got = call(st, x, side)
    sizes = {t.nbytes for t in got} | {t.nbytes for t in x.values()} | {1 << 20, 3 << 20, 8 << 20}
    del x
    others = [torch.full((n,), 0x55, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(4)]
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    torch.cuda.synchronize()
    assert all(bool((t == 0x55).all()) for t in others)
