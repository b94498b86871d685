"""Packed tokens beyond what one cache of the compression pass may hold: a
serving step's number of tokens has no such bound."""
import ctypes

import pytest
import torch

import test_paged_abi as abi
from test_paged_abi import good, st  # noqa: F401  (fixtures)

BF, I32 = torch.bfloat16, torch.int32
MANY = 8 * 49152 + 3  # one layer's tokens and three


def test_many_tokens_are_not_refused(st, good):
    """Everything else is refused for its null address, behind the check of the shape."""
    lib, size, null = st._lib, ctypes.c_size_t(), st.STLITE_EINVAL
    step = abi._pages(st, good, cu_new=good)
    for n, hq, hkv, w in ((MANY, 8, 2, 1), (1 << 28, 4, 1, 1), (1 << 20, 1000, 500, 1), (MANY, 512, 1, 1 << 20)):
        sh = abi._shape(st, n=n, hq=hq, hkv=hkv, w=w)
        assert lib.stlite_rotate_qk(sh, st.make_rope(), abi._tokens(st, good, q=None), good, good, None) == null
        assert lib.stlite_paged_append(sh, st.make_rope(), abi._tokens(st, good, v=None), step, good, good, good, None) == null
    for n, hq, hkv in ((MANY, 8, 2), (1 << 30, 16, 1), (2 ** 31 - 1, 1000, 500)):
        sh = abi._shape(st, n=n, hq=hq, hkv=hkv)
        assert lib.stlite_paged_workspace_size(sh, step, size) == st.STLITE_OK
        assert lib.stlite_paged_attention(sh, step, None, good, good, good, good, 1 << 26, None) == null


@pytest.mark.parametrize("kw", [dict(n=1 << 28, hq=7, hkv=1), dict(n=2 ** 31 - 1, hq=1, hkv=1), dict(hq=1026, hkv=2),
                                dict(hq=4097, hkv=4097), dict(hq=2 ** 31 - 1, hkv=1), dict(hq=2 ** 30, hkv=2 ** 30)], ids=str)
def test_more_than_the_kernels_number(st, good, kw):
    sh, lib = abi._shape(st, **kw), st._lib
    assert lib.stlite_rotate_qk(sh, st.make_rope(), abi._tokens(st, good), good, good + 4096, None) == st.STLITE_EUNSUPPORTED
    step = abi._pages(st, good, cu_new=good)
    assert lib.stlite_paged_append(sh, st.make_rope(), abi._tokens(st, good), step, good, good, good, None) == st.STLITE_EUNSUPPORTED
    if kw.get("n", 4) == 4:
        assert lib.stlite_paged_attention(sh, step, good, good, good, good, good, 1 << 26, None) == st.STLITE_EUNSUPPORTED


@pytest.mark.gpu
def test_many_tokens_match_a_few(st):
    """25,000 sessions' 16 tokens each: the same rows as in calls of a part of the sessions."""
    seqs, w, hq, hkv, page = 25000, 16, 2, 1, 16
    n, some = seqs * w, slice(24500, 25000)
    assert n > MANY
    g = torch.Generator("cuda").manual_seed(5)
    q, k, v = (torch.randn((n, h, 128), generator=g, device="cuda").to(BF) for h in (hq, hkv, hkv))
    pos = torch.arange(n, dtype=I32, device="cuda") % 5000
    rope = st.make_rope()
    qo, ko = st.rotate_qk(q, k, pos, rope)
    part = slice(some.start * w, some.stop * w)
    few = [q[part].contiguous(), k[part].contiguous(), v[part].contiguous()]
    want_q, want_k = st.rotate_qk(few[0], few[1], pos[part], rope)
    assert torch.equal(qo[part], want_q) and torch.equal(ko[part], want_k)
    table = torch.randperm(2 * seqs, generator=g, device="cuda").to(I32).view(seqs, 2)
    lens = torch.randint(w, 2 * page + 1, (seqs,), generator=g, device="cuda").to(I32)
    kp, vp = (torch.randn((2 * seqs, page, hkv, 128), generator=g, device="cuda").to(BF) for _ in range(2))
    kp2, vp2 = kp.clone(), vp.clone()
    cu = torch.arange(0, n + 1, w, dtype=I32, device="cuda")
    for c in (cu, None):
        both = st.make_pages(2 * seqs, page, table, lens, c, max_new=w)
        st.stlite_paged_append(q, k, v, pos, rope, both, qo, kp, vp)
        out = st.paged_attention(qo, kp, vp, both)
        one = st.make_pages(2 * seqs, page, table[some], lens[some], max_new=w)
        st.stlite_paged_append(*few, pos[part], rope, one, want_q, kp2, vp2)
        at = table[some].long().flatten()
        assert torch.equal(kp[at], kp2[at]) and torch.equal(vp[at], vp2[at])
        got = st.paged_attention(want_q, kp2, vp2, one)
        # the split of work, and with it the order of sums, differs: two roundings of nearly the same number
        assert torch.equal(qo[part], want_q)
        assert (out[part].float() - got.float()).abs().max() <= 2 ** -7 * got.float().abs().max()
        kp2.copy_(kp), vp2.copy_(vp)
