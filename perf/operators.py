"""A serving step's operators over a paged key/value cache, as measurable cases.

The compression pass leaves each session a cache of its own length.  A program
that serves many sessions keeps them in pages, and around the pass it

  * rotates the prompt's queries and keys, with a norm for each head in models
    that have one (``stlite_rotate_qk``), which is what the pass takes;
  * moves the rows that the pass keeps into pages (``stlite_compact_paged``);
  * appends each new token's key and value to them, rotated on the way
    (``stlite_paged_append``);
  * and attends from the new tokens over the pages (``stlite_paged_attention``).

``run`` computes each of them either in plain torch operations or through the
library (``own``).  Sizes are those of the repository's workloads: prompts of
screenshots and text, 28 query and 4 key/value heads of 128 (or 12 and 2),
caches as the pass leaves them or uncompressed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

D = 128
HALF = D // 2
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BASE, EPS = 1e6, 1e-6
HEADS = [(28, 4), (12, 2), (14, 2), (16, 8), (32, 8), (40, 8), (16, 1)]


# ------------------------------------------------------------------- cases

def _case(name, kind, **kw):
    """seqs: sessions; new: new tokens of each; ragged: 0 .. new of them instead; lo, hi: cached rows of a
    session (new ones included; lo < hi: spread over the logarithm); idle: every idle-th session has none;
    page: rows of a page; axes: position axes; pad: tokens behind the last session's; fused: q, k and v are
    slices of one projection's output."""
    c = dict(name=name, kind=kind, dtype="bf16", hq=28, hkv=4, seqs=1, new=1, ragged=False, lo=1, hi=1, idle=0,
             page=16, axes=1, interleaved=False, norm=False, pad=0, fused=False, layers=1, n=0, beta=0.2)
    c.update(kw)
    return c


def listed():
    return [
        # the prompt of an 8-step session (32 x 32 patches and 48 text tokens a step), q and k as the projection left
        # them, before the cache is compressed
        _case("rotate_prompt", "rotate", n=8576, axes=3, fused=True),
        # one new screenshot of 24 x 42 patches and its text on the smaller backbone, a norm for each head
        _case("rotate_frame_norm", "rotate", n=1048, hq=12, hkv=2, norm=True),
        # the fp32 reference layer that an integration is checked with
        _case("rotate_fp32", "rotate", n=1152, dtype="f32", axes=3, interleaved=True),
        # one session's next token: latency
        _case("append_one", "append", lo=10757, hi=10757),
        # one token each of 64 sessions, norms of queries and keys on the way
        _case("append_batch", "append", seqs=64, lo=200, hi=2000, norm=True, fused=True),
        # three whole prompts, uncompressed, packed one behind the other with padding after the last
        _case("append_prompt", "append", seqs=3, new=2872, lo=2872, hi=4700, page=64, axes=3, pad=19, fused=True),
        # one session's next token over its compressed cache of a 50-step session: the join of the splits counts
        _case("attend_one", "attend", lo=10757, hi=10757),
        # 32 sessions of very different lengths, the longest an uncompressed 50-step one
        _case("attend_batch", "attend", seqs=32, lo=1000, hi=53600),
        # five drafted tokens each of eight sessions, checked at once; the smaller backbone, larger pages
        _case("attend_draft", "attend", seqs=8, new=5, hq=12, hkv=2, lo=300, hi=9472, page=64),
        # fp32 reference caches on pages of an odd size, one idle slot in the batch
        _case("attend_fp32", "attend", dtype="f32", seqs=4, lo=230, hi=1182, page=24, idle=3),
        # the kept rows of one layer as the prefill finishes it
        _case("compact_layer", "compact", n=23680),
        # the kept rows of every layer of a 50-step session
        _case("compact_layers", "compact", n=53600, layers=28),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: other head counts, page sizes, lengths and batches, odd ones among them."""
    kind = rng.choice(["rotate", "append", "append", "attend", "attend", "attend", "compact"])
    hq, hkv = rng.choice(HEADS)
    c = dict(kind=kind, hq=hq, hkv=hkv, dtype="f32" if rng.random() < 0.25 else "bf16",
             page=rng.choice([1, 8, 16, 16, 16, 24, 32, 64, 100, 128]), norm=rng.random() < 0.4,
             interleaved=rng.random() < 0.3, axes=rng.choice([1, 1, 3]), fused=rng.random() < 0.5)
    f32 = c["dtype"] == "f32"
    if kind == "rotate":
        c["n"] = _log(rng, 1, 2500 if f32 else 7000)
    elif kind == "compact":
        c.update(layers=rng.choice([1, 1, 4, 28]), beta=rng.choice([0.05, 0.1, 0.2, 0.3, 0.4]),
                 n=_log(rng, 60, 11000 if f32 else 26000))
    elif kind == "append":
        c.update(seqs=_log(rng, 1, 96), pad=rng.choice([0, 0, 5]))
        c["new"] = rng.choice([1, 1, 4, _log(rng, 1, max(1, (2500 if f32 else 8000) // c["seqs"]))])
        c["lo"] = c["new"]
        c.update(hi=c["new"] + _log(rng, 1, 1500), ragged=rng.random() < 0.4 and c["new"] > 1)
    else:
        # a session's rows that all fit: at most 100,000 in the batch at its longest, half of it in fp32
        c.update(seqs=_log(rng, 1, 96), new=rng.choice([1, 1, 1, 2, 3, 5, 8]), idle=rng.choice([0, 0, 3]))
        most = (40000 if f32 else 100000) * 4 // (hkv * c["seqs"])
        c["lo"] = _log(rng, 1, max(1, most // 3))
        c.update(hi=_log(rng, c["lo"], max(c["lo"], most)), ragged=rng.random() < 0.4 and c["new"] > 1)
    return {k: v for k, v in _case("", **c).items() if k != "name"}


# ------------------------------------------------------------------ layout

def _lengths(case):
    """(rows, new tokens) of every session: a matter of the case alone."""
    r = random.Random(case["hi"] * 131 + case["seqs"])
    rows, new = [], []
    for i in range(case["seqs"]):
        rows.append(_log(r, case["lo"], case["hi"]) if i else case["hi"])
        new.append(r.randint(0, case["new"]) if case["ragged"] else case["new"])
        if case["idle"] and i % case["idle"] == case["idle"] - 1:
            rows[i] = 0
    return rows, new


def _budget(case):
    return max(1, int(case["beta"] * case["n"] + 1e-9))


def _tokens(case):
    return case["n"] if case["kind"] == "rotate" else sum(_lengths(case)[1]) + case["pad"]


def _frequencies():
    return torch.tensor([BASE ** (-2.0 * i / D) for i in range(HALF)], dtype=torch.float64, device="cuda")


def _sections(case):
    return (16, 24, 24) if case["axes"] == 3 else (HALF, 0, 0)


# ------------------------------------------------------------------ inputs

def _positions(case, total, gen):
    """Positions of `total` tokens on each axis: a session's text counts on all three, a screenshot's
    patches (32 x 32 of every 1,072 tokens) keep the step and count rows and columns."""
    start = torch.randint(0, 120000, (1,), generator=gen, device="cuda")
    t = torch.arange(total, device="cuda")
    if case["axes"] == 1:
        return (start + t).to(torch.int32)
    step, i = t // 1072, t % 1072
    base = start + step * 80
    text = base + 32 + i - 1024
    patch = i < 1024
    pos = torch.stack([torch.where(patch, base, text), torch.where(patch, base + i // 32, text),
                       torch.where(patch, base + i % 32, text)])
    return pos.to(torch.int32).contiguous()


def _pool(case, pages, gen, empty=False):
    shape = (case["layers"], pages, case["page"], case["hkv"], D)
    if empty:
        return torch.zeros(shape, dtype=DTYPES[case["dtype"]], device="cuda")
    return torch.randn(shape, generator=gen, device="cuda", dtype=DTYPES[case["dtype"]])


def _table(rows, page, gen):
    """Every session's pages in random places of a pool with a few to spare: ([S][most] int32, pool size)."""
    count = [-(-n // page) for n in rows]
    pages = sum(count) + 3
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    at = torch.tensor([sum(count[:i]) for i in range(len(rows))], device="cuda")
    slot = at[:, None] + torch.arange(max(1, max(count)), device="cuda")
    # entries past a session's pages name some other page, as stale ones do
    return order[slot.clamp_max(pages - 1)].contiguous(), pages


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt, hq, hkv, kind = DTYPES[case["dtype"]], case["hq"], case["hkv"], case["kind"]
    s = dict(case=case, inv_freq=_frequencies(), q_norm=None, k_norm=None)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda").to(dt)

    if case["norm"]:
        s["q_norm"], s["k_norm"] = (1 + 0.2 * randn(D)).to(dt), (1 + 0.2 * randn(D)).to(dt)
    if kind in ("rotate", "append"):
        total = _tokens(case)
        if case["fused"]:
            x = randn(total, hq + 2 * hkv, D)
            s["q"], s["k"], s["v"] = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
        else:
            s["q"], s["k"], s["v"] = randn(total, hq, D), randn(total, hkv, D), randn(total, hkv, D)
        s["pos"] = _positions(case, total, gen)
        s["axis"] = torch.tensor([a for a, count in enumerate(_sections(case)) for _ in range(count)], device="cuda")
        s["q_out"] = torch.zeros((total, hq, D), dtype=dt, device="cuda")
        s["k_out"] = torch.zeros((total, hkv, D), dtype=dt, device="cuda")
        if own:
            from paper_2603_00188_gb300 import stlite
            s["rope"] = stlite.make_rope(BASE, section=_sections(case), interleaved=case["interleaved"])
    if kind in ("append", "attend"):
        rows, new = _lengths(case)
        s["table"], pages = _table(rows, case["page"], gen)
        s["len"] = torch.tensor(rows, dtype=torch.int32, device="cuda")
        cu = [sum(new[:i]) for i in range(len(new) + 1)]
        s["cu_new"] = torch.tensor(cu, dtype=torch.int32, device="cuda") if case["ragged"] or case["pad"] else None
        s["k_pages"], s["v_pages"] = (_pool(case, pages, gen, kind == "append")[0] for _ in range(2))
        if kind == "attend":
            s["q"] = randn(_tokens(case), hq, D)
            s["out"] = torch.zeros_like(s["q"])
        if own:
            from paper_2603_00188_gb300 import stlite
            s["pages"] = stlite.make_pages(pages, case["page"], s["table"], s["len"], s["cu_new"], case["new"])
            if kind == "attend":
                s["ws"] = stlite.paged_workspace(s["q"], s["k_pages"], s["pages"])
    if kind == "compact":
        L, n, b = case["layers"], case["n"], _budget(case)
        s["k"], s["v"] = (torch.randn((L, n, hkv, D), generator=gen, device="cuda", dtype=dt) for _ in range(2))
        keep = torch.stack([torch.rand((hkv, n), generator=gen, device="cuda").topk(b).indices for _ in range(L)])
        s["idx"] = keep.sort(-1).values.to(torch.int32)  # [L][Hkv][B], ascending as the pass leaves them
        s["table"], pages = _table([b + 500, b, 40], case["page"], gen)
        s["k_pages"], s["v_pages"] = (_pool(case, pages, gen, True) for _ in range(2))
        if own:
            from paper_2603_00188_gb300 import stlite
            s["pages"] = stlite.make_pages(pages, case["page"], s["table"])
            s["io"] = [(s["k"][l], s["v"][l], s["k_pages"][l], s["v_pages"][l], s["idx"][l]) for l in range(L)]
    return s


# ---------------------------------------------------------- the plain forms

def _rotated(x, weight, s):
    """Norm over each head (where the model has one) and rotation by position, in 32 bits, angles in 64."""
    case, x = s["case"], x.float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()
    angle = s["pos"].view(case["axes"], -1)[s["axis"]].T.double() * s["inv_freq"]
    c, n = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if case["interleaved"]:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * c - b * n, b * c + a * n], -1).flatten(-2)
    a, b = x[..., :HALF], x[..., HALF:]
    return torch.cat([a * c - b * n, b * c + a * n], -1)


def _new_rows(s):
    """(session, row in its cache) of every new token, padding left out."""
    S, rows = s["case"]["seqs"], s["len"].long()
    cu = s["cu_new"].long() if s["cu_new"] is not None else torch.arange(S + 1, device="cuda") * s["case"]["new"]
    t = torch.arange(int(sum(_lengths(s["case"])[1])), device="cuda")
    seq = torch.searchsorted(cu, t, right=True) - 1
    return seq, rows[seq] - (cu[seq + 1] - t)


def _slots(s, seq, row):
    """Places in the pools, seen as [pages * page][Hkv][d], of rows of sessions."""
    page = s["case"]["page"]
    return s["table"][seq, row // page].long() * page + row % page


def _attend(s):
    case = s["case"]
    S, w, hq, hkv = case["seqs"], case["new"], case["hq"], case["hkv"]
    seq, row = _new_rows(s)
    i = row - s["len"].long()[seq] + w  # the last of a session's w places for the newest token
    q = torch.zeros((S, w, hq, D), device="cuda")
    q[seq, i] = s["q"].float()
    q = q.view(S, w, hkv, hq // hkv, D).permute(0, 2, 3, 1, 4).reshape(S, hkv, -1, D)
    j = torch.arange(max(1, max(_lengths(case)[0])), device="cuda")
    slot = _slots(s, torch.arange(S, device="cuda")[:, None], torch.minimum(j, (s["len"].long()[:, None] - 1).clamp_min(0)))
    k = s["k_pages"].view(-1, hkv, D)[slot].float().permute(0, 2, 1, 3)
    v = s["v_pages"].view(-1, hkv, D)[slot].float().permute(0, 2, 1, 3)
    x = (q @ k.transpose(-1, -2) / math.sqrt(D)).view(S, hkv, hq // hkv, w, -1)
    last = s["len"].long()[:, None] - w + torch.arange(w, device="cuda")  # newest key each place sees
    x = x.masked_fill_((j > last[..., None])[:, None, None], -math.inf).view(S, hkv, hq // hkv * w, -1)
    p = (x - x.amax(-1, keepdim=True).clamp_min(-1e30)).exp_()
    o = p @ v / p.sum(-1, keepdim=True).clamp_min(1e-30)
    o = o.view(S, hkv, hq // hkv, w, D).permute(0, 3, 1, 2, 4).reshape(S, w, hq, D)
    return s["out"].copy_(o[seq, i])


def _raw(t):
    """The tensor's bit pattern: copied rows are compared as whole values."""
    return t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)


def run(s):
    case, kind = s["case"], s["case"]["kind"]
    if own:
        from paper_2603_00188_gb300 import stlite
    if kind == "rotate":
        if own:
            stlite.stlite_rotate_qk(s["q"], s["k"], s["pos"], s["rope"], s["q_out"], s["k_out"], s["q_norm"],
                                    s["k_norm"], EPS)
        else:
            s["q_out"].copy_(_rotated(s["q"], s["q_norm"], s))
            s["k_out"].copy_(_rotated(s["k"], s["k_norm"], s))
        return dict(q=s["q_out"], k=s["k_out"])
    if kind == "append":
        if own:
            stlite.stlite_paged_append(s["q"], s["k"], s["v"], s["pos"], s["rope"], s["pages"], s["q_out"],
                                       s["k_pages"], s["v_pages"], s["q_norm"], s["k_norm"], EPS)
        else:
            seq, row = _new_rows(s)
            slot, t = _slots(s, seq, row), len(seq)
            s["q_out"][:t] = _rotated(s["q"], s["q_norm"], s)[:t].to(s["q"].dtype)
            s["k_pages"].view(-1, case["hkv"], D)[slot] = _rotated(s["k"], s["k_norm"], s)[:t].to(s["k"].dtype)
            s["v_pages"].view(-1, case["hkv"], D)[slot] = s["v"][:t]
        return dict(q=s["q_out"], k=s["k_pages"], v=_raw(s["v_pages"]))
    if kind == "attend":
        if own:
            stlite.stlite_paged_attention(s["q"], s["k_pages"], s["v_pages"], s["pages"], s["out"], s["ws"])
            return s["out"]
        return _attend(s)
    if own:
        stlite.stlite_compact_paged(s["io"], s["idx"].shape[-1], s["pages"], 1)
    else:
        at = s["idx"].long().transpose(1, 2)[..., None].expand(-1, -1, -1, D)
        row = torch.arange(at.shape[1], device="cuda")
        slot = _slots(s, torch.ones_like(row), row)
        s["k_pages"].view(case["layers"], -1, case["hkv"], D)[:, slot] = s["k"].gather(1, at)
        s["v_pages"].view(case["layers"], -1, case["hkv"], D)[:, slot] = s["v"].gather(1, at)
    return dict(k=_raw(s["k_pages"]), v=_raw(s["v_pages"]))


def work(case):
    e, hq, hkv, kind = (2 if case["dtype"] == "bf16" else 4), case["hq"], case["hkv"], case["kind"]
    if kind == "rotate":
        elems = case["n"] * (hq + hkv) * D
        return dict(bytes=2 * e * elems + 4 * case["axes"] * case["n"], flops=(3 + 4 * case["norm"]) * elems)
    if kind == "compact":
        b = _budget(case) * hkv
        return dict(bytes=case["layers"] * (4 * b * D * e + 4 * b), flops=0)
    rows, new = _lengths(case)
    t = sum(new)
    if kind == "append":
        return dict(bytes=2 * e * t * (hq + 2 * hkv) * D + 4 * case["axes"] * t, flops=(3 + 4 * case["norm"]) * t * (hq + hkv) * D)
    used = [(r, n) for r, n in zip(rows, new) if n]
    return dict(bytes=e * (2 * hkv * sum(r for r, _ in used) + 2 * hq * t) * D,
                flops=4.0 * hq * D * sum(r * n for r, n in used))


# ------------------------------------------------------- the same in 64 bits

def _rotated64(x, weight, s):
    case, x = s["case"], x.double()
    if weight is not None:
        x = weight.double() * x / ((x * x).sum(-1, keepdim=True) / D + EPS).sqrt()
    out = torch.empty_like(x)
    pos, first = s["pos"].view(case["axes"], -1).double(), 0
    for axis, count in enumerate(_sections(case)):
        i = torch.arange(first, first + count, device="cuda")
        first += count
        if not count:
            continue
        turn = torch.polar(torch.ones(1, dtype=torch.float64, device="cuda"),
                           pos[axis][:, None] * BASE ** (-i.double() / HALF))[:, None]
        lo, hi = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + HALF)
        z = torch.complex(x[..., lo], x[..., hi]) * turn
        out[..., lo], out[..., hi] = z.real, z.imag
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind, page, hkv = case["kind"], case["page"], case["hkv"]
    if kind == "rotate":
        return dict(q=_rotated64(s["q"], s["q_norm"], s), k=_rotated64(s["k"], s["k_norm"], s))
    if kind == "compact":
        k, v = s["k_pages"], s["v_pages"]
        row = torch.arange(_budget(case), device="cuda")
        if case["layers"] * hkv * len(row) // page > 20000:
            return None  # a page at a time takes too long
        for r0 in range(0, len(row), page):
            r, p = row[r0:r0 + page], int(s["table"][1, r0 // page])
            for l in range(case["layers"]):
                for h in range(hkv):
                    at = s["idx"][l, h, r0:r0 + page].long()
                    k[l, p, :len(r), h], v[l, p, :len(r), h] = s["k"][l, at, h], s["v"][l, at, h]
        return dict(k=_raw(k), v=_raw(v))
    rows, new = _lengths(case)
    table, t = s["table"].tolist(), 0
    if kind == "append":
        q, k = _rotated64(s["q"], s["q_norm"], s), _rotated64(s["k"], s["k_norm"], s)
        kp, vp = s["k_pages"].double(), s["v_pages"]
        for b, (n, m) in enumerate(zip(rows, new)):
            for first in range(n - m, n):
                if first % page and first > n - m:
                    continue  # whole pages at a time, from the first new row
                end = min(n, first // page * page + page)
                p, i = table[b][first // page], first % page
                kp[p, i:i + end - first] = k[t:t + end - first]
                vp[p, i:i + end - first] = s["v"][t:t + end - first]
                t += end - first
        q[t:] = 0
        return dict(q=q, k=kp, v=_raw(vp))
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    G = case["hq"] // hkv
    for b, (n, m) in enumerate(zip(rows, new)):
        own_pages = s["table"][b, :-(-n // page)].long()
        k, v = (s[x][own_pages].reshape(-1, hkv, D)[:n].double() for x in ("k_pages", "v_pages"))
        for i in range(m):
            sees = n - (m - 1 - i)
            if sees > 0:
                qi = s["q"][t + i].double().view(hkv, G, D)
                p = torch.softmax(torch.einsum("hgd,nhd->hgn", qi, k[:sees]) / math.sqrt(D), -1)
                out[t + i] = torch.einsum("hgn,nhd->hgd", p, v[:sees]).reshape(-1, D)
        t += m
    return out
