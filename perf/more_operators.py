"""A cache held in 4 bits, and the page tables of a serving step, as measurable cases.

A paged cache in 4 bits takes 72 bytes for 128 elements in place of 256: each
group of 16 elements has one e4m3 scale, each element an e2m1 code, and each
key/value head may have a factor.  A program that serves sessions over such a cache

  * moves the rows that the compression pass keeps into it (``stlite_compact_paged_q4``);
  * appends each new token's rotated key and its value (``stlite_paged_append_q4``);
  * attends from the new tokens over it (``stlite_paged_attention_q4``);
  * and takes rows out again as dense ones, to compress a session anew or to move it
    (``stlite_paged_fetch_q4``).

Around every step it gives pages to the sessions that grow, takes back those of
drafted tokens that were refused and of sessions that ended, and says where
each new token goes (``stlite_pages_step``).

``run`` computes each of them either in plain torch operations or through the
library (``own``).  What a pass writes in 4 bits it reads back as the values it
stands for.  Sizes are those of the repository's workloads: 28 query and 4
key/value heads of 128 (or 12 and 2), caches as the pass leaves them or
uncompressed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

D = 128
HALF = D // 2
GROUP = 16
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BASE, EPS = 1e6, 1e-6
HEADS = [(28, 4), (12, 2), (14, 2), (16, 8), (32, 8), (40, 8), (16, 1)]


# ------------------------------------------------------------------- cases

def _case(name, kind, **kw):
    """seqs: sessions; new: new tokens of each; ragged: 0 .. new of them instead; lo, hi: cached rows of a
    session (new ones included; lo < hi: spread over the logarithm); idle: every idle-th session has none;
    page: rows of a page; axes: position axes; pad: tokens behind the last session's; fused: q, k and v are
    slices of one projection's output; factor: every key/value head has a factor.  Page tables: leave: every
    leave-th session ends and another takes its place; short: fewer pages (and places for tokens) than asked for."""
    c = dict(name=name, kind=kind, dtype="bf16", hq=28, hkv=4, seqs=1, new=1, ragged=False, lo=1, hi=1, idle=0,
             page=16, axes=1, interleaved=False, norm=False, pad=0, fused=False, factor=False, layers=1, n=0, beta=0.2,
             leave=0, short=False)
    c.update(kw)
    return c


def listed():
    return [
        # one session's next token into its compressed cache: latency
        _case("append_one", "append", lo=10757, hi=10757),
        # the screenshot and text of one new step (24 x 42 patches and 40 text tokens) of each of two sessions,
        # uncompressed, on the smaller backbone, packed with padding after the last
        _case("append_frames", "append", hq=12, hkv=2, seqs=2, new=1048, lo=1048, hi=3100, page=64, axes=3, pad=19,
              norm=True, fused=True),
        # the kept rows of one layer as the prefill finishes it
        _case("compact_layer", "compact", n=23680),
        # the kept rows of every layer of a 50-step session
        _case("compact_layers", "compact", n=53600, layers=28, factor=True),
        # a short session's rows of one layer, to compress them anew
        _case("fetch_layer", "fetch", lo=4736, hi=4736, new=4736),
        # every layer of 24 sessions leaves the cache, whole
        _case("fetch_sessions", "fetch", seqs=24, lo=300, hi=9472, new=9472, layers=12, page=64),
        # one session's next token over its compressed cache of a 50-step session: the join of the splits counts
        _case("attend_one", "attend", lo=10757, hi=10757),
        # 32 sessions of very different lengths, the longest an uncompressed 50-step one
        _case("attend_batch", "attend", seqs=32, lo=1000, hi=53600),
        # five drafted tokens each of eight sessions, checked at once; the smaller backbone, larger pages, factors
        _case("attend_draft", "attend", seqs=8, new=5, hq=12, hkv=2, lo=300, hi=9472, page=64, factor=True),
        # fp32 queries, pages of an odd size, one idle slot in the batch
        _case("attend_fp32", "attend", dtype="f32", seqs=4, lo=230, hi=9182, page=24, idle=3),
        # 64 sessions with five new drafts each, of the last ones some refused
        _case("step_drafts", "step", seqs=64, new=5, lo=200, hi=10757),
        # 256 sessions with a token each; an eighth of them ends and makes room for one that a prefill begins
        _case("step_admit", "step", seqs=256, new=1, lo=400, hi=26560, leave=8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: other head counts, page sizes, lengths and batches, odd ones among them."""
    kind = rng.choice(["append", "append", "compact", "fetch", "attend", "attend", "attend", "step"])
    hq, hkv = rng.choice(HEADS)
    c = dict(kind=kind, hq=hq, hkv=hkv, dtype="f32" if rng.random() < 0.25 else "bf16",
             page=rng.choice([1, 8, 16, 16, 16, 24, 32, 64, 100, 128]), norm=rng.random() < 0.4,
             interleaved=rng.random() < 0.3, axes=rng.choice([1, 1, 3]), fused=rng.random() < 0.5,
             factor=rng.random() < 0.4)
    if kind == "compact":
        c.update(layers=rng.choice([1, 1, 4, 28]), beta=rng.choice([0.05, 0.1, 0.2, 0.3, 0.4]), n=_log(rng, 60, 13000))
    elif kind == "append":
        c.update(seqs=_log(rng, 1, 96), pad=rng.choice([0, 0, 5]))
        c["new"] = rng.choice([1, 1, 4, _log(rng, 1, max(1, 1200 // c["seqs"]))])
        c["lo"] = c["new"]
        c.update(hi=c["new"] + _log(rng, 1, 1500), ragged=rng.random() < 0.4 and c["new"] > 1)
    elif kind == "fetch":
        c.update(seqs=_log(rng, 1, 24), layers=rng.choice([1, 1, 3, 8]), idle=rng.choice([0, 0, 3]))
        c["new"] = c["hi"] = _log(rng, 1, max(1, 16000 // c["seqs"]))
        c["lo"] = _log(rng, 1, c["hi"])
    elif kind == "attend":
        # a session's rows that all fit: at most 100,000 in the batch at its longest
        c.update(seqs=_log(rng, 1, 96), new=rng.choice([1, 1, 1, 2, 3, 5, 8]), idle=rng.choice([0, 0, 3]))
        most = (40000 if c["dtype"] == "f32" else 100000) * 4 // (hkv * c["seqs"])
        c["lo"] = _log(rng, 1, max(1, most // 3))
        c.update(hi=_log(rng, c["lo"], max(c["lo"], most)), ragged=rng.random() < 0.4 and c["new"] > 1)
    else:
        c.update(seqs=_log(rng, 1, 300), new=rng.choice([1, 1, 3, 5, 40]), leave=rng.choice([0, 0, 3, 8]),
                 idle=rng.choice([0, 3]), short=rng.random() < 0.4, lo=_log(rng, 1, 400))
        c["hi"] = _log(rng, c["lo"], 20000)
    return {k: v for k, v in _case("", **c).items() if k != "name"}


# ------------------------------------------------------------------ layout

def _lengths(case):
    """(rows, new tokens) of every session: a matter of the case alone."""
    r = random.Random(case["hi"] * 131 + case["seqs"])
    rows, new = [], []
    for i in range(case["seqs"]):
        rows.append(_log(r, case["lo"], case["hi"]) if i else case["hi"])
        new.append(r.randint(0, case["new"]) if case["ragged"] and i else case["new"])
        if case["idle"] and i % case["idle"] == case["idle"] - 1:
            rows[i] = 0
        if case["kind"] == "fetch":
            new[i] = rows[i]  # whole sessions
    return rows, new


def _asked(case):
    """Of a step's sessions: (rows so far, rows that stay, new tokens)."""
    r = random.Random(case["hi"] * 137 + case["seqs"])
    rows, _ = _lengths(case)
    keep, fresh = [], []
    for i, n in enumerate(rows):
        keep.append(max(0, n - r.randint(0, case["new"] - 1)))
        fresh.append(case["new"])
        if case["idle"] and i % case["idle"] == case["idle"] - 1:
            fresh[i] = 0
        if case["leave"] and i % case["leave"] == case["leave"] - 1:
            keep[i], fresh[i] = 0, _log(r, case["lo"], case["hi"])
    return rows, keep, fresh


def _budget(case):
    return max(1, int(case["beta"] * case["n"] + 1e-9))


def _tokens(case):
    return sum(_lengths(case)[1]) + case["pad"]


def _frequencies():
    return torch.tensor([BASE ** (-2.0 * i / D) for i in range(HALF)], dtype=torch.float64, device="cuda")


def _sections(case):
    return (16, 24, 24) if case["axes"] == 3 else (HALF, 0, 0)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------ the 4-bit form

def _encode(x, factor):
    """x [..., 128] -> (codes [..., 64], scales [..., 8] e4m3): a group's scale is its largest magnitude over 6,
    rounded, and not below the smallest one; elements go to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4 and 6, ties to
    the even code."""
    g = x.unflatten(-1, (-1, GROUP))
    top = (g.abs().amax(-1) / (6 * factor)).clamp(2.0 ** -9, 448.0)
    scale = top.float().to(torch.float8_e4m3fn)
    z = (g / (factor * scale.to(x.dtype))[..., None]).abs().flatten(-2)
    code = ((z > 0.25).to(torch.uint8) + (z >= 0.75) + (z > 1.25) + (z >= 1.75) + (z > 2.5) + (z >= 3.5) + (z > 5.0)
            + ((x < 0).to(torch.uint8) << 3))
    return code[..., 0::2] | code[..., 1::2] << 4, scale


def _decode(code, scale, factor):
    """The values, 32 bits: code [..., 64], scale [..., 8], factor [..., 1]."""
    c = torch.stack([code & 15, code >> 4], -1).flatten(-2)
    m = (c & 7).float()
    value = torch.where(m < 4, m * 0.5, torch.where(m < 6, m - 2, 2 * m - 8)) * (1.0 - 2.0 * (c >> 3))
    return (value.unflatten(-1, (-1, GROUP)) * (scale.float() * factor)[..., None]).flatten(-2)


def _pools(case, pages, gen, empty=False):
    """Pools of every layer, each [L][pages][Hkv][page][64] or [8], and the heads' factors."""
    shape = (case["layers"], pages, case["hkv"], case["page"])
    p = {}
    for x in "kv":
        f = None
        if case["factor"]:  # powers of two: values stay exact in 16 bits
            f = torch.randint(-2, 3, (case["hkv"],), generator=gen, device="cuda").float().exp2()
        p[x + "_factor"] = f
        if empty:
            p[x] = torch.zeros(shape + (D // 2,), dtype=torch.uint8, device="cuda")
            p[x + "_scale"] = torch.zeros(shape + (D // GROUP,), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        else:
            y = torch.randn(shape + (D,), generator=gen, device="cuda", dtype=torch.bfloat16).float()
            p[x], p[x + "_scale"] = _encode(y, 1.0)  # a cache of normal rows, times the factor
    return p


def _factor(p, x, hkv):
    f = p[x + "_factor"]
    return (torch.ones(hkv, device="cuda") if f is None else f)[:, None]


def _own_pools(p, layer):
    from paper_2603_00188_gb300 import stlite
    return stlite.Q4Pools(p["k"][layer], p["v"][layer], p["k_scale"][layer], p["v_scale"][layer], p["k_factor"],
                          p["v_factor"])


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


def _table(rows, page, gen, most=0, spare=3):
    """Every session's pages in random places of a pool with a few to spare: ([S][most] int32, pool size, the
    spare pages)."""
    count = [-(-n // page) for n in rows]
    pages = sum(count) + spare
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    at = torch.tensor([sum(count[:i]) for i in range(len(rows))], device="cuda")
    slot = at[:, None] + torch.arange(max(1, most, max(count)), device="cuda")
    # entries past a session's pages name some other page, as stale ones do
    return order[slot.clamp_max(pages - 1)].contiguous(), pages, order[sum(count):]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt, hq, hkv, kind, L = DTYPES[case["dtype"]], case["hq"], case["hkv"], case["kind"], case["layers"]
    s = dict(case=case, q_norm=None, k_norm=None)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda").to(dt)

    def rows_out(*shape):  # a fetch's outputs: 16 bits hold every value of a cache whose factors are powers of two
        return [torch.zeros(shape + (hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]

    if kind == "step":
        return _prepare_step(case, gen, s)
    if kind == "compact":
        n, b = case["n"], _budget(case)
        s["k"], s["v"] = (torch.randn((L, n, hkv, D), generator=gen, device="cuda", dtype=dt) for _ in range(2))
        keep = torch.stack([torch.rand((hkv, n), generator=gen, device="cuda").topk(b).indices for _ in range(L)])
        s["idx"] = keep.sort(-1).values.to(torch.int32)  # [L][Hkv][B], ascending as the pass leaves them
        s["table"], pages, _ = _table([b + 500, b, 40], case["page"], gen)
        s["pools"] = _pools(case, pages, gen, True)
        s["len"], s["cu_new"] = _ints([b + 500, b, 40]), _ints([0, 0, b, b])  # what is read back: the second session
        s["k_out"], s["v_out"] = rows_out(L, b)
    else:
        rows, new = _lengths(case)
        s["table"], pages, _ = _table(rows, case["page"], gen)
        s["len"] = _ints(rows)
        cu = [sum(new[:i]) for i in range(len(new) + 1)]
        s["cu_new"] = _ints(cu) if case["ragged"] or case["pad"] or kind == "fetch" else None
        s["pools"] = _pools(case, pages, gen, kind == "append")
        if kind != "attend":
            s["k_out"], s["v_out"] = rows_out(L, _tokens(case))
        else:
            s["q"] = randn(_tokens(case), hq, D)
            s["out"] = torch.zeros_like(s["q"])
    if kind == "append":
        total = _tokens(case)
        if case["norm"]:
            s["q_norm"], s["k_norm"] = (1 + 0.2 * randn(D)).to(dt), (1 + 0.2 * randn(D)).to(dt)
        if case["fused"]:
            x = randn(total, hq + 2 * hkv, D)
            s["q"], s["k"], s["v"] = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
        else:
            s["q"], s["k"], s["v"] = randn(total, hq, D), randn(total, hkv, D), randn(total, hkv, D)
        s["pos"] = _positions(case, total, gen)
        s["axis"] = torch.tensor([a for a, count in enumerate(_sections(case)) for _ in range(count)], device="cuda")
        s["inv_freq"] = _frequencies()
        s["q_out"] = torch.zeros((total, hq, D), dtype=dt, device="cuda")
    if own:
        from paper_2603_00188_gb300 import stlite
        s["q4"] = [_own_pools(s["pools"], l) for l in range(L)]
        s["pages"] = stlite.make_pages(pages, case["page"], s["table"], s["len"], s["cu_new"], case["new"])
        if kind == "append":
            s["rope"] = stlite.make_rope(BASE, section=_sections(case), interleaved=case["interleaved"])
        if kind == "attend":
            s["ws"] = stlite.paged_q4_workspace(s["q"], s["q4"][0], s["pages"])
        else:
            s["rows"] = [(s["q4"][l], s["k_out"][l], s["v_out"][l]) for l in range(L)]
        if kind == "compact":
            s["io"] = [(s["k"][l], s["v"][l], s["q4"][l], s["idx"][l]) for l in range(L)]
    return s


def _prepare_step(case, gen, s):
    rows, keep, fresh = _asked(case)
    page = case["page"]
    after = [k + f for k, f in zip(keep, fresh)]
    wanted = sum(max(0, -(-a // page) - -(-n // page)) for a, n in zip(after, rows))
    spare = wanted // 2 if case["short"] else wanted + 3
    s["table"], pages, free = _table(rows, page, gen, -(-max(after) // page) + 2, spare)
    s["free"] = torch.zeros(pages, dtype=torch.int32, device="cuda")
    s["free"][:spare] = free
    s["n_free"], s["len"], s["keep"], s["fresh"] = _ints([spare]), _ints(rows), _ints(keep), _ints(fresh)
    # which sessions wait, and where each new token goes, changes with the seed: some ask for a token less
    if case["new"] > 1:
        s["fresh"] -= torch.randint(0, 2, (case["seqs"],), generator=gen, device="cuda", dtype=torch.int32) * (s["fresh"] > 0)
    places = sum(fresh)
    s["slot"] = torch.zeros(max(1, places * 3 // 4 if case["short"] else places), dtype=torch.int32, device="cuda")
    s["cu_new"] = torch.zeros(case["seqs"] + 1, dtype=torch.int32, device="cuda")
    if own:
        from paper_2603_00188_gb300 import stlite
        s["pages"] = stlite.make_pages(pages, page, s["table"], s["len"], s["cu_new"], case["new"])
    return s


# ---------------------------------------------------------- the plain forms

def _rotated(x, weight, s):
    """Norm over each head (where the model has one) and rotation by position, in 64 bits: values next to a
    border between two codes."""
    case, x = s["case"], x.double()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.double()
    angle = s["pos"].view(case["axes"], -1)[s["axis"]].T.double() * s["inv_freq"]
    c, n = angle.cos()[:, None], angle.sin()[:, None]
    if case["interleaved"]:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * c - b * n, b * c + a * n], -1).flatten(-2)
    a, b = x[..., :HALF], x[..., HALF:]
    return torch.cat([a * c - b * n, b * c + a * n], -1)


def _new_rows(s):
    """(session, row in its cache) of every new token, padding left out."""
    case = s["case"]
    S, rows = len(s["len"]), s["len"].long()
    cu = s["cu_new"].long() if s["cu_new"] is not None else torch.arange(S + 1, device="cuda") * case["new"]
    t = torch.arange(_budget(case) if case["kind"] == "compact" else int(sum(_lengths(case)[1])), device="cuda")
    seq = torch.searchsorted(cu, t, right=True) - 1
    return seq, rows[seq] - (cu[seq + 1] - t)


def _places(s, seq, row):
    """(page, row of the page) of rows of sessions."""
    page = s["case"]["page"]
    return s["table"][seq, row // page].long(), row % page


def _write(s, x, at, y):
    """y [L][rows][Hkv][128] into the pools of x ("k" or "v") at the places `at`."""
    p = s["pools"]
    code, scale = _encode(y, _factor(p, x, s["case"]["hkv"]).to(y.dtype))
    p[x][:, at[0], :, at[1]] = code.transpose(0, 1)
    p[x + "_scale"].view(torch.uint8)[:, at[0], :, at[1]] = scale.view(torch.uint8).transpose(0, 1)


def _read(s, x, at):
    """Rows of a pool, [L][rows][Hkv][128] in 32 bits."""
    p = s["pools"]
    code, scale = p[x][:, at[0], :, at[1]], p[x + "_scale"].view(torch.uint8)[:, at[0], :, at[1]]
    return _decode(code, scale.view(torch.float8_e4m3fn), _factor(p, x, s["case"]["hkv"])).transpose(0, 1)


def _fetch(s):
    at = _places(s, *_new_rows(s))
    n = len(at[0])
    s["k_out"][:, :n] = _read(s, "k", at)
    s["v_out"][:, :n] = _read(s, "v", at)
    return dict(k=s["k_out"], v=s["v_out"])


def _attend(s):
    case = s["case"]
    S, w, hq, hkv = case["seqs"], case["new"], case["hq"], case["hkv"]
    seq, row = _new_rows(s)
    i = row - s["len"].long()[seq] + w  # the last of a session's w places for the newest token
    q = torch.zeros((S, w, hq, D), device="cuda")
    q[seq, i] = s["q"].float()
    q = q.view(S, w, hkv, hq // hkv, D).permute(0, 2, 3, 1, 4).reshape(S, hkv, -1, D)
    j = torch.arange(max(1, max(_lengths(case)[0])), device="cuda")
    at = _places(s, torch.arange(S, device="cuda")[:, None], torch.minimum(j, (s["len"].long()[:, None] - 1).clamp_min(0)))
    k, v = (_read(s, x, [a.flatten() for a in at])[0].view(S, -1, hkv, D).permute(0, 2, 1, 3) for x in "kv")
    x = (q @ k.transpose(-1, -2) / math.sqrt(D)).view(S, hkv, hq // hkv, w, -1)
    last = s["len"].long()[:, None] - w + torch.arange(w, device="cuda")  # newest key each place sees
    x = x.masked_fill_((j > last[..., None])[:, None, None], -math.inf).view(S, hkv, hq // hkv * w, -1)
    p = (x - x.amax(-1, keepdim=True).clamp_min(-1e30)).exp_()
    o = p @ v / p.sum(-1, keepdim=True).clamp_min(1e-30)
    o = o.view(S, hkv, hq // hkv, w, D).permute(0, 3, 1, 2, 4).reshape(S, w, hq, D)
    return s["out"].copy_(o[seq, i])


def _step(s):
    """Pages past the rows that stay go back, in the sessions' order; then sessions are served in their order, as long
    as pages and places for tokens last; one that needs no page is not held up by pages."""
    page, (S, M), dev = s["case"]["page"], s["table"].shape, "cuda"
    total, places = s["free"].numel(), s["slot"].numel()
    have = s["len"].long().clamp(0, M * page)
    keep, fresh = torch.minimum(s["keep"].long().clamp_min(0), have), s["fresh"].long().clamp_min(0)
    held, kept = (have + page - 1) // page, (keep + page - 1) // page
    back = held - kept
    back_end = back.cumsum(0)
    # released pages on top of the free ones
    j = torch.arange(total, device=dev) - s["n_free"].long()
    who = torch.searchsorted(back_end, j, right=True).clamp_max(S - 1)
    which = kept[who] + j - back_end[who] + back[who]
    s["free"].copy_(torch.where((j >= 0) & (j < back_end[-1]), s["table"][who, which.clamp(0, M - 1)], s["free"]))
    n_free = (s["n_free"].long() + back_end[-1]).clamp_max(total)
    # who is served
    fits = keep + fresh <= M * page
    want = torch.where(fits, (keep + fresh + page - 1) // page - kept, 0)
    may = fits & ((want == 0) | (want.cumsum(0) <= n_free))
    asked = torch.where(may, fresh, 0)
    served = may & ((fresh == 0) | (asked.cumsum(0) <= places))
    got, want = torch.where(served, fresh, 0), torch.where(served, want, 0)
    want_end, cu = want.cumsum(0), torch.cat([torch.zeros(1, dtype=torch.long, device=dev), got.cumsum(0)])
    # the last free pages, one after the other, to the served sessions' next entries
    i = torch.arange(M, device=dev) - kept[:, None]
    take = n_free - 1 - (want_end - want)[:, None] - i
    s["table"].copy_(torch.where((i >= 0) & (i < want[:, None]), s["free"][take.clamp(0, total - 1)], s["table"]))
    s["n_free"].copy_(n_free - want_end[-1])
    s["len"].copy_(keep + got)
    s["cu_new"].copy_(cu)
    t = torch.arange(places, device=dev)
    who = torch.searchsorted(cu[1:], t, right=True).clamp_max(S - 1)
    row = (keep[who] + t - cu[who]).clamp(0, M * page - 1)
    s["slot"].copy_(torch.where(t < cu[-1], s["table"][who, row // page].long() * page + row % page, -1))


def run(s):
    case, kind = s["case"], s["case"]["kind"]
    if own:
        from paper_2603_00188_gb300 import stlite
    if kind == "step":
        if own:
            stlite.stlite_pages_step(s["pages"], s["keep"], s["fresh"], s["free"], s["n_free"], s["slot"])
        else:
            _step(s)
        return {x: s[x] for x in ("table", "len", "cu_new", "free", "n_free", "slot")}
    if kind == "attend":
        if own:
            stlite.stlite_paged_attention_q4(s["q"], s["q4"][0], s["pages"], s["out"], s["ws"])
            return s["out"]
        return _attend(s)
    if kind == "append":
        if own:
            stlite.stlite_paged_append_q4(s["q"], s["k"], s["v"], s["pos"], s["rope"], s["pages"], s["q_out"],
                                          s["q4"][0], s["q_norm"], s["k_norm"], EPS)
        else:
            at = _places(s, *_new_rows(s))
            t = len(at[0])
            s["q_out"][:t] = _rotated(s["q"], s["q_norm"], s)[:t].to(s["q"].dtype)
            _write(s, "k", at, _rotated(s["k"], s["k_norm"], s)[None, :t])
            _write(s, "v", at, s["v"].float()[None, :t])
    if kind == "compact":
        if own:
            stlite.stlite_compact_paged_q4(s["io"], s["idx"].shape[-1], s["pages"], 1)
        else:
            keep = s["idx"].long().transpose(1, 2)[..., None].expand(-1, -1, -1, D)
            at = _places(s, *_new_rows(s))
            _write(s, "k", at, s["k"].gather(1, keep).float())
            _write(s, "v", at, s["v"].gather(1, keep).float())
    if own:
        stlite.stlite_paged_fetch_q4(s["rows"], s["pages"])
        r = dict(k=s["k_out"], v=s["v_out"])
    else:
        r = _fetch(s)
    if kind == "append":
        r["q"] = s["q_out"]
    return r


def work(case):
    e, hq, hkv, kind = (2 if case["dtype"] == "bf16" else 4), case["hq"], case["hkv"], case["kind"]
    row = D // 2 + D // GROUP  # bytes of 128 elements in 4 bits
    if kind == "compact":
        b = _budget(case) * hkv * case["layers"]  # rows of keys, and of values, written and read back
        return dict(bytes=b * 2 * (D * e + 2 * row + 2 * D) + 4 * b, flops=6 * b * D)
    if kind == "step":
        rows, keep, fresh = _asked(case)
        moved = sum(-(-n // case["page"]) - -(-k // case["page"]) for n, k in zip(rows, keep))
        taken = sum(-(-(k + f) // case["page"]) - -(-k // case["page"]) for k, f in zip(keep, fresh))
        return dict(bytes=4 * (5 * case["seqs"] + 2 * moved + 2 * taken + sum(fresh)), flops=0)
    rows, new = _lengths(case)
    t = sum(new)
    if kind == "fetch":
        return dict(bytes=case["layers"] * t * hkv * 2 * (row + 2 * D), flops=4 * case["layers"] * t * hkv * D)
    if kind == "append":
        return dict(bytes=t * (2 * e * hq * D + 2 * hkv * (e * D + 2 * row + 2 * D) + 4 * case["axes"]),
                    flops=(3 + 4 * case["norm"]) * t * (hq + hkv) * D + 12 * t * hkv * D)
    used = [(r, n) for r, n in zip(rows, new) if n]
    return dict(bytes=row * 2 * hkv * sum(r for r, _ in used) + e * 2 * hq * t * D,
                flops=4.0 * hq * D * sum(r * n for r, n in used))


# ------------------------------------------------------- the same in 64 bits

CODES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _scales64():
    """All finite e4m3 numbers above zero, ascending: number i has the code i + 1."""
    x = [m * 2.0 ** -9 for m in range(1, 8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)]
    return torch.tensor(x[:-1], dtype=torch.float64, device="cuda")


def _nearest(x, values, first=0):
    """Which of the ascending values is nearest to each x; ties to the one with the even code (index + first)."""
    hi = torch.searchsorted(values, x).clamp(1, len(values) - 1)
    lo = hi - 1
    a, b = x - values[lo], values[hi] - x
    return torch.where((a < b) | ((a == b) & ((lo + first) % 2 == 0)), lo, hi)


def _through64(x, f):
    """x [..., Hkv, 128] as 4 bits hold it, f [Hkv] or None."""
    f = 1.0 if f is None else f.double()[:, None, None]
    codes, scales = torch.tensor(CODES, dtype=torch.float64, device="cuda"), _scales64()
    g = x.double().view(*x.shape[:-1], D // GROUP, GROUP) / f
    scale = scales[_nearest(g.abs().max(-1, keepdim=True).values / 6, scales, 1)]
    return (codes[_nearest(g.abs() / scale, codes)] * g.sign() * scale * f).view(x.shape)


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


def _session64(s, x, b, n, layer=0):
    """The first n rows of session b, [n][Hkv][128]."""
    p, page = s["pools"], s["case"]["page"]
    ids = s["table"][b, :-(-n // page)].long()
    code = p[x][layer][ids].long().transpose(1, 2).flatten(0, 1)[:n]
    scale = p[x + "_scale"].view(torch.uint8)[layer][ids].long().transpose(1, 2).flatten(0, 1)[:n]
    table = torch.tensor(CODES + tuple(-c for c in CODES), dtype=torch.float64, device="cuda")
    value = table[torch.stack([code % 16, code // 16], -1)].view(*code.shape[:-1], D // GROUP, GROUP)
    size = torch.cat([torch.zeros(1, dtype=torch.float64, device="cuda"), _scales64()])[scale]
    f = p[x + "_factor"]
    y = (value * size[..., None]).flatten(-2)
    return y if f is None else y * f.double()[:, None]


def _step64(s):
    """A step, session by session, on lists."""
    page = s["case"]["page"]
    table, free, n = s["table"].tolist(), s["free"].tolist(), int(s["n_free"])
    M, places = len(table[0]), s["slot"].numel()
    have, keep, fresh = (s[x].tolist() for x in ("len", "keep", "fresh"))
    keep = [min(k, h) for k, h in zip(keep, have)]
    top = n
    for row, h, k in zip(table, have, keep):
        for i in range(-(-k // page), -(-h // page)):
            free[top] = row[i]
            top += 1
    pages_asked = tokens_asked = 0
    slot, cu, at = [], [0], top
    for b, (row, k, f) in enumerate(zip(table, keep, fresh)):
        first, need = -(-k // page), -(-(k + f) // page)
        ok = k + f <= M * page
        if ok:
            pages_asked += need - first
            ok = need == first or pages_asked <= top
        if ok:
            tokens_asked += f
            ok = f == 0 or tokens_asked <= places
        if not ok:
            f, need = 0, first
        for i in range(first, need):
            at -= 1
            row[i] = free[at]
        slot += [row[r // page] * page + r % page for r in range(k, k + f)]
        cu.append(cu[-1] + f)
        have[b] = k + f
    slot += [-1] * (places - len(slot))
    return dict(table=_ints(table), len=_ints(have), cu_new=_ints(cu), free=_ints(free), n_free=_ints([at]), slot=_ints(slot))


def exact(case, seed):
    s = prepare(case, seed)
    kind, hkv = case["kind"], case["hkv"]
    if kind == "step":
        return _step64(s)
    if kind == "compact":
        return {x: torch.stack([_through64(torch.stack([s[x][l, s["idx"][l, h].long(), h] for h in range(hkv)], 1),
                                           s["pools"][x + "_factor"]) for l in range(case["layers"])]) for x in "kv"}
    rows, new = _lengths(case)
    if kind == "append":
        t = sum(new)
        q = _rotated64(s["q"], s["q_norm"], s)
        q[t:] = 0
        kv = dict(k=_through64(_rotated64(s["k"], s["k_norm"], s), s["pools"]["k_factor"]), v=_through64(s["v"], s["pools"]["v_factor"]))
        for x in "kv":
            kv[x][t:] = 0
            kv[x] = kv[x][None]
        return dict(q=q, **kv)
    if kind == "fetch":
        return {x: torch.stack([torch.cat([_session64(s, x, b, n, l) for b, n in enumerate(rows)]) for l in range(case["layers"])])
                for x in "kv"}
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    G, t = case["hq"] // hkv, 0
    for b, (n, m) in enumerate(zip(rows, new)):
        k, v = (_session64(s, x, b, n) for x in "kv")
        for i in range(m):
            sees = n - (m - 1 - i)
            if sees > 0:
                qi = s["q"][t + i].double().view(hkv, G, D)
                p = torch.softmax(torch.einsum("hgd,nhd->hgn", qi, k[:sees]) / math.sqrt(D), -1)
                out[t + i] = torch.einsum("hgn,nhd->hgd", p, v[:sees]).reshape(-1, D)
        t += m
    return out
