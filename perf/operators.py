"""The operators around a key/value cache that is held in 4 bits, in pages: plain forms and cases.

A case is a dict of plain values.  `listed()` gives the named ones, `draw()` more of the same ranges, `prepare()` what a
program holds before the call, `run()` one pass -- the plain form in elementary torch operations, or with `own` the
library's entry points -- `work()` the bytes and operations a pass cannot do without, `exact()` the same outputs from the
operators' definitions in 64 bits.

Kinds of pass:
  append     rows of a QKV projection: RMSNorm of each head's query and key, rotary embedding, the rotated queries out, keys and
             values into the cache in 4 bits; then what the cache holds of these tokens is read back
  attention  new tokens of every request against the request's own pages: one token each (decode), a few, or prompts (causal)
  fork       rows of the page table become other rows (beams, samples): full pages shared, partial ones copied, pages for the
             next tokens taken, rows that nobody continues freed
  compact    live pages move to the front of the pool

The cache: a page holds 64 positions of all cache heads of one layer, per head 68 * D bytes: 32 D of key codes, 2 D of key scales,
32 D of value codes, 2 D of value scales.  A value is an e2m1 code (0 .5 1 1.5 2 3 4 6 and a sign bit, two to a byte, the lower
index in the low bits) times 2^(byte - 127), one scale byte for 32 neighbouring values of a row (255: not a number).
  key codes     [position][d / 2]
  key scales    [d / 32][position % 16][position / 16]
  value codes   [d / 32][position % 16 / 4][d % 32 / 2][position / 16][position % 4]
  value scales  [d / 32][position % 16 / 4][position / 16][position % 4]
"""
from __future__ import annotations

import math
import random

import torch

own = False

PAGE = 64
EPS = 1e-6
HEADS = {"tiny": (8, 8, 64), "7b": (32, 32, 128), "13b": (40, 40, 128), "30b": (52, 52, 128), "70b": (64, 8, 128)}


def _heads(shape):
    Hq, Hkv, D = HEADS[shape]
    return dict(Hq=Hq, Hkv=Hkv, D=D)


def listed():
    return [
        # one interactive request on a small model: latency and launches
        dict(kind="append", **_heads("7b"), T=1, P=40, norm=True, far=4000, name="append_7b_t1"),
        # the everyday decode step of a served batch, far into long contexts
        dict(kind="append", **_heads("70b"), T=32, P=4000, norm=True, far=130000, name="append_70b_t32"),
        # a long prompt of a model without norms of queries and keys, an odd number of tokens
        dict(kind="append", **_heads("13b"), T=4001, P=90, norm=False, far=8000, name="append_13b_t4001"),
        # a toy or draft model with two requests
        dict(kind="attention", **_heads("tiny"), B=2, S=468, Q=1, name="decode_tiny_b2"),
        # the everyday decode batch: one token of each of 32 requests of unequal lengths
        dict(kind="attention", **_heads("7b"), B=32, S=2048, Q=1, name="decode_7b_b32"),
        # few requests with long documents, grouped heads
        dict(kind="attention", **_heads("70b"), B=4, S=131000, Q=1, name="decode_70b_b4_long"),
        # chunks of prompts next to single tokens, on caches that are there already
        dict(kind="attention", **_heads("70b"), B=6, S=8029, Q=333, name="chunks_70b_b6"),
        # one whole prompt
        dict(kind="attention", **_heads("13b"), B=1, S=4096, Q=4096, name="prompt_13b_4096"),
        # one request answered by four samples, a model's last layer only
        dict(kind="fork", **_heads("7b"), layers=1, rows=1, out=4, S=300, MP=16, P=64, name="fork_7b_4"),
        # a beam step over 64 requests of four beams, ten layers of a pipeline stage
        dict(kind="fork", **_heads("70b"), layers=10, rows=256, out=256, S=500, MP=40, P=3000, name="fork_70b_256"),
        # a small pool with a few holes
        dict(kind="compact", **_heads("tiny"), layers=4, rows=8, S=400, MP=16, P=128, name="compact_tiny_8"),
        # a pool of which a third is live, before its tail is given back
        dict(kind="compact", **_heads("70b"), layers=10, rows=64, S=700, MP=40, P=2000, name="compact_70b_64"),
    ]


def draw(rng):
    def span(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    while True:
        kind = rng.choice(["append", "append", "attention", "attention", "attention", "attention", "fork", "compact"])
        shape = _heads(rng.choice(list(HEADS)))
        if kind == "append":
            T = span(1, 5000)
            c = dict(kind=kind, **shape, T=T, P=T // PAGE + span(2, 400), norm=rng.random() < 0.7, far=span(100, 130000))
        elif kind == "attention":
            form = rng.choice(["one", "one", "few", "chunk", "prompt"])
            S = span(30, 100000) if form == "one" else span(30, 20000) if form == "few" else span(64, 8000)
            Q = 1 if form == "one" else rng.randint(2, 8) if form == "few" else span(9, 700) if form == "chunk" else S
            c = dict(kind=kind, **shape, B=span(1, 64) if form in ("one", "few") else rng.randint(1, 8), S=S, Q=min(Q, S))
        elif kind == "fork":
            rows, S = span(1, 300), span(20, 3000)
            out, MP = max(1, int(rows * rng.choice([0.5, 1, 1, 2, 4]))), S // PAGE + rng.randint(2, 20)
            c = dict(kind=kind, **shape, layers=span(1, 12), rows=rows, out=out, S=S, MP=MP, P=0)
            c["P"] = sum(-(-n // PAGE) for n in _lengths(c)) + 2 * out + span(4, 400)
        else:
            S = span(20, 3000)
            c = dict(kind=kind, **shape, layers=span(1, 12), rows=span(1, 100), S=S, MP=S // PAGE + rng.randint(2, 20), P=0)
            c["P"] = int(sum(-(-n // PAGE) for n in _lengths(c)) * rng.uniform(1.1, 3.5)) + 4
        w = work(c)
        if w["bytes"] <= 600e6 and w["flops"] <= 160e9 and _held(c) <= 2.5e9:
            return c


def _page_bytes(c):
    return c["Hkv"] * 68 * c["D"]


def _held(c):
    """Bytes of the pages that prepare() makes."""
    return _pages(c) * _page_bytes(c) * c.get("layers", 1)


def _lengths(c):
    """Positions of each request: unequal, the first the longest; a later one in a dozen is empty."""
    r = random.Random("lengths %s %s" % (c["S"], c.get("B", c.get("rows"))))
    n = c.get("B", c.get("rows"))
    return [c["S"]] + [0 if r.random() < 0.08 else max(1, int(c["S"] * r.uniform(0.25, 1.0))) for _ in range(n - 1)]


def _new_tokens(c, lens):
    """New tokens of each request: one each, or the first with Q and the others with some of Q, a single one among them."""
    r = random.Random("new %s %s %s" % (c["S"], c["B"], c["Q"]))
    if c["Q"] == 1:
        return [1] * len(lens)
    return [c["Q"]] + [r.choice([1, max(1, c["Q"] // 3), r.randint(1, c["Q"]), c["Q"]]) for _ in lens[1:]]


def _pages(c):
    if c["kind"] == "attention":
        return sum(-(-n // PAGE) for n in _lengths(c)) + 3
    return c["P"]


def _parents(c):
    """A beam step: each row's parent is drawn from the rows, a few rows end."""
    r = random.Random("parents %s %s" % (c["rows"], c["out"]))
    return [-1 if r.random() < 0.05 else min(c["rows"] - 1, int(c["rows"] * (i + r.uniform(-0.5, 1.5)) / c["out"])) if i else 0 for i in range(c["out"])]


# ---- the cache's values -------------------------------------------------------------------------------------------

_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _values_of(device):
    codes = torch.tensor(_GRID + tuple(-x for x in _GRID), device=device)
    scales = torch.tensor([2.0 ** (b - 127) for b in range(255)] + [math.nan], device=device)
    return codes, scales


def _quantise(x):
    """(codes, scale bytes) of x [..., D] in 64 bits, in blocks of 32."""
    x = x.unflatten(-1, (-1, 32))
    big = x.abs().amax(-1, keepdim=True)
    fine = torch.isfinite(big)
    part, power = torch.frexp(torch.where(fine, big, 0.0))
    e = torch.where(part <= 0.875, power - 3, power - 2).clamp(-23, 13)
    y = torch.where(fine, x, 0.0) * torch.exp2(-e.to(x.dtype))
    a = y.abs()
    code = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    code = code + 8 * torch.signbit(y)
    return code.to(torch.uint8).flatten(-2), torch.where(fine, e + 127, 255).to(torch.uint8).squeeze(-1)


def _pairs(code):
    return code[..., 0::2] | code[..., 1::2] << 4


def _store(blocks, k, v):
    """Head blocks [n, 68 D] of whole pages from keys and values [n, 64, D] (64 bits)."""
    n, _, D = k.shape
    kc, ks = _quantise(k)
    vc, vs = _quantise(v)
    blocks[:, : 32 * D] = _pairs(kc).reshape(n, -1)
    blocks[:, 32 * D: 34 * D] = ks.reshape(n, 4, 16, -1).permute(0, 3, 2, 1).reshape(n, -1)
    blocks[:, 34 * D: 66 * D] = _pairs(vc).reshape(n, 4, 4, 4, D // 32, 16).permute(0, 4, 2, 5, 1, 3).reshape(n, -1)
    blocks[:, 66 * D:] = vs.reshape(n, 4, 4, 4, D // 32).permute(0, 4, 2, 1, 3).reshape(n, -1)


def _load(blocks, D):
    """Keys and values [..., 64, D] in 32 bits of head blocks [..., 68 D]."""
    codes, scales = _values_of(blocks.device)
    lead = blocks.shape[:-1]
    kc, ks, vc, vs = blocks.split([32 * D, 2 * D, 32 * D, 2 * D], -1)

    def values(b):
        return torch.stack([codes[(b & 15).int()], codes[(b >> 4).int()]], -1)

    k = values(kc).reshape(*lead, 4, 16, D // 32, 32)
    k = k * scales[ks.int()].reshape(*lead, D // 32, 16, 4).movedim((-1, -2, -3), (-3, -2, -1)).unsqueeze(-1)
    v = values(vc).reshape(*lead, D // 32, 4, 16, 4, 4, 2)                     # [d / 32][hi][pair][i][r][2]
    v = v * scales[vs.int()].reshape(*lead, D // 32, 4, 1, 4, 4, 1)
    v = v.movedim((-3, -5, -2, -6, -4, -1), (-6, -5, -4, -3, -2, -1))           # [i][hi][r][d / 32][pair][2]
    return k.reshape(*lead, PAGE, D), v.reshape(*lead, PAGE, D)


def _places(slots, Hkv, D, page_bytes):
    """Byte addresses in the pool of tokens' key codes, key scales, value codes and value scales: [T, Hkv, D / 2 or D / 32]."""
    dev = slots.device
    page, at = (slots // PAGE).long(), (slots % PAGE).long()
    base = (page * page_bytes).view(-1, 1, 1) + (torch.arange(Hkv, device=dev) * 68 * D).view(1, -1, 1)
    at = at.view(-1, 1, 1)
    j, t = torch.arange(D // 2, device=dev), torch.arange(D // 32, device=dev)
    i, hi, r = at // 16, at % 16 // 4, at % 4
    return (base + at * (D // 2) + j, base + 32 * D + t * 64 + at % 16 * 4 + i,
            base + 34 * D + j // 16 * 1024 + hi * 256 + j % 16 * 16 + i * 4 + r, base + 66 * D + t * 64 + hi * 16 + i * 4 + r)


# ---- inputs -------------------------------------------------------------------------------------------------------


def _pool(c, g):
    """Pages of keys with a few strong channels and plain values, quantised."""
    P, Hkv, D = _pages(c), c["Hkv"], c["D"]
    pages = torch.empty(P, Hkv, 68 * D, dtype=torch.uint8, device="cuda")
    spread = torch.exp(0.5 * torch.randn(Hkv, 1, D, device="cuda", generator=g))
    flat, step = pages.view(P * Hkv, -1), max(1, (1 << 18) // (PAGE * D)) * Hkv
    for a in range(0, P * Hkv, step):
        n = min(step, P * Hkv - a)
        k = torch.randn(n, PAGE, D, device="cuda", generator=g) * spread.repeat(-(-n // Hkv), 1, 1)[:n]
        _store(flat[a: a + n], k, torch.randn(n, PAGE, D, device="cuda", generator=g))
    return pages


def _table(c, g, lens, MP):
    """Pages dealt to the requests in random order."""
    order = torch.randperm(_pages(c), device="cuda", generator=g).to(torch.int32)
    table = torch.full((len(lens), MP), -1, dtype=torch.int32, device="cuda")
    need = torch.tensor([-(-n // PAGE) for n in lens], device="cuda")
    mask = torch.arange(MP, device="cuda") < need[:, None]
    table[mask] = order[: int(need.sum())]
    return table


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    s = dict(case=c, **{k: c[k] for k in ("Hq", "Hkv", "D")})
    if c["kind"] == "append":
        T = c["T"]
        N = (Hq + 2 * Hkv) * D
        s["qkv"] = (randn(T, N) * torch.exp(0.5 * randn(N))).half()
        s["q_gamma"] = (1 + 0.2 * randn(D)).half() if c["norm"] else None
        s["k_gamma"] = (1 + 0.2 * randn(D)).half() if c["norm"] else None
        s["theta"] = torch.tensor([10000.0 ** (-2 * i / D) for i in range(D // 2)], device="cuda")
        # a prompt's run of positions in pages of random order, or the next token of each of many requests
        if T > 64:
            pos = torch.arange(T, device="cuda") + int(torch.randint(0, max(1, c["far"] - T + 1), (1,), device="cuda", generator=g))
            page = torch.randperm(c["P"], device="cuda", generator=g)
            run = pos - pos[0] // PAGE * PAGE
            slots = page[run // PAGE] * PAGE + run % PAGE
        else:
            pos = torch.randint(0, c["far"], (T,), device="cuda", generator=g)
            slots = torch.randperm(c["P"], device="cuda", generator=g).repeat(T)[:T] * PAGE + torch.arange(T, device="cuda") % PAGE
        s["positions"], s["slots"] = pos.int(), slots.int()
        s["pages"] = torch.zeros(c["P"], Hkv, 68 * D, dtype=torch.uint8, device="cuda")
        s["q_out"] = torch.empty(T, Hq, D, dtype=torch.float16, device="cuda")
        s["k_out"], s["v_out"] = (torch.empty(T, Hkv, D, dtype=torch.float16, device="cuda") for _ in range(2))
    elif c["kind"] == "attention":
        lens = _lengths(c)
        new = _new_tokens(c, lens)
        s["pages"], s["lens"] = _pool(c, g), ints(lens)
        s["table"] = _table(c, g, lens, -(-c["S"] // PAGE))
        s["max_q"], T = max(new), sum(new)
        s["offsets"] = None if c["Q"] == 1 else ints([sum(new[:i]) for i in range(len(new) + 1)])
        s["q"] = (2 * randn(T, Hq, D)).half()
        s["scale"] = D ** -0.5
        s["out"] = torch.empty(T, Hq, D, dtype=torch.float16, device="cuda")
    else:
        lens = _lengths(c)
        s["lens"], s["table"] = ints(lens), _table(c, g, lens, c["MP"])
        s["pool"] = torch.randint(-2 ** 31, 2 ** 31, (c["layers"], c["P"], _page_bytes(c) // 4), dtype=torch.int32, device="cuda", generator=g)
        held = s["table"][s["table"] >= 0].long()
        s["refs"] = torch.zeros(c["P"], dtype=torch.int32, device="cuda")
        s["refs"][held] = 1
        if c["kind"] == "fork":
            s["parents"], s["headroom"] = ints(_parents(c)), torch.ones(c["out"], dtype=torch.int32, device="cuda")
        rows = c.get("out", c["rows"])
        s["table_out"] = torch.empty(rows, c["MP"], dtype=torch.int32, device="cuda")
        s["refs_out"] = torch.empty_like(s["refs"])
        s["lens_out"] = torch.empty(rows, dtype=torch.int32, device="cuda")
        s["info"] = torch.empty(2, dtype=torch.int32, device="cuda")
    return s


# ---- plain forms --------------------------------------------------------------------------------------------------


def _rotated(x, gamma, positions, theta):
    """RMSNorm of each head and the rotation of neighbouring pairs, in 64 bits: far positions times their frequency need them, and so do
    values next to the border between two codes."""
    x = x.double()
    if gamma is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gamma.double()
    angle = (positions.double()[:, None] * theta.double())[:, None, :]
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1).flatten(-2)


def _append(s):
    T, Hq, Hkv, D = s["qkv"].shape[0], s["Hq"], s["Hkv"], s["D"]
    q, k, v = s["qkv"].view(T, Hq + 2 * Hkv, D).split([Hq, Hkv, Hkv], 1)
    q = _rotated(q, s["q_gamma"], s["positions"], s["theta"]).half()
    kc, ks = _quantise(_rotated(k, s["k_gamma"], s["positions"], s["theta"]))
    vc, vs = _quantise(v.double())
    pool = s["pages"].view(-1)
    at = _places(s["slots"], Hkv, D, Hkv * 68 * D)
    for place, what in zip(at, (_pairs(kc), ks, _pairs(vc), vs)):
        pool[place] = what
    codes, scales = _values_of(pool.device)
    back = []
    for c, e in ((at[0], at[1]), (at[2], at[3])):
        b = pool[c]
        x = torch.stack([codes[(b & 15).int()], codes[(b >> 4).int()]], -1).unflatten(2, (-1, 16)) * scales[pool[e].int()][..., None, None]
        back.append(x.flatten(2).half())
    return q, back[0], back[1]


def _attention(s):
    B, MP = s["table"].shape
    T, Hq, D = s["q"].shape
    Hkv, dev = s["Hkv"], s["q"].device
    off = torch.arange(B + 1, device=dev) if s["offsets"] is None else s["offsets"].long()
    new, i = off[1:] - off[:-1], torch.arange(s["max_q"], device=dev)
    there = i < new[:, None]
    rows = (off[:-1, None] + i).clamp(max=T - 1)
    live = (s["table"] >= 0) & (s["table"] < s["pages"].shape[0])
    k, v = _load(s["pages"][torch.where(live, s["table"], 0).long()], D)
    k, v = (x.transpose(1, 2).reshape(B, Hkv, MP * PAGE, D) for x in (k, v))
    q = s["q"][rows].float().reshape(B, s["max_q"], Hkv, -1, D).permute(0, 2, 1, 3, 4)
    t = (q.reshape(B, Hkv, -1, D) @ k.transpose(-1, -2)).view(B, Hkv, s["max_q"], -1, MP * PAGE) * s["scale"]
    last = s["lens"].long()[:, None] - new[:, None] + i
    at = torch.arange(MP * PAGE, device=dev)
    seen = (at <= last[..., None]) & (at < s["lens"][:, None, None]) & live.repeat_interleave(PAGE, 1)[:, None]
    t = t.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = t.amax(-1, keepdim=True)
    t = torch.exp(t.sub_(torch.where(torch.isneginf(top), 0.0, top)))
    total = t.sum(-1, keepdim=True)
    o = (t.flatten(2, 3) @ v).view(*t.shape[:-1], D)
    o = torch.where(total == 0, 0.0, o / total)
    o = o.permute(0, 2, 1, 3, 4).reshape(B, s["max_q"], Hq, D).half()
    out = torch.empty(T, Hq, D, dtype=torch.float16, device=dev)
    out[rows[there]] = o[there]
    return out


def _fork(s):
    table, lens, refs, parents = s["table"].long(), s["lens"].long(), s["refs"], s["parents"].long()
    (R, MP), N, P, dev = table.shape, parents.numel(), refs.numel(), table.device
    ok = (parents >= 0) & (parents < R)
    p, row, j = parents.clamp(0, R - 1), torch.arange(N, device=dev), torch.arange(MP, device=dev)
    n = torch.where(ok, lens[p].clamp(0, MP * PAGE), 0)
    full, used = (n // PAGE)[:, None], (-(-n // PAGE))[:, None]
    want = (-(-(n + s["headroom"].clamp(min=0)) // PAGE)).clamp(max=MP)[:, None]
    first = torch.full((R,), N, device=dev).scatter_reduce_(0, p, torch.where(ok, row, N), "amin")
    src = table[p]
    valid = ok[:, None] & (src >= 0) & (src < P)
    mine = valid & (ok & (first[p] == row))[:, None] & (refs[src.clamp(0, P - 1)] == 1)      # its parent's pages that no other row has
    part = (j >= full) & (j < used)
    fresh = (part & valid | (j >= used) & (j < want)) & ~mine
    rank = (fresh.flatten().long().cumsum(0) - 1).view(N, MP)
    free = (refs == 0).nonzero().flatten()
    got = fresh & (rank < free.numel())
    page = torch.cat([free, free.new_zeros(1)])[torch.where(got, rank, free.numel())]
    kept = ~fresh & valid & (j < torch.maximum(used, want))
    out = torch.where(got, page, torch.where(kept, src, -1))
    copy = got & part
    s["pool"][:, page[copy]] = s["pool"][:, src[copy]]

    def count(t):
        t = t[(t >= 0) & (t < P)]
        return torch.zeros(P, dtype=torch.int32, device=dev).index_add_(0, t, torch.ones_like(t, dtype=torch.int32))

    info = torch.stack([got.sum(), (fresh & ~got).sum()]).int()
    return refs - count(table) + count(out), out.int(), n.int(), info, s["pool"]


def _compact(s):
    table, refs = s["table"].long(), s["refs"]
    P, live = refs.numel(), refs > 0
    L = live.sum()
    index = torch.arange(P, device=refs.device)
    holes, movers = (~live & (index < L)).nonzero().flatten(), (live & (index >= L)).nonzero().flatten()
    to = index.clone()
    to[movers] = holes
    there = (table >= 0) & (table < P)
    e = table.clamp(0, P - 1)
    out = torch.where(there & live[e], to[e], -1)
    refs_out = torch.zeros_like(refs)
    refs_out[to[live]] = refs[live]
    s["pool"][:, holes] = s["pool"][:, movers]
    return refs_out, out.int(), torch.stack([L, torch.tensor(holes.numel(), device=L.device)]).int(), s["pool"]


def _library(s):
    """The same through the library, with the workspace that a program keeps."""
    import paper_2605_25655_amd as thi
    kind = s["case"]["kind"]
    if kind == "append":
        thi.thi_qk_norm_rope_kv4(s["qkv"], s["q_gamma"], s["k_gamma"], EPS, s["positions"], s["theta"], s["slots"], s["q_out"], s["pages"])
        thi.thi_kv4_read(s["pages"], s["slots"], s["k_out"], s["v_out"])
        return s["q_out"], s["k_out"], s["v_out"]
    if kind == "attention":
        if "ws" not in s:
            B, MP = s["table"].shape
            s["ws"] = thi.Workspace(thi.thi_kv4_attention_workspace_bytes(B, s["q"].shape[0], s["Hq"], s["Hkv"], s["D"], s["max_q"], MP), init=False)
        thi.thi_kv4_attention(s["q"], s["pages"], s["table"], s["lens"], s["offsets"], s["scale"], s["out"], s["max_q"], s["ws"])
        return s["out"]
    if "ws" not in s:
        s["ws"] = thi.Workspace(thi.thi_kv4_pages_workspace_bytes(s["table_out"].shape[0], *s["table"].shape, s["refs"].numel()), init=False)
    if kind == "fork":
        thi.thi_kv4_fork(s["refs"], s["table"], s["lens"], s["parents"], s["headroom"], s["refs_out"], s["table_out"], s["lens_out"],
                         s["info"], s["pool"], s["ws"])
        return s["refs_out"], s["table_out"], s["lens_out"], s["info"], s["pool"]
    thi.thi_kv4_compact(s["refs"], s["table"], s["refs_out"], s["table_out"], s["info"], s["pool"], s["ws"])
    return s["refs_out"], s["table_out"], s["info"], s["pool"]


def run(state):
    """Fork and compaction take tables and counts and give others, so a pass can be repeated: it copies the same pages again."""
    if own:
        return _library(state)
    return {"append": _append, "attention": _attention, "fork": _fork, "compact": _compact}[state["case"]["kind"]](state)


# ---- what a pass cannot do without --------------------------------------------------------------------------------


def work(case):
    c = case
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    if c["kind"] == "append":
        T, held = c["T"], c["T"] * 2 * Hkv * D * 17 / 32
        return {"bytes": T * (2 * Hq + 2 * Hkv) * D * 2 + held + held + T * 2 * Hkv * D * 2 + 12 * T, "flops": 12 * T * (Hq + 2 * Hkv) * D}
    lens = _lengths(c)
    if c["kind"] == "attention":
        new = _new_tokens(c, lens)
        pairs = sum(sum(max(0, n - m + i + 1) for i in range(m)) for n, m in zip(lens, new))
        return {"bytes": sum(lens) * 2 * Hkv * D * 17 / 32 + 2 * 2 * sum(new) * Hq * D + 4 * sum(-(-n // PAGE) for n in lens), "flops": 4 * D * Hq * pairs}
    if c["kind"] == "fork":
        parents, seen, copies = _parents(c), set(), 0
        for p in parents:
            copies += p >= 0 and p in seen and lens[p] % PAGE > 0
            seen.add(p)
        small = 4 * c["MP"] * (c["rows"] + c["out"]) + 8 * c["P"]
    else:
        live = sum(-(-n // PAGE) for n in lens)
        copies = live * (1 - live / c["P"])           # of randomly dealt pages, those behind the live ones' number
        small = 8 * c["MP"] * c["rows"] + 8 * c["P"]
    return {"bytes": 2 * copies * c["layers"] * _page_bytes(c) + small, "flops": 0}


# ---- definitions in 64 bits ---------------------------------------------------------------------------------------


def _held_at(pool, page, at, heads, D, page_bytes):
    """Keys and values that the cache holds at positions `at` of pages `page` [n]: [n, heads, D], byte by byte from the layout."""
    d = torch.arange(D, device=pool.device)
    h = torch.arange(heads, device=pool.device)[:, None]
    page, at = page[:, None, None], at[:, None, None]
    base = page * page_bytes + h * (68 * D)
    i, hi, r = at.div(16, rounding_mode="floor"), at.remainder(16).div(4, rounding_mode="floor"), at.remainder(4)

    def value(code_at, scale_at):
        b = pool[code_at].int() >> (4 * (d % 2)).int() & 15
        power, half = b >> 1 & 3, (b & 1).double()
        size = torch.where(power == 0, half / 2, (1 + half / 2) * torch.exp2(power.double() - 1))
        e = pool[scale_at].int()
        return torch.where(b >= 8, -size, size) * torch.where(e == 255, math.nan, torch.exp2(e.double() - 127))

    k = value(base + at * (D // 2) + d // 2, base + 32 * D + d // 32 * 64 + at.remainder(16) * 4 + i)
    v = value(base + 34 * D + d // 32 * 1024 + hi * 256 + d % 32 // 2 * 16 + i * 4 + r, base + 66 * D + d // 32 * 64 + hi * 16 + i * 4 + r)
    return k, v


def _nearest(x):
    """What 4 bits hold of x [..., D]: of each 32 values the smallest scale that keeps the largest within 7, then the nearest of the grid."""
    x = x.unflatten(-1, (-1, 32))
    big = x.abs().amax(-1, keepdim=True)
    scales = 2.0 ** torch.arange(-23, 14, device=x.device, dtype=torch.float64)
    scale = scales[(7 * scales < big).sum(-1, keepdim=True).clamp(max=36)]
    order = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7], device=x.device)             # of two that are as near the one with the even code
    grid = torch.tensor(_GRID, device=x.device, dtype=torch.float64)[order]
    best = grid[((x / scale).abs().unsqueeze(-1) - grid).abs().argmin(-1)]
    return (best * scale * torch.sign(x)).flatten(-2)


def exact(case, seed):
    c = case
    if c["kind"] in ("fork", "compact"):
        return None                                                           # whole numbers, and pages copied as they are
    s = prepare(c, seed)
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    if c["kind"] == "append":
        x = s["qkv"].double().view(c["T"], -1, D)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * s["theta"].double())[:, None]

        def one(y, gamma):
            if gamma is not None:
                y = y / (y.square().sum(-1, keepdim=True) / D + EPS).sqrt() * gamma.double()
            return torch.view_as_real(torch.view_as_complex(y.reshape(*y.shape[:-1], D // 2, 2).contiguous()) * turn).flatten(-2)

        q, k = one(x[:, :Hq], s["q_gamma"]), one(x[:, Hq: Hq + Hkv], s["k_gamma"])
        back = [torch.cat([_nearest(y[a: a + 256]) for a in range(0, c["T"], 256)]) for y in (k, x[:, Hq + Hkv:])]
        return q, back[0], back[1]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    pool, page_bytes = s["pages"].view(-1), _page_bytes(c)
    lens, first = s["lens"].tolist(), 0
    for b, m in enumerate(_new_tokens(c, lens)):
        n, q = lens[b], s["q"][first: first + m].double()
        at = torch.arange(n, device="cuda")
        parts = [_held_at(pool, s["table"][b, a // PAGE].long(), a % PAGE, Hkv, D, page_bytes) for a in at.split(8192)]
        k, v = (torch.cat(x) for x in zip(*parts)) if parts and n else (torch.zeros(0, Hkv, D, dtype=torch.float64, device="cuda"),) * 2
        for h in range(Hq):
            g = h // (Hq // Hkv)
            for a in range(0, m, 2048):
                rows = torch.arange(a, min(m, a + 2048), device="cuda")
                t = q[rows, h] @ k[:, g].T * s["scale"]
                w = torch.where(at <= n - m + rows[:, None], torch.exp(t - t.amax(-1, keepdim=True)) if n else t, 0.0)
                total = w.sum(-1, keepdim=True)
                out[first + rows, h] = torch.where(total > 0, w @ v[:, g] / total, 0.0)
        first += m
    return out
