"""Serving several conversations about the same images: rotary positions, paged caches, attention over a shared prefix.

Three operators, each as its definition in elementary torch operations (`own = False`) and as the calls of the library (`own = True`):

  rotate   rotary positions with several axes (frame, row, column) on the queries and keys of a layer
  append   new keys and values into the pages of a cache, the keys (and, where given, the queries) rotated on the way
  decode   one query per head against the pages of its conversation and those of a prefix that several conversations share

`listed` holds the cases that are looked at one by one, `draw` makes more of the same ranges.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
GAMMA = 1.75           # strength of the queries' common direction in the synthetic inputs
THETA = 10000.0
GOLDEN = 0.6180339887498949


def listed():
    return [
        # one new token each of eight conversations, text only: the call between two launches of a decode step, all latency
        dict(name="rotate-step-8", kind="rotate", B=8, Hq=28, Hkv=4, n=1, d=128, dtype="bf16", sections="64", layout="halves", inverse=False, order="head"),
        # a long video: frame, row and column as axes, queries and keys as slices of one projection
        dict(name="rotate-video-18432", kind="rotate", B=1, Hq=28, Hkv=4, n=18432, d=128, dtype="bf16", sections="16-24-24", layout="halves", inverse=False, order="token"),
        # an image on a grid, half of the channels rotated, neighbours paired, the rotation taken back (also: the gradient)
        dict(name="rotate-image-2933-back-f32", kind="rotate", B=2, Hq=8, Hkv=8, n=2933, d=64, dtype="f32", sections="8-8", layout="neighbours", inverse=True, order="head"),
        # a decode step of 64 conversations: queries and keys rotated, keys and values into their pages
        dict(name="append-step-64", kind="append", B=64, Hq=28, Hkv=4, n=1, d=128, dtype="bf16", page=64, sections="16-24-24", queries=True, kept=1.0, ragged=False, start=300),
        # the next piece of five prompts of unequal lengths, in small pages, fp32
        dict(name="append-chunk-777-f32", kind="append", B=5, Hq=8, Hkv=8, n=777, d=64, dtype="f32", page=16, sections="32", queries=True, kept=1.0, ragged=True, start=200),
        # the tokens that a video layer keeps move into pages (keys rotated before they were scored)
        dict(name="append-video-evicted", kind="append", B=1, Hq=28, Hkv=4, n=18432, d=128, dtype="bf16", page=64, sections="", queries=False, kept=0.39, ragged=False, start=0),
        # every token of a stack layer into empty pages
        dict(name="append-stack-8192", kind="append", B=4, Hq=32, Hkv=32, n=8192, d=128, dtype="bf16", page=128, sections="64", queries=False, kept=1.0, ragged=False, start=0),
        # two short questions about one small image, fp32: the smallest step
        dict(name="decode-image-2-f32", kind="decode", B=2, Hq=4, Hkv=4, d=64, dtype="f32", page=16, groups=1, prefix=576, own=40),
        # eight questions about one video whose cache was thinned: every KV head has kept another number of tokens
        dict(name="decode-video-8", kind="decode", B=8, Hq=28, Hkv=4, d=128, dtype="bf16", page=64, groups=1, prefix=7200, own=300),
        # many conversations about three images, a KV head for every query head, small pages
        dict(name="decode-images-32", kind="decode", B=32, Hq=32, Hkv=32, d=128, dtype="bf16", page=16, groups=3, prefix=2933, own=200),
        # a server's batch: 64 conversations over four long videos, none thinned
        dict(name="decode-videos-64", kind="decode", B=64, Hq=32, Hkv=8, d=128, dtype="bf16", page=128, groups=4, prefix=18432, own=2000),
        # nothing shared, unequal lengths up to a very long one
        dict(name="decode-unshared-16", kind="decode", B=16, Hq=28, Hkv=4, d=128, dtype="bf16", page=256, groups=0, prefix=0, own=33000),
    ]


HEADS = [(4, 4), (8, 2), (8, 8), (14, 2), (28, 4), (32, 8), (32, 32), (40, 40)]     # (Hq, Hkv) of the repository's configurations and tests
SECTIONS = {64: ["32", "8-12-12", "16-16", "16", "8-8"], 128: ["64", "16-24-24", "32-32", "32", "16-16"]}


def draw(rng):
    """One more case: sizes spread over their logarithm, odd ones as likely as round ones, every type and layout."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        kind = rng.choice(["rotate", "append", "append", "decode", "decode", "decode"])
        Hq, Hkv = rng.choice(HEADS)
        d = rng.choice([64, 128, 128])
        c = dict(kind=kind, B=spread(1, 64), Hq=Hq, Hkv=Hkv, d=d, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]))
        if kind == "rotate":
            c.update(n=spread(1, 20000), sections=rng.choice(SECTIONS[d]), layout=rng.choice(["halves", "neighbours"]), inverse=rng.random() < 0.25,
                     order=rng.choice(["head", "token"]))
        elif kind == "append":
            n = rng.choice([1, 1, spread(2, 20000)])
            c.update(n=n, page=rng.choice([16, 32, 64, 128, 256]), sections=rng.choice(SECTIONS[d] + [""]), queries=rng.random() < 0.5,
                     kept=1.0, ragged=n > 1 and rng.random() < 0.5, start=rng.choice([0, spread(1, 2000)]))
            if n > 1 and rng.random() < 0.4:
                c.update(kept=round(rng.uniform(0.12, 0.6), 3), queries=False, ragged=False, sections="")
            c["queries"] = c["queries"] and c["sections"] != ""
        else:
            groups = rng.choice([0, 1, 1, 2, 3, 4])
            c.update(page=rng.choice([16, 32, 64, 128, 256]), groups=min(groups, c["B"]), prefix=spread(100, 20000) if groups else 0,
                     own=spread(1, 2000) if groups else spread(20, 33000))
        w = work(c)
        rate = 16.0 if c["dtype"] == "f32" else 1.0                      # fp32 products run at a sixteenth of the bf16 rate
        if w["bytes"] > 1.0e9 or w["flops"] * rate > 3e11 or state_bytes(c) > 3e9:
            continue
        return c


def elem(case):
    return 2 if case["dtype"] == "bf16" else 4


def counts(case):
    """append: tokens that each batch element (or, where tokens were dropped, each unit) brings."""
    n, B = case["n"], case["B"]
    if case["kept"] < 1.0:
        return [max(1, int(n * case["kept"] * (0.8 + 0.4 * ((u * GOLDEN) % 1.0)))) for u in range(B * case["Hkv"])]
    if case["ragged"]:
        return [int(n * ((1 + b) * GOLDEN % 1.0)) if b else n for b in range(B)]
    return [n] * B


def lengths(case):
    """decode: (own length of each conversation, prefix length of each group and KV head, first conversation of each group)."""
    B, P = case["B"], case["groups"]
    own_len = [case["own"] if b == B // 2 else max(1, int(case["own"] * (0.08 + 0.6 * (((b + 1) * GOLDEN) % 1.0) ** 2))) for b in range(B)]
    pre_len = [max(1, int(case["prefix"] * (1.0 if u == 0 else 0.85 + 0.15 * ((u * GOLDEN) % 1.0)))) for u in range(P * case["Hkv"])]
    begin = [int(round(B * (p / P) ** 1.2)) for p in range(P + 1)] if P else [0]
    return own_len, pre_len, begin


def state_bytes(case):
    if case["kind"] == "decode":
        own_len, pre_len, _ = lengths(case)
        # the plain form gathers the conversations' rows in 32 bits, all as long as the longest
        return (case["B"] * case["Hkv"] * max(own_len) + sum(pre_len)) * case["d"] * 8.0
    return (2.0 * case["Hq"] + 6.0 * case["Hkv"]) * case["B"] * case["n"] * case["d"] * elem(case)


def work(case):
    """What one pass cannot do without: inputs read once, outputs written once; a rotation is six operations a pair."""
    B, Hq, Hkv, d, e = case["B"], case["Hq"], case["Hkv"], case["d"], elem(case)
    if case["kind"] == "rotate":
        axes = len(case["sections"].split("-"))
        x = float(B) * (Hq + Hkv) * case["n"] * d
        pairs = sum(int(s) for s in case["sections"].split("-"))
        return {"bytes": 2.0 * x * e + 4.0 * axes * B * case["n"], "flops": 6.0 * pairs * x / d}
    if case["kind"] == "append":
        cnt = counts(case)
        tokens = float(sum(cnt))
        rows = tokens if case["kept"] < 1.0 else tokens * Hkv
        turned = (rows if case["sections"] else 0.0) + (tokens * Hq if case["queries"] else 0.0)
        pairs = sum(int(s) for s in case["sections"].split("-")) if case["sections"] else 0
        b = 4.0 * rows * d * e + (2.0 * tokens * Hq * d * e if case["queries"] else 0.0) + (4.0 * rows if case["kept"] < 1.0 else 0.0)
        return {"bytes": b, "flops": 6.0 * pairs * turned}
    own_len, pre_len, begin = lengths(case)
    rows = float(sum(own_len)) * Hkv + float(sum(pre_len))
    pairs = float(sum(own_len)) * Hq
    for p in range(case["groups"]):
        pairs += (begin[p + 1] - begin[p]) * (Hq // Hkv) * float(sum(pre_len[p * Hkv:(p + 1) * Hkv]))
    return {"bytes": 2.0 * rows * d * e + 2.0 * B * Hq * d * e, "flops": 4.0 * d * pairs}


# ---------------------------------------------------------------- inputs
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEVICE, dtype=torch.float32)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _positions(case, g, axes):
    """[axes, B, n]: some text (all axes alike), then frames of 12 x 12 patches (frame, row, column), somewhere in a conversation;
    the decode step has the same position on every axis."""
    B, n = case["B"], case["n"]
    t = torch.arange(n, device=DEVICE)
    text = n if n < 32 else n // 8
    v = (t - text).clamp(min=0)
    seen = t >= text
    grid = [torch.where(seen, text + v // 144, t), torch.where(seen, text + v % 144 // 12, t), torch.where(seen, text + v % 12, t)]
    grid = grid[3 - axes:] if axes > 1 else [t]
    first = torch.randint(0, 60000, (1, B, 1), generator=g, device=DEVICE)
    return (torch.stack(grid)[:, None, :] + first).to(torch.int32).contiguous()


def _frequencies(case):
    """Radians a position, and the axis, of every pair: a geometric row over all pairs, cut into the axes' sections."""
    sections = [int(s) for s in case["sections"].split("-")]
    pairs = sum(sections)
    return [THETA ** (-i / pairs) for i in range(pairs)], [a for a, s in enumerate(sections) for _ in range(s)]


def _layer(case, g):
    """Q, K, V of a layer, [B, H, n, d]; in order "token" as slices of one projection [B, n, Hq + 2 Hkv, d]."""
    B, Hq, Hkv, n, d = case["B"], case["Hq"], case["Hkv"], case["n"], case["d"]
    u = _randn(g, B, Hkv, 1, d)
    u = u / u.norm(dim=-1, keepdim=True)
    Q = (_randn(g, B, Hq, n, d) + GAMMA * math.sqrt(d) * u.repeat_interleave(Hq // Hkv, dim=1)).to(_dtype(case))
    K = (_randn(g, B, Hkv, n, d) + 2.5 * u * (torch.rand((B, Hkv, n, 1), generator=g, device=DEVICE) < 0.1)).to(_dtype(case))
    V = _randn(g, B, Hkv, n, d).to(_dtype(case))
    if case.get("order") == "token":
        x = torch.cat([Q, K, V], dim=1).transpose(1, 2).contiguous().transpose(1, 2)
        Q, K, V = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    return Q, K, V


def _pages(g, num_pages, rows, width):
    """A table [rows, width] of different pages, in no order: what an allocator leaves after a while."""
    return torch.randperm(num_pages, generator=g, device=DEVICE)[:rows * width].view(rows, width).to(torch.int32)


def _append_inputs(case, seed):
    g = _generator(seed)
    B, Hkv, n, d, page = case["B"], case["Hkv"], case["n"], case["d"], case["page"]
    units = B * Hkv
    s = {}
    s["Q"], s["K"], s["V"] = _layer(case, g)
    cnt = counts(case)
    if case["kept"] < 1.0:
        order = torch.rand((units, n), generator=g, device=DEVICE).argsort(dim=1)
        s["idx"] = torch.zeros((units, n), dtype=torch.int32, device=DEVICE)
        for u in range(units):
            s["idx"][u, :cnt[u]] = order[u, :cnt[u]].sort().values.to(torch.int32)
        s["k"] = _ints(cnt)
    else:
        s["idx"] = None
        s["k"] = _ints([c for c in cnt for _ in range(Hkv)]) if case["ragged"] else None
    s["start"] = _ints([case["start"] * (3 + u * 7 % 5) // 7 for u in range(units)])
    width = -(-(case["start"] + (max(cnt) if cnt else n)) // page)
    num_pages = units * width + 3
    s["table"] = _pages(g, num_pages, units, width)
    s["pool_K"], s["pool_V"] = _randn(g, num_pages, page, d).to(_dtype(case)), _randn(g, num_pages, page, d).to(_dtype(case))
    s["pos"] = _positions(case, g, len(case["sections"].split("-"))) if case["sections"] else None
    return s


def _decode_inputs(case, seed):
    g = _generator(seed)
    B, Hq, Hkv, d, page, P = case["B"], case["Hq"], case["Hkv"], case["d"], case["page"], case["groups"]
    own_len, pre_len, begin = lengths(case)
    s = {}
    wide_own, wide_pre = -(-max(own_len) // page), -(-max(pre_len) // page) if P else 0
    # only the pages in use exist; a conversation's table is as wide as the longest needs and repeats its last page behind its end
    used_own = [-(-own_len[b] // page) for b in range(B) for _ in range(Hkv)]
    used_pre = [-(-x // page) for x in pre_len]
    num_pages = sum(used_own) + sum(used_pre) + 2
    order = torch.randperm(num_pages, generator=g, device=DEVICE).to(torch.int32)

    def tables(used, width, first):
        column = torch.arange(width, device=DEVICE)
        uses = torch.tensor(used, device=DEVICE)
        at = first + torch.cumsum(uses, 0) - uses
        return order[(at[:, None] + torch.minimum(column[None, :], uses[:, None] - 1)).reshape(-1)].view(len(used), width).contiguous()

    s["table"] = tables(used_own, wide_own, 0)
    s["prefix_table"] = tables(used_pre, wide_pre, sum(used_own)) if P else None
    u = _randn(g, Hkv, d)
    u = u / u.norm(dim=-1, keepdim=True)
    lean = torch.zeros((num_pages, d), device=DEVICE)                     # the page's KV head leans towards that head's queries
    lean[s["table"].long().reshape(-1)] = u.repeat(B, 1).repeat_interleave(wide_own, dim=0)
    if P:
        lean[s["prefix_table"].long().reshape(-1)] = u.repeat(P, 1).repeat_interleave(wide_pre, dim=0)
    spiked = torch.rand((num_pages, page, 1), generator=g, device=DEVICE) < 0.1
    s["pool_K"] = (_randn(g, num_pages, page, d) + 2.5 * spiked * lean[:, None, :]).to(_dtype(case))
    s["pool_V"] = _randn(g, num_pages, page, d).to(_dtype(case))
    s["q"] = (_randn(g, B, Hq, d) + GAMMA * math.sqrt(d) * u.repeat_interleave(Hq // Hkv, dim=0)).to(_dtype(case)).view(B * Hq, d)
    s["len"] = _ints([x for x in own_len for _ in range(Hkv)])
    s["prefix_len"] = _ints(pre_len) if P else None
    s["group_begin"] = _ints(begin) if P else None
    return s


def prepare(case, seed):
    kind, B, Hq, Hkv, d = case["kind"], case["B"], case["Hq"], case["Hkv"], case["d"]
    if own:
        import paper_2410_08584_amd as z
    if kind == "rotate":
        g = _generator(seed)
        s = {}
        s["Q"], s["K"], _ = _layer(case, g)
        s["pos"] = _positions(case, g, len(case["sections"].split("-")))
    elif kind == "append":
        s = _append_inputs(case, seed)
    else:
        s = _decode_inputs(case, seed)
    s["case"] = dict(case)
    if kind != "decode" and case["sections"]:
        freqs, axis = _frequencies(case)
        layout = case.get("layout", "halves")
        s["layout"], s["back"] = layout, bool(case.get("inverse"))
        if own:
            s["rope"] = z.Rope(freqs, axis, z.ROPE_NEIGHBOURS if layout == "neighbours" else z.ROPE_HALVES)
        s["freqs"], s["axis"] = torch.tensor(freqs, dtype=torch.float64, device=DEVICE), torch.tensor(axis, device=DEVICE)
    elif own:
        s["rope"] = None
    if kind == "rotate":
        s["Qo"], s["Ko"] = torch.empty_like(s["Q"], memory_format=torch.contiguous_format), torch.empty_like(s["K"], memory_format=torch.contiguous_format)
    if kind == "append":
        s["Qo"] = torch.zeros_like(s["Q"], memory_format=torch.contiguous_format) if case["queries"] else None
        s["len"] = torch.zeros_like(s["start"])
        if own:
            s["cache"] = z.PagedCache(s["pool_K"], s["pool_V"])
    if kind == "decode":
        s["scale"] = 1.0 / math.sqrt(d)
        s["o"] = torch.zeros_like(s["q"])
        s["begin"] = lengths(case)[2]
        s["own_max"], s["prefix_max"] = max(lengths(case)[0]), max(lengths(case)[1], default=0)
        if own:
            s["cache"] = z.PagedCache(s["pool_K"], s["pool_V"])
            s["ws"] = z.decode_paged_workspace(s["cache"], s["table"], s["prefix_table"], B=B, Hq=Hq, Hkv=Hkv)
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    if not own:
        return {"rotate": plain_rotate, "append": plain_append, "decode": plain_decode}[case["kind"]](s)
    import paper_2410_08584_amd as z
    if case["kind"] == "rotate":
        z.zipvl_rotate(s["Q"], s["K"], s["pos"], s["rope"], z.ROTATE_INVERSE if s["back"] else 0, Qo=s["Qo"], Ko=s["Ko"])
        return {"Q": s["Qo"], "K": s["Ko"]}
    if case["kind"] == "append":
        z.zipvl_paged_append(s["K"], s["V"], s["cache"], s["table"], s["start"], idx=s["idx"], k=s["k"], pos=s["pos"], rope=s["rope"],
                             Q=s["Q"] if case["queries"] else None, Qo=s["Qo"], length=s["len"])
        out = {"K": s["pool_K"], "V": s["pool_V"], "len": s["len"]}
        return dict(out, Q=s["Qo"]) if case["queries"] else out
    return z.zipvl_decode_attn_paged(s["q"], s["cache"], s["table"], s["len"], s["scale"], B=case["B"], Hq=case["Hq"], Hkv=case["Hkv"],
                                     prefix_table=s["prefix_table"], prefix_len=s["prefix_len"], group_begin=s["group_begin"], o=s["o"], ws=s["ws"])


def _turned(x, pos, freqs, axis, layout, back):
    """x [B, H, n, d] with pair i turned by pos[axis_i] * freqs_i; angles in 64 bits (a far position times a frequency)."""
    pairs = freqs.numel()
    angle = pos[axis].permute(1, 2, 0).to(torch.float64) * freqs         # [B, n, pairs]
    c, sn = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if back:
        sn = -sn
    f = x.float()
    if layout == "halves":
        a, b = f[..., :pairs], f[..., pairs:2 * pairs]
        out = torch.cat([a * c - b * sn, a * sn + b * c, f[..., 2 * pairs:]], dim=-1)
    else:
        a, b = f[..., 0:2 * pairs:2], f[..., 1:2 * pairs:2]
        out = torch.cat([torch.stack([a * c - b * sn, a * sn + b * c], dim=-1).flatten(-2), f[..., 2 * pairs:]], dim=-1)
    return out.to(x.dtype)


def plain_rotate(s):
    turn = (s["pos"], s["freqs"], s["axis"], s["layout"], s["back"])
    return {"Q": _turned(s["Q"], *turn), "K": _turned(s["K"], *turn)}


def plain_append(s):
    case = s["case"]
    B, Hq, Hkv, n, d, page = case["B"], case["Hq"], case["Hkv"], case["n"], case["d"], case["page"]
    units = B * Hkv
    K, V = s["K"], s["V"]
    if case["sections"]:
        K = _turned(K, s["pos"], s["freqs"], s["axis"], "halves", False)
    rows = torch.arange(n, device=DEVICE)
    cnt = torch.full((units,), n, device=DEVICE) if s["k"] is None else s["k"].long()
    new = rows[None, :] < cnt[:, None]                                    # [units, n]
    at = s["start"].long()[:, None] + rows[None, :]
    where = torch.gather(s["table"].long(), 1, (at // page).clamp(max=s["table"].shape[1] - 1)) * page + at % page
    K, V = K.reshape(units, n, d), V.reshape(units, n, d)
    if s["idx"] is not None:
        pick = s["idx"].long()[:, :, None].expand(units, n, d)
        K, V = torch.gather(K, 1, pick), torch.gather(V, 1, pick)
    s["pool_K"].view(-1, d)[where[new]] = K[new]
    s["pool_V"].view(-1, d)[where[new]] = V[new]
    s["len"].copy_(s["start"] + cnt)
    out = {"K": s["pool_K"], "V": s["pool_V"], "len": s["len"]}
    if case["queries"]:
        turned = _turned(s["Q"], s["pos"], s["freqs"], s["axis"], "halves", False)
        seen = (rows[None, :] < cnt.view(B, Hkv)[:, :1])[:, None, :, None]
        s["Qo"].copy_(torch.where(seen, turned, s["Qo"]))
        out["Q"] = s["Qo"]
    return out


def plain_decode(s):
    case = s["case"]
    B, Hq, Hkv, d, P = case["B"], case["Hq"], case["Hkv"], case["d"], case["groups"]
    G = Hq // Hkv
    q = s["q"].float().view(B * Hkv, G, d)

    def rows(pool, table, longest):
        return pool[table.long()].view(table.shape[0], -1, d)[:, :longest].float()

    K, V = rows(s["pool_K"], s["table"], s["own_max"]), rows(s["pool_V"], s["table"], s["own_max"])
    logits = torch.matmul(q, K.transpose(1, 2).contiguous()) * s["scale"]                      # [units, G, own]
    behind = torch.arange(s["own_max"], device=DEVICE)[None, None, :] >= s["len"][:, None, None]
    logits = logits.masked_fill(behind, -math.inf)
    if P == 0:
        w = torch.exp(logits - logits.amax(dim=-1, keepdim=True))
        o = torch.matmul(w, V) / w.sum(dim=-1, keepdim=True)
        return o.view(B * Hq, d).to(s["q"].dtype)
    Kp, Vp = rows(s["pool_K"], s["prefix_table"], s["prefix_max"]), rows(s["pool_V"], s["prefix_table"], s["prefix_max"])
    column = torch.arange(s["prefix_max"], device=DEVICE)
    out = torch.empty((B, Hkv, G, d), device=DEVICE)
    for p in range(P):                                                    # the group's queries against its prefix, once
        a, b = s["begin"][p], s["begin"][p + 1]
        if a == b:
            continue
        mine = slice(p * Hkv, (p + 1) * Hkv)
        qg = q.view(B, Hkv, G, d)[a:b].transpose(0, 1).reshape(Hkv, (b - a) * G, d)
        lp = torch.matmul(qg, Kp[mine].transpose(1, 2).contiguous()) * s["scale"]              # [Hkv, S G, prefix]
        lp = lp.masked_fill(column[None, None, :] >= s["prefix_len"][mine, None, None], -math.inf)
        lo = logits.view(B, Hkv, G, -1)[a:b]
        top = torch.maximum(lp.amax(dim=-1).view(Hkv, b - a, G).transpose(0, 1), lo.amax(dim=-1))[..., None]
        wp = torch.exp(lp - top.transpose(0, 1).reshape(Hkv, (b - a) * G, 1))
        wo = torch.exp(lo - top)
        num = torch.matmul(wp, Vp[mine]).view(Hkv, b - a, G, d).transpose(0, 1) + torch.matmul(wo, V.view(B, Hkv, -1, d)[a:b])
        out[a:b] = num / (wp.sum(dim=-1).view(Hkv, b - a, G).transpose(0, 1) + wo.sum(dim=-1))[..., None]
    return out.view(B * Hq, d).to(s["q"].dtype)


# ---------------------------------------------------------------- the definitions in 64 bits, token by token or unit by unit
def _exact_rotation(x, pos, case):
    """x [B, H, n, d] in 64 bits, one pair of channels after the other."""
    freqs, axis = _frequencies(case)
    pairs, out = len(freqs), x.double().clone()
    for i in range(pairs):
        a, b = (i, i + pairs) if case.get("layout", "halves") == "halves" else (2 * i, 2 * i + 1)
        angle = (-1.0 if case.get("inverse") else 1.0) * pos[axis[i]].double() * freqs[i]      # [B, n]
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]
        pair = torch.complex(x[..., a].double(), x[..., b].double()) * turn
        out[..., a], out[..., b] = pair.real, pair.imag
    return out


def exact(case, seed):
    kind, B, Hq, Hkv, d = case["kind"], case["B"], case["Hq"], case["Hkv"], case["d"]
    if kind == "rotate":
        g = _generator(seed)
        Q, K, _ = _layer(case, g)
        pos = _positions(case, g, len(case["sections"].split("-")))
        return {"Q": _exact_rotation(Q, pos, case), "K": _exact_rotation(K, pos, case)}
    if kind == "append":
        s, page = _append_inputs(case, seed), case["page"]
        K, V, cnt = s["K"].double(), s["V"].double(), counts(case)
        if case["sections"]:
            K = _exact_rotation(s["K"], s["pos"], case)
        pool_K, pool_V = s["pool_K"].double(), s["pool_V"].double()
        start, table, length = s["start"].tolist(), s["table"].long(), []
        for u in range(B * Hkv):
            b, h = divmod(u, Hkv)
            m = cnt[u] if case["kept"] < 1.0 else cnt[b]
            token = s["idx"][u, :m].long() if s["idx"] is not None else torch.arange(m, device=DEVICE)
            row = start[u] + torch.arange(m, device=DEVICE)
            pool_K[table[u, row // page], row % page] = K[b, h, token]
            pool_V[table[u, row // page], row % page] = V[b, h, token]
            length.append(start[u] + m)
        out = {"K": pool_K, "V": pool_V, "len": _ints(length)}
        if case["queries"]:
            out["Q"] = torch.zeros_like(s["Q"], dtype=torch.float64, memory_format=torch.contiguous_format)
            turned = _exact_rotation(s["Q"], s["pos"], case)
            for b in range(B):
                out["Q"][b, :, :cnt[b]] = turned[b, :, :cnt[b]]
        return out
    s, page, G = _decode_inputs(case, seed), case["page"], Hq // Hkv
    own_len, pre_len, begin = lengths(case)
    out = torch.zeros((B * Hq, d), dtype=torch.float64, device=DEVICE)

    def unit(table, length):
        used = table[:-(-length // page)].long()
        return s["pool_K"][used].reshape(-1, d)[:length].double(), s["pool_V"][used].reshape(-1, d)[:length].double()

    group = [next((p for p in range(case["groups"]) if begin[p] <= b < begin[p + 1]), None) for b in range(B)]
    for h in range(Hkv):
        shared = {p: unit(s["prefix_table"][p * Hkv + h], pre_len[p * Hkv + h]) for p in set(group) if p is not None}
        for b in range(B):
            K, V = unit(s["table"][b * Hkv + h], own_len[b])
            if group[b] is not None:
                K, V = torch.cat([shared[group[b]][0], K]), torch.cat([shared[group[b]][1], V])
            heads = slice(b * Hq + h * G, b * Hq + (h + 1) * G)
            w = torch.softmax(s["q"][heads].double() @ K.T / math.sqrt(d), dim=1)
            out[heads] = w @ V
    return out
