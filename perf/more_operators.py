"""Pieces of prompts over paged caches, and caches that stay within a budget.

Three operators, each as its definition in elementary torch operations (`own = False`) and as the calls of the library (`own = True`):

  chunk   attention of several new tokens of every conversation to its pages and those of a prefix that conversations share, with the logarithm of every sum
  weigh   the attention weight that the rows of a cache get from new queries, on top of what they had
  evict   rows leave a cache by that weight: the first and the latest tokens and the heaviest others stay, in the pages where they are

`listed` holds the cases that are looked at one by one, `draw` makes more of the same ranges.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
GAMMA = 1.75           # strength of the queries' common direction in the synthetic inputs
GOLDEN = 0.6180339887498949


def listed():
    return [
        # two short questions about one small image, fp32: the smallest piece, all latency
        dict(name="chunk-image-5-f32", kind="chunk", B=2, Hq=4, Hkv=4, n=5, d=64, dtype="f32", page=16, groups=1, prefix=576, before=40, ragged=False),
        # eight conversations ask questions of up to 24 tokens about one video whose cache was thinned
        dict(name="chunk-questions-24", kind="chunk", B=8, Hq=28, Hkv=4, n=24, d=128, dtype="bf16", page=64, groups=1, prefix=7200, before=300, ragged=True),
        # the next 2048 tokens of a long video's prompt
        dict(name="chunk-video-2048", kind="chunk", B=1, Hq=28, Hkv=4, n=2048, d=128, dtype="bf16", page=128, groups=0, prefix=0, before=16384, ragged=False),
        # the next piece of five prompts of unequal lengths, in small pages, fp32
        dict(name="chunk-prompts-777-f32", kind="chunk", B=5, Hq=8, Hkv=8, n=777, d=64, dtype="f32", page=16, groups=0, prefix=0, before=200, ragged=True),
        # a piece of four prompts of a stack layer, a KV head for every query head
        dict(name="chunk-stack-1024", kind="chunk", B=4, Hq=32, Hkv=32, n=1024, d=128, dtype="bf16", page=256, groups=0, prefix=0, before=3000, ragged=False),
        # four drafted tokens of each of sixteen conversations are looked at, unequal lengths up to a very long one
        dict(name="chunk-draft-4", kind="chunk", B=16, Hq=28, Hkv=4, n=4, d=128, dtype="bf16", page=256, groups=0, prefix=0, before=33000, ragged=False),
        # the weights of one decode step of sixteen conversations
        dict(name="weigh-step-16", kind="weigh", B=16, Hq=28, Hkv=4, n=1, d=128, dtype="bf16", page=64, before=2048, ragged=False),
        # the last 64 queries of a video's prompt look back over its cache
        dict(name="weigh-video-64", kind="weigh", B=1, Hq=28, Hkv=4, n=64, d=128, dtype="bf16", page=128, before=18368, ragged=False),
        # every query of a piece of three prompts, fp32
        dict(name="weigh-prompts-511-f32", kind="weigh", B=3, Hq=14, Hkv=2, n=511, d=64, dtype="f32", page=32, before=3000, ragged=True),
        # 64 conversations are 16 tokens over their budget of 2048
        dict(name="evict-step-64", kind="evict", B=64, Hkv=4, d=128, dtype="bf16", page=64, rows=2064, budget=2048, sinks=4, recent=64, ragged=False),
        # a long video's cache is thinned to what fits
        dict(name="evict-video-7200", kind="evict", B=1, Hkv=4, d=128, dtype="bf16", page=128, rows=18432, budget=7200, sinks=4, recent=256, ragged=False),
        # four prompts of a stack layer, unequal lengths, fp32, small pages, the weight alone decides
        dict(name="evict-stack-2048-f32", kind="evict", B=4, Hkv=32, d=64, dtype="f32", page=16, rows=8192, budget=2048, sinks=0, recent=0, ragged=True),
    ]


HEADS = [(4, 4), (8, 2), (8, 8), (14, 2), (28, 4), (32, 8), (32, 32), (40, 40)]     # (Hq, Hkv) of the repository's configurations and tests


def draw(rng):
    """One more case: sizes spread over their logarithm, odd ones as likely as round ones, every type and page."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        kind = rng.choice(["chunk", "chunk", "chunk", "weigh", "weigh", "evict", "evict"])
        Hq, Hkv = rng.choice(HEADS)
        c = dict(kind=kind, B=spread(1, 64), Hkv=Hkv, d=rng.choice([64, 128, 128]), dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), page=rng.choice([16, 32, 64, 128, 256]))
        if kind == "evict":
            rows = spread(20, 33000)
            over = rng.choice([spread(1, 64), int(rows * rng.uniform(0.05, 0.9))])
            budget = max(8, rows - over)
            c.update(rows=rows, budget=budget, sinks=rng.choice([0, 4]), recent=rng.choice([0, min(64, budget // 4), budget // 8]), ragged=rng.random() < 0.5)
        else:
            c.update(Hq=Hq, n=rng.choice([1, spread(2, 16), spread(2, 64), spread(16, 4096), spread(16, 4096)]))
            c["ragged"] = c["n"] > 1 and rng.random() < 0.5
            c["before"] = rng.choice([0, spread(1, 2000), spread(20, 33000)]) if c["n"] > 1 else spread(20, 33000)
            if kind == "chunk":
                groups = min(rng.choice([0, 0, 1, 2, 3]), c["B"])
                c.update(groups=groups, prefix=spread(100, 20000) if groups else 0)
                if groups:
                    c["before"] = min(c["before"], 2000)
        w = work(c)
        rate = 16.0 if c["dtype"] == "f32" else 1.0                      # fp32 products run at a sixteenth of the bf16 rate
        if w["bytes"] > 8e8 or w["flops"] * rate > 4.9e11 or state_bytes(c) > 3e9:
            continue
        if kind != "evict" and float(c["B"]) * Hq * c["n"] * longest(c) > 1.1e9:      # logits of the plain form
            continue
        return c


def elem(case):
    return 2 if case["dtype"] == "bf16" else 4


def counts(case):
    """chunk, weigh: how many of the n tokens every unit brings (all heads of a conversation alike)."""
    n, B = case["n"], case["B"]
    per = [max(1, int(n * ((1 + b) * GOLDEN % 1.0))) if b and case["ragged"] else n for b in range(B)]
    return [c for c in per for _ in range(case["Hkv"])]


def lengths(case):
    """chunk, weigh: own rows of every unit, its new ones among them (heads of a conversation have kept other numbers); rows of every prefix; group bounds."""
    B, Hkv, P = case["B"], case["Hkv"], case.get("groups", 0)
    cnt = counts(case)
    rows = []
    for u in range(B * Hkv):
        b = u // Hkv
        part = 1.0 if b == B // 2 else 0.08 + 0.6 * (((b + 1) * GOLDEN) % 1.0) ** 2 if B > 4 else 0.6 + 0.4 * ((b * GOLDEN) % 1.0)
        rows.append(int(case["before"] * part * (1.0 if u % Hkv == 0 else 0.9 + 0.1 * ((u * GOLDEN) % 1.0))) + cnt[u])
    pre = [max(1, int(case["prefix"] * (1.0 if u == 0 else 0.85 + 0.15 * ((u * GOLDEN) % 1.0)))) for u in range(P * Hkv)]
    begin = [int(round(B * (p / P) ** 1.2)) for p in range(P + 1)] if P else [0]
    return rows, pre, begin


def held(case):
    """evict: rows of every unit before the call."""
    units = case["B"] * case["Hkv"]
    return [max(1, int(case["rows"] * (0.5 + 0.5 * ((u * GOLDEN) % 1.0)))) if u and case["ragged"] else case["rows"] for u in range(units)]


def longest(case):
    rows, pre, _ = lengths(case)
    return max(rows) + max(pre, default=0)


def state_bytes(case):
    if case["kind"] == "evict":
        return 2.0 * sum(held(case)) * case["d"] * elem(case)
    # the plain form gathers the conversations' rows in 32 bits, all as long as the longest
    return float(case["B"]) * case["Hkv"] * longest(case) * case["d"] * 8.0


def work(case):
    """What one pass cannot do without: inputs read once, outputs written once; products of the pairs (query, row that it sees)."""
    B, Hkv, d, e = case["B"], case["Hkv"], case["d"], elem(case)
    if case["kind"] == "evict":
        b = 0.0
        for rows in held(case):
            kept = min(rows, case["budget"])
            late, sure = rows - kept, min(case["sinks"] + case["recent"], kept)
            tail = min(case["recent"], late)
            moved = tail + (late - tail) * (kept - sure) / max(1, rows - sure)             # kept rows at or behind the new length: expected, of weights in no order
            b += 16.0 * rows + 4.0 * d * e * moved
        return {"bytes": b, "flops": 0.0}
    Hq, n = case["Hq"], case["n"]
    rows, pre, begin = lengths(case)
    cnt, G, P = counts(case), Hq // Hkv, case.get("groups", 0)
    pairs = sum(float(G) * (c * (L - c) + c * (c + 1) / 2.0) for L, c in zip(rows, cnt))
    queries = float(G) * sum(cnt)
    if case["kind"] == "weigh":
        return {"bytes": (float(sum(rows)) + queries) * d * e + 4.0 * queries + 8.0 * sum(rows), "flops": 2.0 * d * pairs}
    for p in range(P):
        pairs += sum(float(G) * cnt[b * Hkv + g] * pre[p * Hkv + g] for b in range(begin[p], begin[p + 1]) for g in range(Hkv))
    return {"bytes": 2.0 * (float(sum(rows)) + sum(pre)) * d * e + 2.0 * queries * d * e + 4.0 * queries, "flops": 4.0 * d * pairs}


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


def _tables(g, page, lists):
    """For every list of lengths a table as wide as its longest needs, of different pages in no order, as an allocator leaves them after a while; behind a
    unit's end its last page stands again."""
    used = [[max(1, -(-x // page)) for x in rows] for rows in lists]
    total = sum(sum(u) for u in used) + 2
    order = torch.randperm(total, generator=g, device=DEVICE).to(torch.int32)
    tables, first = [], 0
    for u in used:
        if not u:
            tables.append(None)
            continue
        width, need = max(u), torch.tensor(u, device=DEVICE)
        at = first + torch.cumsum(need, 0) - need
        column = torch.arange(width, device=DEVICE)
        tables.append(order[(at[:, None] + torch.minimum(column[None, :], need[:, None] - 1)).reshape(-1)].view(len(u), width).contiguous())
        first += sum(u)
    return total, tables


def _attention_inputs(case, seed):
    g = _generator(seed)
    B, Hq, Hkv, n, d, page = case["B"], case["Hq"], case["Hkv"], case["n"], case["d"], case["page"]
    rows, pre, begin = lengths(case)
    P = len(begin) - 1
    s = {}
    total, (s["table"], s["prefix_table"]) = _tables(g, page, [rows, pre])
    u = _randn(g, Hkv, d)
    u = u / u.norm(dim=-1, keepdim=True)
    lean = torch.zeros((total, d), device=DEVICE)                         # the page's KV head leans towards that head's queries
    lean[s["table"].long().reshape(-1)] = u.repeat(B, 1).repeat_interleave(s["table"].shape[1], dim=0)
    if P:
        lean[s["prefix_table"].long().reshape(-1)] = u.repeat(P, 1).repeat_interleave(s["prefix_table"].shape[1], dim=0)
    spiked = torch.rand((total, page, 1), generator=g, device=DEVICE) < 0.1
    s["pool_K"] = (_randn(g, total, page, d) + 2.5 * spiked * lean[:, None, :]).to(_dtype(case))
    s["pool_V"] = _randn(g, total, page, d).to(_dtype(case))
    # queries as a projection leaves them, [B, n, Hq, d] in memory
    s["Q"] = (_randn(g, B, n, Hq, d) + GAMMA * math.sqrt(d) * u.repeat_interleave(Hq // Hkv, dim=0)).to(_dtype(case)).transpose(1, 2)
    s["len"], s["k"] = _ints(rows), _ints(counts(case)) if case["ragged"] else None
    s["prefix_len"], s["group_begin"] = (_ints(pre), _ints(begin)) if P else (None, None)
    s["scale"] = 1.0 / math.sqrt(d)
    if case["kind"] == "weigh":
        s["before"] = torch.rand((B * Hkv, s["table"].shape[1] * page), generator=g, device=DEVICE) ** 6
        s["lse"] = _log_sums(dict(s, case=case))
    return s


def _evict_inputs(case, seed):
    g = _generator(seed)
    rows, page, units = held(case), case["page"], case["B"] * case["Hkv"]
    s = {}
    total, (s["table"],) = _tables(g, page, [rows])
    s["pool_K"], s["pool_V"] = (_randn(g, total, page, case["d"]).to(_dtype(case)) for _ in range(2))
    room = s["table"].shape[1] * page
    r, length = torch.arange(room, device=DEVICE)[None, :], torch.tensor(rows, device=DEVICE)[:, None]
    # few rows have most of the weight; one in sixteen was hardly looked at, in equal parts
    weight = torch.exp(2.0 * _randn(g, units, room))
    weight = torch.where(torch.rand((units, room), generator=g, device=DEVICE) < 1.0 / 16, torch.full_like(weight, 2.0 ** -8), weight)
    s["weight"] = torch.where(r < length, weight, torch.zeros_like(weight))
    # an earlier eviction has left the rows up to `settled` in no order, with gaps between their tokens; those behind it are new
    settled = torch.clamp(torch.full_like(length, min(case["budget"], case["rows"])), max=length - 1)
    order = torch.rand((units, room), generator=g, device=DEVICE).masked_fill(r >= settled, 2.0).argsort(dim=1)
    s["tokens"] = torch.where(r < settled, order * 3 // 2, torch.full_like(order, -1)).to(torch.int32)
    s["len"] = _ints(rows)
    return s


def prepare(case, seed):
    s = _evict_inputs(case, seed) if case["kind"] == "evict" else _attention_inputs(case, seed)
    s["case"] = dict(case)
    if case["kind"] == "chunk":
        s["O"] = torch.zeros_like(s["Q"])                                 # laid out as the queries are
        s["lse"] = torch.zeros(s["Q"].shape[:3], device=DEVICE)
    elif case["kind"] == "weigh":
        s["weight"] = torch.zeros_like(s["before"])
    else:
        s["weight_out"], s["tokens_out"], s["len_out"] = torch.zeros_like(s["weight"]), torch.full_like(s["tokens"], -1), torch.zeros_like(s["len"])
    if own:
        import paper_2410_08584_amd as z
        s["cache"] = z.PagedCache(s["pool_K"], s["pool_V"])
        if case["kind"] == "chunk":
            s["ws"] = z.chunk_paged_workspace(s["cache"], s["table"], s["prefix_table"], B=case["B"], Hq=case["Hq"], Hkv=case["Hkv"], n=case["n"])
        if case["kind"] == "evict":
            s["ws"] = z.paged_evict_workspace(s["cache"], s["table"], case["budget"])
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    if not own:
        return {"chunk": plain_chunk, "weigh": plain_weigh, "evict": plain_evict}[case["kind"]](s)
    import paper_2410_08584_amd as z
    if case["kind"] == "chunk":
        O, lse = z.zipvl_chunk_attn_paged(s["Q"], s["cache"], s["table"], s["len"], s["scale"], k=s["k"], prefix_table=s["prefix_table"], prefix_len=s["prefix_len"],
                                          group_begin=s["group_begin"], O=s["O"], lse=s["lse"], ws=s["ws"])
        return {"O": O, "lse": lse}
    if case["kind"] == "weigh":
        return z.zipvl_paged_weigh(s["Q"], s["cache"], s["table"], s["len"], s["lse"], s["scale"], k=s["k"], before=s["before"], weight=s["weight"])
    z.zipvl_paged_evict(s["cache"], s["table"], s["len"], s["weight"], case["budget"], tokens=s["tokens"], sinks=case["sinks"], recent=case["recent"],
                        length_out=s["len_out"], weight_out=s["weight_out"], tokens_out=s["tokens_out"], ws=s["ws"])
    return {"K": s["pool_K"], "V": s["pool_V"], "len": s["len_out"], "weight": s["weight_out"], "tokens": s["tokens_out"]}


def _rows(pool, table, width):
    """The first `width` rows of every unit of a table, in 32 bits."""
    return pool[table.long()].view(table.shape[0], -1, pool.shape[2])[:, :width].float()


def _seen(s, width):
    """[units, n, width]: own rows that a unit's queries see, causally."""
    case = s["case"]
    n = case["n"]
    cnt = torch.full_like(s["len"], n) if s["k"] is None else s["k"]
    last = s["len"][:, None] - cnt[:, None] + torch.arange(n, device=DEVICE)[None, :]
    return torch.arange(width, device=DEVICE)[None, None, :] <= last[:, :, None], torch.arange(n, device=DEVICE)[None, :] < cnt[:, None]


def _grouped(s):
    """Queries in 32 bits, [units, G, n, d]."""
    case = s["case"]
    return s["Q"].float().reshape(case["B"] * case["Hkv"], case["Hq"] // case["Hkv"], case["n"], case["d"])


def _own_logits(s):
    case = s["case"]
    width = max(lengths(case)[0])
    q = _grouped(s)
    K = _rows(s["pool_K"], s["table"], width)
    logits = torch.matmul(q.flatten(1, 2), K.transpose(1, 2).contiguous()).view(*q.shape[:3], width) * s["scale"]
    seen, there = _seen(s, width)
    return logits.masked_fill(~seen[:, None], -math.inf), there[:, None]


def _log_sums(s):
    """weigh: lse of every query over its own rows, as the attention before it leaves it; zero for tokens that were not brought."""
    case = s["case"]
    logits, there = _own_logits(s)
    top = logits.amax(dim=-1, keepdim=True)
    lse = (top + torch.log(torch.exp(logits - top).sum(dim=-1, keepdim=True)))[..., 0]
    return torch.where(there, lse, torch.zeros_like(lse)).view(case["B"], case["Hq"], case["n"])


def plain_chunk(s):
    case = s["case"]
    B, Hq, Hkv, n, d, P = case["B"], case["Hq"], case["Hkv"], case["n"], case["d"], case["groups"]
    logits, there = _own_logits(s)
    V = _rows(s["pool_V"], s["table"], logits.shape[-1])
    if P:
        b = torch.arange(B, device=DEVICE)
        group = (b[:, None] >= s["group_begin"][None, 1:]).sum(dim=1)                      # every conversation is in a group
        unit = (group[:, None] * Hkv + torch.arange(Hkv, device=DEVICE)[None, :]).reshape(-1)
        width = max(lengths(case)[1])
        Kp, Vp = _rows(s["pool_K"], s["prefix_table"], width)[unit], _rows(s["pool_V"], s["prefix_table"], width)[unit]
        lp = torch.matmul(_grouped(s).flatten(1, 2), Kp.transpose(1, 2).contiguous()).view(B * Hkv, Hq // Hkv, n, width) * s["scale"]
        behind = torch.arange(width, device=DEVICE)[None, :] >= s["prefix_len"][unit][:, None]
        logits = torch.cat([lp.masked_fill(behind[:, None, None], -math.inf), logits], dim=-1)
        V = torch.cat([Vp, V], dim=1)
    top = logits.amax(dim=-1, keepdim=True)
    w = torch.exp(logits - top)
    total = w.sum(dim=-1, keepdim=True)
    o = torch.matmul(w.flatten(1, 2), V).view(B * Hkv, Hq // Hkv, n, d) / total
    lse = (top + torch.log(total))[..., 0]
    o, lse = o.view(B, Hq, n, d).to(s["Q"].dtype), lse.view(B, Hq, n)
    there = there.expand(B * Hkv, Hq // Hkv, n).reshape(B, Hq, n)
    s["O"].copy_(torch.where(there[..., None], o, s["O"]))
    s["lse"].copy_(torch.where(there, lse, s["lse"]))
    return {"O": s["O"], "lse": s["lse"]}


def plain_weigh(s):
    case = s["case"]
    logits, there = _own_logits(s)
    w = torch.exp(logits - s["lse"].view(logits.shape[:3])[..., None])
    w = torch.where(there[..., None], w, torch.zeros_like(w)).sum(dim=(1, 2))
    held_rows = torch.arange(w.shape[1], device=DEVICE)[None, :] < s["len"][:, None]
    s["weight"][:, :w.shape[1]] = torch.where(held_rows, s["before"][:, :w.shape[1]] + w, s["weight"][:, :w.shape[1]])
    return s["weight"]


def plain_evict(s):
    case = s["case"]
    page, units, room = case["page"], s["weight"].shape[0], s["weight"].shape[1]
    r, length = torch.arange(room, device=DEVICE)[None, :], s["len"].long()[:, None]
    held_rows = r < length
    new = (s["tokens"] < 0) & held_rows
    newest = torch.where(held_rows, s["tokens"], torch.full_like(s["tokens"], -1)).amax(dim=1, keepdim=True).clamp(min=-1)
    tokens = torch.where(new, (newest + torch.cumsum(new, dim=1)).to(torch.int32), s["tokens"])
    last = torch.where(held_rows, tokens, torch.full_like(tokens, -1)).amax(dim=1, keepdim=True)
    sure = (tokens < case["sinks"]) | (tokens > last - case["recent"])
    bits = s["weight"].clamp(min=0).view(torch.int32).long()
    key = torch.where(held_rows, bits + (sure.long() << 31), torch.full_like(bits, -1))
    k = length.clamp(max=case["budget"])
    place = torch.sort(key, dim=1, descending=True, stable=True).indices
    kept = torch.zeros((units, room), dtype=torch.bool, device=DEVICE).scatter_(1, place, r.expand(units, room) < k)
    gap, late = (~kept & (r < k)).nonzero(as_tuple=True), (kept & (r >= k)).nonzero(as_tuple=True)      # as many of both in every unit, in the order of rows
    source = torch.arange(room, device=DEVICE).repeat(units, 1)
    source[gap] = late[1]

    def at(unit, row):
        return s["table"].long()[unit, row // page] * page + row % page

    for pool in (s["pool_K"], s["pool_V"]):
        flat = pool.view(-1, case["d"])
        flat[at(*gap)] = flat[at(*late)]
    s["len_out"].copy_(k[:, 0])
    stays = r < k
    s["weight_out"].copy_(torch.where(stays, torch.gather(s["weight"], 1, source), torch.where(held_rows, torch.zeros_like(s["weight"]), s["weight_out"])))
    s["tokens_out"].copy_(torch.where(stays, torch.gather(tokens, 1, source), torch.where(held_rows, torch.full_like(tokens, -1), s["tokens_out"])))
    return {"K": s["pool_K"], "V": s["pool_V"], "len": s["len_out"], "weight": s["weight_out"], "tokens": s["tokens_out"]}


# ---------------------------------------------------------------- the definitions in 64 bits, unit by unit
def exact(case, seed):
    B, Hkv, d, page = case["B"], case["Hkv"], case["d"], case["page"]
    if case["kind"] == "evict":
        return _exact_evict(case, seed) if sum(held(case)) < 3e6 else None
    if work(case)["flops"] > 1.2e12:
        return None
    s, G, n = _attention_inputs(case, seed), case["Hq"] // Hkv, case["n"]
    rows, pre, begin = lengths(case)
    cnt = counts(case)

    def unit(pool, table, length):
        used = table[:-(-length // page)].long()
        return pool[used].reshape(-1, d)[:length].double()

    O = torch.zeros((B, case["Hq"], n, d), dtype=torch.float64, device=DEVICE)
    lse = torch.zeros((B, case["Hq"], n), dtype=torch.float64, device=DEVICE)
    weight = torch.zeros((B * Hkv, s["table"].shape[1] * page), dtype=torch.float64, device=DEVICE)
    for u in range(B * Hkv):
        b, g = divmod(u, Hkv)
        L, c = rows[u], cnt[u]
        keys = unit(s["pool_K"], s["table"][u], L)
        first = 0
        if case["kind"] == "chunk" and case["groups"]:
            p = max(p for p in range(case["groups"]) if begin[p] <= b)
            first = pre[p * Hkv + g]
            keys = torch.cat([unit(s["pool_K"], s["prefix_table"][p * Hkv + g], first), keys])
        hidden = torch.ones((c, first + L), dtype=torch.bool, device=DEVICE).triu(first + L - c + 1)
        if case["kind"] == "weigh":
            weight[u, :L] = s["before"][u, :L].double()
        else:
            values = unit(s["pool_V"], s["table"][u], L)
            if first:
                values = torch.cat([unit(s["pool_V"], s["prefix_table"][p * Hkv + g], first), values])
        for h in range(g * G, (g + 1) * G):
            z = (s["Q"][b, h, :c].double() @ keys.T / math.sqrt(d)).masked_fill_(hidden, -math.inf)
            if case["kind"] == "weigh":
                weight[u, :L] += z.sub_(s["lse"][b, h, :c].double()[:, None]).exp_().sum(dim=0)
            else:
                lse[b, h, :c] = torch.logsumexp(z, dim=1)
                O[b, h, :c] = torch.softmax(z, dim=1) @ values
    return weight if case["kind"] == "weigh" else {"O": O.transpose(1, 2).contiguous().transpose(1, 2), "lse": lse}


def _exact_evict(case, seed):
    s, page, units = _evict_inputs(case, seed), case["page"], case["B"] * case["Hkv"]
    table = s["table"].cpu().long()
    weight, tokens = s["weight"].cpu().numpy(), s["tokens"].cpu().numpy()
    weight_out, tokens_out = weight.astype("f8") * 0.0, tokens * 0 - 1
    to, come = [], []
    for u, length in enumerate(held(case)):
        kept_n = min(length, case["budget"])
        token = [int(t) for t in tokens[u, :length]]
        following = max(max(token), -1) + 1
        for r in range(length):
            if token[r] < 0:
                token[r], following = following, following + 1
        oldest = max(token) - case["recent"]
        order = sorted(range(length), key=lambda r: (not (token[r] < case["sinks"] or token[r] > oldest), -float(weight[u, r]), r))
        stay = set(order[:kept_n])
        holder = list(range(kept_n))
        for gap, row in zip((r for r in range(kept_n) if r not in stay), (r for r in range(kept_n, length) if r in stay)):
            holder[gap] = row
            to.append(int(table[u, gap // page]) * page + gap % page)
            come.append(int(table[u, row // page]) * page + row % page)
        weight_out[u, :kept_n] = weight[u, holder]
        tokens_out[u, :kept_n] = [token[r] for r in holder]
    K, V = s["pool_K"].double(), s["pool_V"].double()
    for pool in (K, V):
        flat = pool.view(-1, case["d"])
        flat[torch.tensor(to, dtype=torch.long, device=DEVICE)] = flat[torch.tensor(come, dtype=torch.long, device=DEVICE)]
    return {"K": K, "V": V, "len": _ints([min(x, case["budget"]) for x in held(case)]), "weight": torch.from_numpy(weight_out), "tokens": torch.from_numpy(tokens_out)}
