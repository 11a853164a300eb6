"""Attention of several tokens to pages, the weights that cached rows get and eviction by them, against plain forms in 64 bits.

Tolerances.  u = 2^-24 is the rounding of fp32, h(t) = finfo(t).eps / 2 that of an output or of a number in type t.
  attention  a logit is a sum of d products: off by (d + 1) u scale sum|q k|, and by u of itself twice more (the scale, the exponent); a weight carries that as a
             factor, with 4 u of the exponential, once in the numerator and once in the denominator; sums over L rows are off by L u at most.  bf16 weights of units with
             more than 32 queries are rounded, h(bf16) each, above and below.  Relative to A = sum of weight |v|:
             T = 2 ((d + 4) u max(scale sum|q k|) + (L + 64) u + [bf16, more than 32 queries] h(bf16)).  Output: T A + h |result|.
  lse        (d + 4) u max(scale sum|q k|) + (L + 64) u, and 4 u of itself and of the largest logit (offset and logarithm).
  weights    exp(logit - lse): off by (d + 6) u (max(scale sum|q k|) + |lse|) + 4 u of itself; sums of N of them, and what was there before, (N + 8) u.
  eviction   whole numbers and copies: equal.
"""
import ctypes as C
import math

import pytest
import torch

import paper_2410_08584_amd as z

DEV = "cuda:0"
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
NONE = -2 ** 31


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def say(msg):
    print(msg, flush=True)


# ---------------------------------------------------------------- inputs and plain forms, 64 bits, on the CPU
class Setting:
    """Queries, pages and tables; `lens`: own rows of a unit, its new ones among them; `pre`: rows of a prefix, by KV head of each group."""

    def __init__(self, B, Hq, Hkv, n, d, dtype, page, lens, k=None, groups=(), pre=(), order="head", seed=0, gain=1.0, spare=1):
        g = torch.Generator().manual_seed(seed)
        self.B, self.Hq, self.Hkv, self.n, self.d, self.page, self.G = B, Hq, Hkv, n, d, page, Hq // Hkv
        units = B * Hkv
        self.lens = [lens[u % len(lens)] for u in range(units)]
        self.k = None if k is None else [k[u % len(k)] for u in range(units)]
        self.begin = list(groups)
        P = max(0, len(self.begin) - 1)
        self.pre = [pre[u % len(pre)] for u in range(P * Hkv)]
        width, pre_width = -(-max(self.lens + [1]) // page) + spare, -(-max(self.pre + [1]) // page) + spare
        pages = units * width + P * Hkv * pre_width + 2
        order_of = torch.randperm(pages, generator=g).to(torch.int32)
        self.table = order_of[:units * width].view(units, width).clone()
        self.prefix_table = order_of[units * width:units * width + P * Hkv * pre_width].view(P * Hkv, pre_width).clone() if P else None
        self.K = torch.randn((pages, page, d), generator=g).to(DT[dtype])
        self.V = torch.randn((pages, page, d), generator=g).to(DT[dtype])
        Q = (gain * torch.randn((B, Hq, n, d), generator=g)).to(DT[dtype])
        if order == "token":                                  # rows of a wider projection
            wide = torch.randn((B, n, Hq + 3, d), generator=g).to(DT[dtype])
            wide[:, :, 1:1 + Hq] = Q.transpose(1, 2)
            self.Q = wide.to(DEV)[:, :, 1:1 + Hq].transpose(1, 2) if torch.cuda.is_available() else wide[:, :, 1:1 + Hq].transpose(1, 2)
        else:
            self.Q = Q.to(DEV) if torch.cuda.is_available() else Q
        self.scale = 1.0 / math.sqrt(d)
        self.dtype = DT[dtype]

    def count(self, u):
        return self.n if self.k is None else min(max(self.k[u], 0), self.n)

    def spoil(self):
        """Everything that no query may read: NaN behind lengths, in unused pages and in queries that are not there."""
        used = torch.zeros(self.K.shape[:2], dtype=torch.bool)
        for tab, lens in ((self.table, self.lens), (self.prefix_table, self.pre)):
            for u, L in enumerate(lens):
                for r in range(min(max(L, 0), tab.shape[1] * self.page)):
                    e = int(tab[u, r // self.page])
                    if 0 <= e < self.K.shape[0]:
                        used[e, r % self.page] = True
        self.K[~used] = float("nan")
        self.V[~used] = float("nan")
        Q = self.Q
        for u in range(self.B * self.Hkv):
            b, g = divmod(u, self.Hkv)
            Q[b, g * self.G:(g + 1) * self.G, self.count(u):] = float("nan")

    def cache(self):
        return z.PagedCache(self.K.to(DEV), self.V.to(DEV))

    def ints(self, v):
        return None if v is None else torch.tensor(v, dtype=torch.int32, device=DEV)

    def args(self):
        P = len(self.begin) > 1
        return dict(k=self.ints(self.k), prefix_table=self.prefix_table.to(DEV) if P else None, prefix_len=self.ints(self.pre) if P else None,
                    group_begin=self.ints(self.begin) if P else None)

    def rows(self, pool, tab, u, L):
        """(rows, which of them there are) of a unit, 64 bits."""
        L = min(max(L, 0), tab.shape[1] * self.page)
        e = tab[u].long().repeat_interleave(self.page)[:L]
        there = (e >= 0) & (e < pool.shape[0])
        x = pool[e.clamp(0, pool.shape[0] - 1), torch.arange(L) % self.page].double()
        return torch.where(there[:, None], x, torch.zeros_like(x)), there

    def group(self, b):
        B = self.B
        for p in range(len(self.begin) - 1):
            lo = min(max(self.begin[p], 0), B)
            if lo <= b < min(max(self.begin[p + 1], lo), B):
                return p
        return None

    def plain(self, u):
        """For unit u: (o, lse, bound of o without the output's rounding, bound of lse, weights of own rows [G, c, L])."""
        b, g = divmod(u, self.Hkv)
        c, L = self.count(u), min(max(self.lens[u], 0), self.table.shape[1] * self.page)
        K, there = self.rows(self.K, self.table, u, L)
        V, _ = self.rows(self.V, self.table, u, L)
        own = torch.arange(L)[None, :] <= (L - c + torch.arange(c))[:, None]
        seen = own & there[None, :]
        first = 0
        p = self.group(b)
        if p is not None:
            Kp, therep = self.rows(self.K, self.prefix_table, p * self.Hkv + g, self.pre[p * self.Hkv + g])
            Vp, _ = self.rows(self.V, self.prefix_table, p * self.Hkv + g, self.pre[p * self.Hkv + g])
            first = Kp.shape[0]
            K, V = torch.cat([Kp, K]), torch.cat([Vp, V])
            seen = torch.cat([therep[None, :].expand(c, first), seen], dim=1)
        q = self.Q[b, g * self.G:(g + 1) * self.G, :c].cpu().double()
        logits = (q @ K.T * self.scale).masked_fill(~seen[None], -math.inf)
        lse = torch.logsumexp(logits, dim=-1) if K.shape[0] else torch.full(q.shape[:2], -math.inf, dtype=torch.float64)
        w = torch.exp(logits - torch.where(lse > -math.inf, lse, torch.zeros_like(lse))[..., None])
        big = float((q.abs() @ K.abs().T * seen[None]).max()) * self.scale if K.shape[0] and c else 0.0
        off = (self.d + 4) * U * big + (K.shape[0] + 64) * U
        groups = len(self.begin) - 1
        packed = groups > 0 and 2 * groups <= self.B and self.n * self.G * self.B // groups > 32       # a group's rows of queries in tiles together
        rounded = half_step(torch.bfloat16) if self.dtype == torch.bfloat16 and (self.n * self.G > 32 or packed) else 0.0
        return w @ V, lse, 2 * (off + rounded) * (w @ V.abs()), off + 4 * U * (lse.abs().nan_to_num(0, 0, 0) + big), w[..., first:], big


def chunk(s, cache=None, want_lse=True, **more):
    return z.zipvl_chunk_attn_paged(s.Q, cache or s.cache(), s.table.to(DEV), s.ints(s.lens), s.scale, want_lse=want_lse, **{**s.args(), **more})


def assert_chunk(s, O, lse, fill=0.0):
    O, lse = O.cpu().double(), lse.cpu().double()
    for u in range(s.B * s.Hkv):
        b, g = divmod(u, s.Hkv)
        heads, c = slice(g * s.G, (g + 1) * s.G), s.count(u)
        o, ref, bound, lse_bound, _, _ = s.plain(u)
        over = ((O[b, heads, :c] - o).abs() - bound - half_step(s.dtype) * o.abs())
        assert not c or over.max().item() <= 0, f"unit {u}: output {over.max().item():.3e} over"
        got = lse[b, heads, :c]
        assert torch.equal(got == -math.inf, ref == -math.inf), f"unit {u}: queries that see nothing"
        fine = ref > -math.inf
        assert not fine.any() or ((got - ref).abs()[fine] - lse_bound[fine]).max().item() <= 0, f"unit {u}: lse {((got - ref).abs()[fine] - lse_bound[fine]).max().item():.3e} over"
        assert (O[b, heads, :c][~fine] == 0).all()
        assert (O[b, heads, c:] == fill).all() and (lse[b, heads, c:] == fill).all(), f"unit {u}: queries that are not there"


CHUNK = [  # B, Hq, Hkv, n, d, dtype, page, lens, k, groups, pre, order
    (1, 4, 4, 1, 64, "f32", 16, [1], None, (), (), "head"),
    (2, 8, 2, 1, 128, "bf16", 16, [0, 1, 33, 700], None, (), (), "head"),
    (3, 28, 4, 2, 128, "bf16", 64, [2, 65, 1, 0, 900], [2, 1, 0], (0, 2, 3), (100, 0, 7, 33), "token"),
    (2, 4, 4, 5, 64, "f32", 16, [45, 5, 3], None, (0, 2), (576, 500, 1), "head"),
    (2, 6, 1, 5, 128, "f32", 32, [45, 2000], [5, 4], (), (), "token"),
    (3, 32, 1, 1, 64, "bf16", 128, [129, 1], None, (0, 1, 1, 2), (40, 41, 64), "head"),
    (1, 40, 1, 1, 128, "bf16", 16, [100], None, (), (), "head"),
    (2, 33, 3, 7, 64, "bf16", 256, [7, 263, 1000], [7, 3, 0], (0, 0, 1), (260, 9), "token"),
    (2, 14, 2, 24, 128, "bf16", 64, [24, 84, 10, 400], [24, 17, 9], (0, 2), (333, 700), "token"),
    (1, 8, 8, 129, 128, "bf16", 16, [129, 130, 200, 1300], None, (), (), "token"),
    (2, 2, 2, 300, 64, "bf16", 32, [300, 299, 1, 511], [300, 255, 256, 1], (), (), "head"),
    (1, 28, 4, 64, 128, "bf16", 128, [64, 640, 2000, 63], None, (0, 1), (100, 3, 64, 128), "head"),
    (2, 8, 8, 77, 64, "f32", 16, [77, 100, 500, 40], [77, 60, 1], (), (), "token"),
    (1, 7, 1, 70, 128, "f32", 64, [700], None, (0, 1), (97,), "token"),
    (2, 5, 1, 13, 128, "f32", 256, [13, 270], None, (1, 2), (31,), "head"),
    (5, 16, 8, 33, 64, "bf16", 16, [33, 40, 1030, 0, 12, 77, 64], [33, 32, 0, 5], (0, 1, 4), (1025, 64, 17), "token"),
    (6, 28, 4, 2, 128, "bf16", 64, [2, 65, 1, 0, 900], [2, 1, 0], (0, 4, 6), (700, 0, 65, 1300, 100), "token"),
    (9, 4, 1, 10, 64, "f32", 16, [10, 50, 100], [10, 3, 0, 7], (0, 2, 2, 7), (129, 64, 0), "head"),
    (16, 7, 1, 18, 128, "bf16", 16, [18, 300, 0, 40], [18, 0, 0, 5, 17], (0, 16), (2000,), "token"),
    (4, 2, 2, 256, 64, "bf16", 32, [256, 700, 300], [256, 255, 1], (0, 4), (333, 1), "head"),
    (8, 40, 2, 1, 128, "f32", 16, [1, 30, 0], None, (2, 6), (500, 77), "token"),
    (40, 1, 1, 1, 64, "bf16", 16, [1, 2, 90], [1, 1, 0], (0, 40), (640,), "head"),
]


def case_id(c):
    return f"B{c[0]}Hq{c[1]}Hkv{c[2]}n{c[3]}d{c[4]}{c[5]}page{c[6]}P{max(0, len(c[9]) - 1)}{c[11]}"


@pytest.mark.gpu
@pytest.mark.parametrize("case", CHUNK, ids=case_id)
def test_chunk_attn_paged(case):
    say(f"chunk {case}")
    s = Setting(*case[:11], order=case[11], seed=5)
    s.spoil()
    O = torch.full((s.B, s.n, s.Hq + 2, s.d), 7.0, dtype=s.dtype, device=DEV)
    view = O[:, :, 1:1 + s.Hq].transpose(1, 2)
    lse = torch.full((s.B, s.Hq, s.n), 7.0, device=DEV)
    cache = s.cache()
    chunk(s, cache, O=view, lse=lse)
    assert_chunk(s, view, lse, fill=7.0)
    assert (O[:, :, 0] == 7).all() and (O[:, :, 1 + s.Hq:] == 7).all()
    # contiguous, without lse, from a workspace that holds anything: the same bits
    ws = z.chunk_paged_workspace(cache, s.table.to(DEV), s.args()["prefix_table"], B=s.B, Hq=s.Hq, Hkv=s.Hkv, n=s.n).fill_(0x7F)
    again, none = chunk(s, cache, want_lse=False, ws=ws)
    assert none is None
    there = torch.stack([torch.arange(s.n) < s.count(u) for u in range(s.B * s.Hkv)]).view(s.B, s.Hkv, s.n).repeat_interleave(s.G, dim=1).to(DEV)
    assert torch.equal(again[there], view[there])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("Hq,Hkv,n", [(2, 1, 3), (28, 4, 1), (4, 2, 40)])
def test_chunk_attn_paged_long(dtype, d, Hq, Hkv, n):
    """Keys cut into many pieces, tables wider than what a wave sees at once, lengths far apart."""
    s = Setting(3, Hq, Hkv, n, d, dtype, 16, [9000, n, 3000, 70, 5], None, (0, 1, 3), (5000, 31, 2049), order="token", seed=6)
    s.spoil()
    assert_chunk(s, *chunk(s))


@pytest.mark.gpu
@pytest.mark.parametrize("n,lens", [(1, [0, 1, 40]), (5, [5, 12])])
def test_chunk_attn_paged_of_thousands_of_units(n, lens):
    s = Setting(2100, 2, 1, n, 64, "bf16", 16, lens, None, (0, 1000, 2100), (33, 7), seed=7)
    assert_chunk(s, *chunk(s))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,n,B,tile,wgs,groups", [("bf16", 64, 40, 540, 64, 512, ()), ("bf16", 128, 40, 400, 64, 512, ()), ("bf16", 64, 40, 300, 64, 512, ()), ("f32", 64, 36, 520, 32, 512, ()),
                                                         ("bf16", 64, 2, 540, 32, 512, ()), ("f32", 128, 3, 300, 32, 256, ()), ("bf16", 64, 4, 400, 64, 512, (0, 40, 400)),
                                                         ("f32", 64, 4, 500, 32, 512, (0, 200, 500))])
def test_chunk_attn_paged_of_many_short_units_and_few_long_ones(dtype, d, n, B, tile, wgs, groups):
    """Hundreds of tiles of rows that have a workgroup each leave too few for the pieces of the long ones: pieces are made larger, in one case after another."""
    say(f"short and long {dtype} {d} {n} {B} {groups}")
    s = Setting(B, 1, 1, n, d, dtype, 16, [n, n + 5, n + 14], None, groups, (70, 33), seed=54, spare=0)
    width = 400 * tile // 16
    s.table = torch.randint(0, s.K.shape[0], (B, width), generator=torch.Generator().manual_seed(55)).to(torch.int32)
    long = [3, B // 2, B // 2 + 1, B - 1]
    for u in long:
        s.lens[u] = 400 * tile - u % 7
    # the pieces, as the device counts them: a tile of rows is cut into its tiles of keys / q, at least one
    loads = [-(-L // tile) for L in s.lens]
    items = B
    if groups:
        P = len(groups) - 1
        for p in range(P):
            packed = n * (groups[p + 1] - groups[p])
            loads += [-(-s.pre[p] // tile)] * -(-packed // 128)
        items += B * n // 128 + P + 1
    limit = max(wgs + 64, (items + 21) // 8 * 8) - 14
    q = max(4, -(-sum(loads) // wgs))
    assert items <= 2048 and sum(max(1, x // q) for x in loads) > limit
    assert_chunk(s, *chunk(s))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 4, 50])
def test_chunk_attn_paged_skips_rows_without_a_page_and_clamps_lengths(dtype, n):
    s = Setting(2, 4, 2, n, 128, dtype, 16, [200, 77, 150, 64], None, (0, 1), (100, 60), seed=8)
    pages = s.K.shape[0]
    s.table[0, 2] = -1
    s.table[0, 5:8] = pages
    s.table[1, :] = NONE
    s.table[2, 3] = 2 ** 31 - 1
    s.table[3, 0] = -7
    s.prefix_table[0, 1:3] = pages + 5
    s.lens[2] = 10 ** 9
    s.pre[1] = 2 ** 31 - 1
    s.spoil()
    assert_chunk(s, *chunk(s))
    s.lens[0], s.pre[0] = -5, NONE
    s.k = [n + 7, -3, 2 ** 31 - 1, n]
    assert_chunk(s, *chunk(s))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n", [("bf16", 2), ("bf16", 70), ("f32", 2), ("f32", 70)])
@pytest.mark.parametrize("gain", [40.0, 1e-3])
def test_chunk_attn_paged_of_large_and_small_logits(dtype, n, gain):
    s = Setting(1, 4, 2, n, 128, dtype, 32, [600, 333], None, seed=9, gain=gain)
    assert_chunk(s, *chunk(s))


@pytest.mark.gpu
@pytest.mark.parametrize("d,n", [(64, 3), (64, 70), (128, 70)])
@pytest.mark.parametrize("of_queries,of_values", [(2.0 ** 101, 1.0), (2.0 ** -101, 1.0), (1.0, 2.0 ** 115), (1.0, 2.0 ** -100)])
def test_chunk_attn_paged_of_huge_and_small_numbers(d, n, of_queries, of_values):
    """fp32 whose products fit, with numbers that planes of bf16 do not hold in full range: the output of their like of ordinary size, times what values were."""
    say(f"huge {d} {n} {of_queries} {of_values}")
    s = Setting(2, 4, 2, n, d, "f32", 16, [200, 100, 80, 75], None, seed=24)
    s.Q.mul_(of_queries)
    s.K.mul_(1 / of_queries)
    s.V.mul_(of_values)
    assert_chunk(s, *chunk(s))


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,groups", [(3, ()), (70, ()), (70, (0, 2))])
@pytest.mark.parametrize("of_values", [2.0 ** -110, 2.0 ** -122])
def test_chunk_attn_paged_of_values_near_the_smallest(d, n, groups, of_values):
    """fp32 values whose third plane of bf16 would end below bf16's smallest number: the outputs have all their bits."""
    say(f"small values {d} {n} {groups} {of_values}")
    s = Setting(2, 4, 2, n, d, "f32", 16, [200, 100, 80, 75], None, groups, (300, 70), seed=52)
    s.V.mul_(of_values)
    assert_chunk(s, *chunk(s))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("gain", [40.0, 1.0])
def test_chunk_attn_paged_of_groups_with_large_logits_and_missing_pages(dtype, d, gain):
    """A group's queries together: sums that leave the middle of fp32's range, rows of the prefix without a page, counts and lengths beyond what there is."""
    say(f"groups {dtype} {d} {gain}")
    s = Setting(7, 14, 2, 12, d, dtype, 64, [300, 12, 5, 0], [12, 1, 0, 7, 12], (0, 4, 7), (900, 640, 1500, 63), seed=23, gain=gain)
    if gain == 1.0:
        pages = s.K.shape[0]
        s.prefix_table[0, 1:3] = pages
        s.prefix_table[1, :] = -1
        s.prefix_table[2, 20] = NONE
        s.pre[2] = 2 ** 31 - 1
        s.k[3], s.k[8] = 2 ** 31 - 1, -4
        s.lens[2] = 10 ** 9
    s.spoil()
    assert_chunk(s, *chunk(s))


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hot,late,values", [(43.75, 41.5, 8.0), (43.75, 41.5, 1000.0), (17.5, 0.0, 2.0 ** 80), (60.0, 55.0, 1.0)])
@pytest.mark.parametrize("where", ["own", "prefix", "packed"])
def test_chunk_attn_paged_of_keys_far_above_the_first(where, hot, late, values, d):
    """Tiles of 64 keys whose first has logits near 0 and a later one a logit of 2 `hot`, then new tokens' keys of 2 `late`: whatever the sums are by the first maximum, the outputs
    are those of the formula.  In powers of two 17.5, 41.5 and 43.75 are 50, 120 and 126."""
    say(f"hot {where} {hot} {late} {values} {d}")
    n = 70
    if where == "own":
        s = Setting(1, 1, 1, n, d, "bf16", 16, [384], seed=51, spare=0)
    else:
        B = 1 if where == "prefix" else 2
        s = Setting(B, 1, 1, n, d, "bf16", 16, [96], None, (0, B), (256,), seed=51, spare=0)
    tab, at = (s.table, 150) if where == "own" else (s.prefix_table, 150)
    s.V.mul_(values)
    s.Q[..., 0] = 2.0 * math.sqrt(d)                          # times the scale: 2
    s.K[..., 0] = 0.0
    s.K[int(tab[0, at // 16]), at % 16, 0] = hot
    for u, L in enumerate(s.lens):
        for r in range(L - n, L):
            s.K[int(s.table[u, r // 16]), r % 16, 0] = late
    assert_chunk(s, *chunk(s))


@pytest.mark.gpu
def test_chunk_attn_paged_of_one_token_is_decode():
    s = Setting(4, 28, 4, 1, 128, "bf16", 64, [500, 1, 70, 1300], None, (0, 3, 4), (300, 41), seed=10)
    cache = s.cache()
    O, _ = chunk(s, cache)
    a = s.args()
    o = z.zipvl_decode_attn_paged(s.Q.reshape(-1, s.d), cache, s.table.to(DEV), s.ints(s.lens), s.scale, B=s.B, Hq=s.Hq, Hkv=s.Hkv,
                                  prefix_table=a["prefix_table"], prefix_len=a["prefix_len"], group_begin=a["group_begin"])
    assert torch.allclose(O.reshape(-1, s.d).float(), o.float(), rtol=2 * half_step(torch.bfloat16), atol=1e-6)


@pytest.mark.gpu
def test_over_more_than_4_gib():
    """Pages behind 4 GiB."""
    page, d, n = 256, 128, 3
    pages = (5 << 30) // (page * d * 2)
    K = torch.empty((pages, page, d), dtype=torch.bfloat16, device=DEV)
    V = torch.empty((pages, page, d), dtype=torch.bfloat16, device=DEV)
    s = Setting(1, 4, 2, n, d, "bf16", page, [700, 300], None, seed=11)
    at = torch.tensor([pages - 1, 3, pages - 2, 7, pages // 2 + 9, pages - 40, 1, 2, 5, 9, 11][:s.table.numel()], dtype=torch.int32)
    for i, e in enumerate(at.tolist()):
        K[e] = s.K[int(s.table.view(-1)[i])].to(DEV)
        V[e] = s.V[int(s.table.view(-1)[i])].to(DEV)
    table = at.view(s.table.shape).to(DEV)
    cache = z.PagedCache(K, V)
    O, lse = z.zipvl_chunk_attn_paged(s.Q, cache, table, s.ints(s.lens), s.scale, want_lse=True)
    assert_chunk(s, O, lse)
    w = z.zipvl_paged_weigh(s.Q, cache, table, s.ints(s.lens), lse, s.scale)
    assert_weights(s, w, lse, None)
    length = s.ints(s.lens)
    z.zipvl_paged_evict(cache, table, length, w.clone(), 290)
    assert length.tolist() == [290, 290]
    _, source = evicted(s, w.cpu(), None, 290, 0, 0)
    for u in range(2):
        got = cache.K[table[u].long()].view(-1, d)[:290].cpu()
        want, _ = s.rows(s.K, s.table, u, s.lens[u])
        assert torch.equal(got.double(), want[source[u]])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [3, 70])
def test_queries_and_outputs_far_apart(dtype, n):
    """Heads and batch elements of Q and O more than 2^31 elements from each other."""
    s = Setting(2, 2, 1, n, 64, dtype, 16, [200, 90], None, seed=26)
    strides = (2 ** 31 + 2 ** 20, 2 ** 31 - 2 ** 19 + 64, 64, 1)
    size = sum(x * (k - 1) for x, k in zip(strides, (2, 2, n, 64))) + 1
    Q, O = (torch.empty(size, dtype=s.dtype, device=DEV).as_strided((2, 2, n, 64), strides) for _ in range(2))
    Q.copy_(s.Q)
    cache, table, length = s.cache(), s.table.to(DEV), s.ints(s.lens)
    got, lse = z.zipvl_chunk_attn_paged(Q, cache, table, length, s.scale, O=O, want_lse=True)
    assert got is O
    assert_chunk(s, O, lse)
    assert_weights(s, z.zipvl_paged_weigh(Q, cache, table, length, lse, s.scale), lse, None)


# ---------------------------------------------------------------- weights
def assert_weights(s, weight, lse, before, fill=0.0):
    weight, lse = weight.cpu().double(), lse.cpu().double()
    for u in range(s.B * s.Hkv):
        b, g = divmod(u, s.Hkv)
        heads, c = slice(g * s.G, (g + 1) * s.G), s.count(u)
        L = min(max(s.lens[u], 0), s.table.shape[1] * s.page)
        K, there = s.rows(s.K, s.table, u, L)
        q = s.Q[b, heads, :c].cpu().double()
        seen = (torch.arange(L)[None, :] <= (L - c + torch.arange(c))[:, None]) & there[None, :]
        logits = (q @ K.T * s.scale).masked_fill(~seen[None], -math.inf)
        row = lse[b, heads, :c, None]
        w = torch.where(row > -math.inf, torch.exp(logits - torch.where(row > -math.inf, row, torch.zeros_like(row))), torch.zeros_like(logits)).sum(dim=(0, 1))
        big = float((q.abs() @ K.abs().T * seen[None]).max()) * s.scale if L and c else 0.0
        far = float(row[row > -math.inf].abs().max()) if (row > -math.inf).any() else 0.0
        old = torch.zeros(L, dtype=torch.float64) if before is None else before[u, :L].cpu().double()
        tol = w * ((s.d + 6) * U * (big + far) + 4 * U + (c * s.G + 8) * U) + (old + w) * 8 * U
        over = (weight[u, :L] - old - w).abs() - tol
        assert not L or over.max().item() <= 0, f"unit {u}: weight {over.max().item():.3e} over"
        assert (weight[u, L:] == fill).all(), f"unit {u}: rows that are not there"


@pytest.mark.gpu
@pytest.mark.parametrize("case", CHUNK, ids=case_id)
def test_paged_weigh(case):
    say(f"weigh {case}")
    s = Setting(*case[:11], order=case[11], seed=15)
    cache = s.cache()
    _, lse = chunk(s, cache)
    s.spoil()
    cache = s.cache()
    cache.V.fill_(float("nan"))                               # not looked at
    g = torch.Generator().manual_seed(1)
    before = torch.rand((s.B * s.Hkv, s.table.shape[1] * s.page), generator=g).to(DEV)
    weight = torch.full_like(before, 7.0)
    got = z.zipvl_paged_weigh(s.Q, cache, s.table.to(DEV), s.ints(s.lens), lse, s.scale, k=s.ints(s.k), before=before, weight=weight)
    assert got is weight
    assert_weights(s, weight, lse, before, fill=7.0)
    # on top of itself, the same bits; and from nothing
    place = before.clone()
    z.zipvl_paged_weigh(s.Q, cache, s.table.to(DEV), s.ints(s.lens), lse, s.scale, k=s.ints(s.k), before=place, weight=place)
    live = torch.arange(place.shape[1])[None, :] < torch.tensor(s.lens).clamp(min=0)[:, None]
    assert torch.equal(place.cpu()[live], weight.cpu()[live]) and torch.equal(place.cpu()[~live], before.cpu()[~live])
    fresh = z.zipvl_paged_weigh(s.Q, cache, s.table.to(DEV), s.ints(s.lens), lse, s.scale, k=s.ints(s.k))
    assert_weights(s, fresh, lse, None)


@pytest.mark.gpu
def test_paged_weigh_sums_to_the_number_of_queries():
    """What the rows of a unit get from a query adds up to 1, to what the prefix has left of it, and to 0 where it saw nothing."""
    s = Setting(2, 14, 2, 50, 64, "f32", 32, [800, 50, 20, 333], None, seed=16)
    cache = s.cache()
    _, lse = chunk(s, cache)
    w = z.zipvl_paged_weigh(s.Q, cache, s.table.to(DEV), s.ints(s.lens), lse, s.scale)
    for u, total in enumerate(w.double().sum(dim=1).tolist()):
        want = s.G * min(s.n, s.lens[u])
        assert abs(total - want) <= want * ((s.d + 6) * U * 60 + 900 * U), (u, total, want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_paged_weigh_of_the_last_queries(dtype):
    s = Setting(2, 8, 2, 40, 128, dtype, 64, [300, 40, 64, 1000], None, order="token", seed=17)
    cache = s.cache()
    _, lse = chunk(s, cache)
    m = 7
    w = z.zipvl_paged_weigh(s.Q[:, :, -m:], cache, s.table.to(DEV), s.ints(s.lens), lse[:, :, -m:], s.scale)
    s.Q, s.n = s.Q[:, :, -m:], m
    assert_weights(s, w, lse[:, :, -m:], None)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("spare", [100, 300])
def test_paged_weigh_where_tables_are_wide(dtype, d, spare):
    """Many rows may be there, so that a wave has more of them: few are."""
    say(f"weigh {dtype} {d} {spare} spare pages")
    s = Setting(2, 6, 2, 70, d, dtype, 256, [700, 90, 64, 1], [70, 33, 64, 65], order="token", seed=19, spare=spare)
    s.table[1, 0] = -1
    cache = s.cache()
    _, lse = chunk(s, cache)
    weight = torch.full((4, s.table.shape[1] * s.page), 7.0, device=DEV)
    z.zipvl_paged_weigh(s.Q, cache, s.table.to(DEV), s.ints(s.lens), lse, s.scale, k=s.ints(s.k), weight=weight)
    assert_weights(s, weight, lse, None, fill=7.0)


@pytest.mark.gpu
@pytest.mark.parametrize("B,Hkv,n,dtype", [(3, 5, 3500, "f32"), (1, 1, 26000, "f32"), (9, 1, 11500, "bf16"), (2, 3, 8300, "bf16")])
def test_paged_weigh_of_many_queries(B, Hkv, n, dtype):
    """More queries than the caches hold: units are dealt out another way.  Rows of the last tokens and the first, against the plain form."""
    say(f"weigh {B} {Hkv} {n} {dtype}")
    s = Setting(B, 2 * Hkv, Hkv, n, 64 if B > 2 else 128, dtype, 64, [90, 300, 33, 1], [n, n - 5, 40, n], seed=21)
    _, lse = chunk(s)
    w = z.zipvl_paged_weigh(s.Q, s.cache(), s.table.to(DEV), s.ints(s.lens), lse, s.scale, k=s.ints(s.k))
    assert_weights(s, w, lse, None)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,n", [("bf16", 128, 64), ("bf16", 128, 127), ("bf16", 64, 128), ("bf16", 64, 180), ("f32", 128, 64), ("f32", 128, 95), ("f32", 64, 96), ("f32", 64, 90)])
def test_paged_weigh_of_tiles_of_one_head(dtype, d, n):
    """Room for many rows, and tokens that nearly fill their last tile: waves share tiles of one head."""
    say(f"weigh one head {dtype} {d} {n}")
    s = Setting(2, 6, 2, n, d, dtype, 256, [700, 90, n, 300], [n, 33, n - 1, 1], order="token", seed=56, spare=64)
    tile = 64 if dtype == "bf16" else 32
    assert s.table.numel() * s.page // 32 >= 2048 and -(-n // tile) * tile <= n + n // 8
    s.table[0, 1] = -1
    _, lse = chunk(s)
    s.spoil()
    weight = torch.full((4, s.table.shape[1] * s.page), 7.0, device=DEV)
    z.zipvl_paged_weigh(s.Q, s.cache(), s.table.to(DEV), s.ints(s.lens), lse, s.scale, k=s.ints(s.k), weight=weight)
    assert_weights(s, weight, lse, None, fill=7.0)


@pytest.mark.gpu
@pytest.mark.parametrize("B,G,n,d,dtype", [(13, 2, 7680, 64, "bf16"), (7, 4, 1760, 128, "f32")])
def test_paged_weigh_of_many_queries_in_tiles_of_one_head(B, G, n, d, dtype):
    """As before, with more queries than the caches hold, so that units are dealt out another way: eight, four, two and one at a time."""
    say(f"weigh many queries, one head {B} {G} {n} {d} {dtype}")
    s = Setting(B, G, 1, n, d, dtype, 64, [90, 300, 33, 1], [n, n - 5, 40, n], seed=57, spare=148)
    tile = 64 if dtype == "bf16" else 32
    assert s.table.numel() * s.page // 32 >= 2048 and -(-n // tile) * tile <= n + n // 8 and s.Q.numel() * s.Q.element_size() >= 24 << 20
    _, lse = chunk(s)
    w = z.zipvl_paged_weigh(s.Q, s.cache(), s.table.to(DEV), s.ints(s.lens), lse, s.scale, k=s.ints(s.k))
    assert_weights(s, w, lse, None)


@pytest.mark.gpu
@pytest.mark.parametrize("d,n", [(64, 64), (128, 96)])
@pytest.mark.parametrize("of_queries", [2.0 ** 101, 2.0 ** -101])
def test_paged_weigh_of_huge_numbers_in_tiles_of_one_head(d, n, of_queries):
    s = Setting(1, 4, 2, n, d, "f32", 256, [200, 100], None, seed=58, spare=128)
    assert s.table.numel() * s.page // 32 >= 2048
    _, lse = chunk(s)
    s.Q.mul_(of_queries)
    s.K.mul_(1 / of_queries)
    w = z.zipvl_paged_weigh(s.Q, s.cache(), s.table.to(DEV), s.ints(s.lens), lse, s.scale)
    assert_weights(s, w, lse, None)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [3, 70])
@pytest.mark.parametrize("of_queries", [2.0 ** 101, 2.0 ** -101])
def test_paged_weigh_of_huge_numbers(n, of_queries):
    """fp32 whose products fit, with queries or keys that the planes of bf16 do not hold in full range: the same weights as of their like of ordinary size."""
    s = Setting(1, 4, 2, n, 64, "f32", 16, [200, 100], None, seed=20)
    _, lse = chunk(s)
    s.Q.mul_(of_queries)
    s.K.mul_(1 / of_queries)
    w = z.zipvl_paged_weigh(s.Q, s.cache(), s.table.to(DEV), s.ints(s.lens), lse, s.scale)
    assert_weights(s, w, lse, None)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("n,spare", [(3, 1), (70, 1), (64, 300), (70, 300)])
@pytest.mark.parametrize("size", [1e10, 1e30, 3e38])
def test_paged_weigh_of_queries_that_weigh_nothing(dtype, d, n, spare, size):
    """An lse of -infinity leaves a query out, however large its (finite) numbers are."""
    say(f"weigh nothing {dtype} {d} {n} {spare} {size}")
    s = Setting(1, 4, 2, n, d, dtype, 256, [300, 90], None, seed=53, spare=spare)
    _, lse = chunk(s)
    out = (torch.arange(n) % 3 == 1).to(DEV)
    lse[:, 1:3, out] = -math.inf
    Q = s.Q.clone()
    Q[:, 1:3, out] = torch.where(Q[:, 1:3, out] < 0, -size, size).to(s.dtype)
    w = z.zipvl_paged_weigh(Q, s.cache(), s.table.to(DEV), s.ints(s.lens), lse, s.scale)
    assert_weights(s, w, lse, None)                           # which gives such queries' weights as 0


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 4, 50])
def test_paged_weigh_skips_rows_without_a_page_and_clamps_lengths(n):
    s = Setting(2, 4, 2, n, 128, "bf16", 16, [200, 77, 150, 64], None, seed=18)
    s.table[0, 2] = -1
    s.table[0, 5:8] = s.K.shape[0]
    s.table[1, :] = NONE
    s.lens[2] = 10 ** 9
    s.k = [n + 7, -3, 2 ** 31 - 1, n]
    _, lse = chunk(s)
    s.spoil()
    w = z.zipvl_paged_weigh(s.Q, s.cache(), s.table.to(DEV), s.ints(s.lens), lse, s.scale, k=s.ints(s.k))
    assert_weights(s, w, lse, None)


# ---------------------------------------------------------------- eviction
def evicted(s, weight, tokens, budget, sinks, recent, k=None):
    """Plain form: per unit (kept count, the tokens that all rows held), and the row that each of the new rows held before."""
    seen, source = [], []
    for u in range(s.B * s.Hkv):
        L = min(max(s.lens[u], 0), s.table.shape[1] * s.page)
        stay_n = min(L, budget if k is None else max(0, min(budget, k[u])))
        held = list(range(L)) if tokens is None else tokens[u, :L].tolist()
        following = max(held + [-1]) + 1
        for r in range(L):
            if held[r] < 0:
                held[r], following = following, following + 1
        latest = max(held + [-1])
        value = [float(x) if x > 0 else 0.0 for x in weight[u, :L].tolist()]          # no number is not above 0
        order = sorted(range(L), key=lambda r: (not (held[r] < sinks or held[r] > latest - recent), -value[r], r))
        stay = set(order[:stay_n])
        rows = list(range(stay_n))
        for gap, late in zip((r for r in range(stay_n) if r not in stay), (r for r in range(stay_n, L) if r in stay)):
            rows[gap] = late
        seen.append((stay_n, held))
        source.append(rows)
    return seen, source


EVICT = [  # B, Hkv, d, dtype, page, lens, budget, sinks, recent, tokens, weights, k
    (1, 1, 64, "f32", 16, [1], 0, 0, 0, False, "random", None),
    (1, 2, 128, "bf16", 16, [0, 1], 1, 0, 1, True, "random", None),
    (2, 2, 128, "bf16", 64, [100, 37, 64, 65], 64, 0, 0, False, "random", None),
    (2, 4, 64, "bf16", 32, [500, 20, 300, 1], 100, 4, 16, True, "random", None),
    (1, 3, 128, "f32", 16, [1000, 1023, 1025], 700, 0, 1000, True, "random", None),
    (1, 3, 128, "f32", 256, [1024, 2048, 2049], 2048, 2, 7, True, "ties", None),
    (2, 1, 64, "f32", 16, [333, 100], 50, 300, 3, True, "zeros", None),
    (3, 2, 128, "bf16", 128, [3000, 700, 0, 5000, 4097, 2], 999, 4, 64, True, "odd", None),
    (1, 4, 64, "bf16", 16, [900, 800, 700, 600], 10 ** 9, 0, 0, True, "random", [100, -1, 2 ** 31 - 1, 0]),
    (1, 2, 128, "bf16", 64, [34000, 20000], 12345, 4, 100, True, "ties", None),
    (70, 2, 64, "bf16", 16, [40, 33, 48], 32, 1, 4, False, "random", None),
    (1, 2, 64, "bf16", 128, [16000, 9000], 7000, 4, 100, True, "zeros", None),
    (1, 2, 64, "bf16", 256, [40000, 36900], 11111, 4, 100, True, "odd", None),
    (1, 2, 64, "f32", 16, [40000, 39970], 39960, 4, 100, True, "random", None),
    (2, 2, 128, "f32", 64, [4097, 8192, 4096, 20479], 4096, 0, 1, False, "ties", None),
]


def weights_of(kind, shape, seed):
    g = torch.Generator().manual_seed(seed)
    w = torch.exp(3 * torch.randn(shape, generator=g))
    if kind == "ties":
        w = torch.randint(0, 5, shape, generator=g).float() * 0.25
    elif kind == "zeros":
        w = torch.zeros(shape)
    elif kind == "odd":
        pick = torch.randint(0, 12, shape, generator=g)
        for i, x in enumerate([-0.0, -1.0, float("inf"), float("nan"), -float("inf"), 1e-45, -float("nan")]):
            w[pick == i] = x
    return w


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("case", EVICT, ids=lambda c: f"B{c[0]}Hkv{c[1]}d{c[2]}{c[3]}page{c[4]}to{c[6]}s{c[7]}r{c[8]}{'t' if c[9] else ''}{c[10]}{'k' if c[11] else ''}")
def test_paged_evict(case, in_place):
    B, Hkv, d, dtype, page, lens, budget, sinks, recent, with_tokens, kind, k = case
    say(f"evict {case}")
    s = Setting(B, Hkv, Hkv, 1, d, dtype, page, lens, seed=25)
    units, room = B * Hkv, s.table.shape[1] * page
    g = torch.Generator().manual_seed(3)
    weight = weights_of(kind, (units, room), 4)
    tokens = None
    if with_tokens:                                          # the first two thirds in no order, with gaps; the others new
        tokens = torch.full((units, room), -1, dtype=torch.int32)
        for u, L in enumerate(s.lens):
            known = L * 2 // 3
            tokens[u, :known] = (torch.randperm(known, generator=g) * 3).to(torch.int32)
            tokens[u, L:] = 10 ** 6                          # not looked at
    seen, source = evicted(s, weight, tokens, budget, sinks, recent, k)
    cache, length, w = s.cache(), s.ints(s.lens), weight.to(DEV)
    t = None if tokens is None else tokens.to(DEV)
    outs = {} if in_place else dict(length_out=torch.full_like(length, -9), weight_out=torch.full_like(w, 7.0), tokens_out=None if t is None else torch.full_like(t, 7))
    got = z.zipvl_paged_evict(cache, s.table.to(DEV), length, w, budget, k=s.ints(k), tokens=t, sinks=sinks, recent=recent, **outs)
    if not in_place:
        assert torch.equal(length.cpu(), torch.tensor(s.lens, dtype=torch.int32)) and torch.equal(w.cpu().view(torch.int32), weight.view(torch.int32))
        w, t = outs["weight_out"], outs["tokens_out"]
    assert got.tolist() == [n for n, _ in seen]
    K, V = s.K.clone(), s.V.clone()
    w, old = w.cpu(), weight if in_place else torch.full_like(weight, 7.0)
    for u in range(units):
        n, held = seen[u]
        for pool, ref in ((s.K, K), (s.V, V)):
            for to, come in enumerate(source[u]):
                if to != come:
                    ref[int(s.table[u, to // page]), to % page] = pool[int(s.table[u, come // page]), come % page]
        L = len(held)
        assert torch.equal(w[u, :n].view(torch.int32), weight[u, source[u]].view(torch.int32)), f"unit {u}: weights"
        assert (w[u, n:L] == 0).all() and torch.equal(w[u, L:].view(torch.int32), old[u, L:].view(torch.int32)), f"unit {u}: weights behind"
        if t is not None:
            assert t[u, :n].tolist() == [held[r] for r in source[u]], f"unit {u}: tokens"
            assert (t[u, n:L] == -1).all() and (t[u, L:] == (10 ** 6 if in_place else 7)).all(), f"unit {u}: tokens behind"
    assert torch.equal(cache.K.cpu(), K) and torch.equal(cache.V.cpu(), V)


@pytest.mark.gpu
def test_paged_evict_where_pages_are_missing():
    """Moves from or to rows that no page holds are left out; nothing else is written."""
    s = Setting(1, 2, 2, 1, 64, "f32", 16, [300, 200], seed=26)
    pages = s.K.shape[0]
    s.table[0, 1], s.table[0, 10], s.table[1, :] = -1, pages, NONE
    weight = weights_of("random", (2, s.table.shape[1] * 16), 5)
    seen, source = evicted(s, weight, None, 120, 0, 10)
    cache, length, w = s.cache(), s.ints(s.lens), weight.to(DEV)
    z.zipvl_paged_evict(cache, s.table.to(DEV), length, w, 120, recent=10)
    assert length.tolist() == [120, 120]
    K = s.K.clone()
    for u in range(2):
        for to, come in enumerate(source[u]):
            a, b = int(s.table[u, to // 16]), int(s.table[u, come // 16])
            if to != come and 0 <= a < pages and 0 <= b < pages:
                K[a, to % 16] = s.K[b, come % 16]
        assert torch.equal(w[u, :120].cpu(), weight[u, source[u]])
    assert torch.equal(cache.K.cpu(), K)


# ---------------------------------------------------------------- a run of them together
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,Hq,Hkv", [("bf16", 128, 8, 2), ("f32", 64, 4, 4)])
def test_conversations_within_a_budget(dtype, d, Hq, Hkv):
    """Pieces and single tokens of three conversations about one image: into pages, attention, weights, and rows leave; every step against a cache kept
    as lists of (token, key, value, weight)."""
    B, page, budget, sinks, recent = 3, 16, 40, 2, 8
    G, units, scale, T = Hq // Hkv, B * Hkv, 1.0 / math.sqrt(d), DT[dtype]
    g = torch.Generator().manual_seed(31)
    width, pre_width = 6, 5
    pages = units * width + Hkv * pre_width
    order = torch.randperm(pages, generator=g).to(torch.int32)
    table, prefix_table = order[:units * width].view(units, width).to(DEV), order[units * width:].view(Hkv, pre_width).to(DEV)
    cache = z.PagedCache.empty(pages, page, d, T, DEV)
    image = [torch.randn((1, Hkv, 70, d), generator=g).to(T) for _ in range(2)]
    prefix_len = torch.zeros(Hkv, dtype=torch.int32, device=DEV)
    z.zipvl_paged_append(image[0].to(DEV), image[1].to(DEV), cache, prefix_table, prefix_len)
    begin = torch.tensor([0, B], dtype=torch.int32, device=DEV)
    length = torch.zeros(units, dtype=torch.int32, device=DEV)
    weight = torch.zeros((units, width * page), device=DEV)
    tokens = torch.full((units, width * page), -1, dtype=torch.int32, device=DEV)
    lists = [[] for _ in range(units)]
    count = [0] * units
    for step, n in enumerate([30, 1, 1, 17, 1, 25, 1]):
        Q, K, V = (torch.randn((B, h, n, d), generator=g).to(T) for h in (Hq, Hkv, Hkv))
        ragged = [max(0, n - 5 * (u // Hkv)) if n > 1 else 1 for u in range(units)]
        k = torch.tensor(ragged, dtype=torch.int32, device=DEV)
        z.zipvl_paged_append(K.to(DEV), V.to(DEV), cache, table, length, k=k)
        O, lse = z.zipvl_chunk_attn_paged(Q.to(DEV), cache, table, length, scale, k=k, prefix_table=prefix_table, prefix_len=prefix_len, group_begin=begin, want_lse=True)
        z.zipvl_paged_weigh(Q.to(DEV), cache, table, length, lse, scale, k=k, before=weight, weight=weight)
        mine = weight.cpu()
        for u in range(units):
            b, h = divmod(u, Hkv)
            for i in range(ragged[u]):
                lists[u].append([count[u], K[b, h, i], V[b, h, i], 0.0])
                count[u] += 1
            c, L = ragged[u], len(lists[u])
            if c == 0:
                continue
            keys = torch.cat([image[0][0, h], torch.stack([x[1] for x in lists[u]])]).double()
            values = torch.cat([image[1][0, h], torch.stack([x[2] for x in lists[u]])]).double()
            q = Q[b, h * G:(h + 1) * G, :c].double()
            hidden = torch.ones((c, 70 + L), dtype=torch.bool).triu(70 + L - c + 1)
            w = torch.softmax((q @ keys.T * scale).masked_fill(hidden[None], -math.inf), dim=-1)
            big = float((q.abs() @ keys.abs().T).max()) * scale
            T_ = 2 * ((d + 4) * U * big + (len(keys) + 64) * U + (half_step(T) if T == torch.bfloat16 else 0))
            o = w @ values
            assert ((O[b, h * G:(h + 1) * G, :c].cpu().double() - o).abs() <= T_ * (w @ values.abs()) + half_step(T) * o.abs()).all(), f"step {step}, unit {u}"
            got = w.sum(dim=(0, 1))[70:]
            was = torch.tensor([x[3] for x in lists[u]], dtype=torch.float64)
            assert ((mine[u, :L].double() - was - got).abs() <= got * ((d + 6) * U * 2 * (big + 10) + (c * G + 80) * U) + 8 * U * (was + got)).all(), f"step {step}, unit {u}"
            for r in range(L):
                lists[u][r][3] = float(mine[u, r])            # what the cache holds: eviction goes by that
        z.zipvl_paged_evict(cache, table, length, weight, budget, tokens=tokens, sinks=sinks, recent=recent)
        for u in range(units):
            L = len(lists[u])
            n2 = min(L, budget)
            latest = max([x[0] for x in lists[u]] + [-1])
            rank = sorted(range(L), key=lambda r: (not (lists[u][r][0] < sinks or lists[u][r][0] > latest - recent), -lists[u][r][3], r))
            stay = set(rank[:n2])
            rows = list(range(n2))
            for gap, late in zip((r for r in range(n2) if r not in stay), (r for r in range(n2, L) if r in stay)):
                rows[gap] = late
            lists[u] = [lists[u][r] for r in rows]
            assert int(length[u]) == n2
            assert tokens[u, :n2].tolist() == [x[0] for x in lists[u]], f"step {step}, unit {u}: tokens"
            assert (tokens[u, n2:] == -1).all() and (weight[u, n2:] == 0).all()
            got = cache.K[table[u].long()].view(-1, d)[:n2].cpu()
            assert n2 == 0 or torch.equal(got, torch.stack([x[1] for x in lists[u]]).to(T))
        # the decode step sees the same rows, whatever their order
        q = torch.randn((B, Hq, 1, d), generator=g).to(T).to(DEV)
        one, _ = z.zipvl_chunk_attn_paged(q, cache, table, length, scale, prefix_table=prefix_table, prefix_len=prefix_len, group_begin=begin)
        o = z.zipvl_decode_attn_paged(q.reshape(-1, d), cache, table, length, scale, B=B, Hq=Hq, Hkv=Hkv, prefix_table=prefix_table, prefix_len=prefix_len, group_begin=begin)
        assert torch.allclose(one.reshape(-1, d).float(), o.float(), rtol=2 * half_step(T), atol=2e-6)


def steps(s, cache, table, length, weight, tokens, Q, K, V, ws, ews, O, lse, budget):
    z.zipvl_paged_append(K, V, cache, table, length)
    z.zipvl_chunk_attn_paged(Q, cache, table, length, s.scale, O=O, lse=lse, ws=ws)
    z.zipvl_paged_weigh(Q, cache, table, length, lse, s.scale, before=weight, weight=weight)
    z.zipvl_paged_evict(cache, table, length, weight, budget, tokens=tokens, sinks=1, recent=4, ws=ews)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 9])
def test_steps_as_a_graph_and_on_another_stream(n):
    """The four calls captured and replayed, with eager work between, and two graphs in turn: bits as when called one after the other."""
    B, Hq, Hkv, d, page, budget = 2, 14, 2, 128, 16, 900
    s = Setting(B, Hq, Hkv, n, d, "bf16", page, [1000 + n, 800 + n, 900 + n, 20 + n], seed=41)
    g = torch.Generator().manual_seed(42)
    Ks = [torch.randn((B, Hkv, n, d), generator=g).to(torch.bfloat16).to(DEV) for _ in range(5)]
    Qs = [torch.randn((B, Hq, n, d), generator=g).to(torch.bfloat16).to(DEV) for _ in range(5)]
    start = [x - n for x in s.lens]

    def state():
        cache, table = s.cache(), s.table.to(DEV)
        x = dict(cache=cache, table=table, length=s.ints(start), weight=torch.rand((B * Hkv, table.shape[1] * page), generator=torch.Generator().manual_seed(1)).to(DEV),
                 tokens=torch.full((B * Hkv, table.shape[1] * page), -1, dtype=torch.int32, device=DEV), Q=torch.empty_like(Qs[0]), K=torch.empty_like(Ks[0]), V=torch.empty_like(Ks[0]),
                 ws=z.chunk_paged_workspace(cache, table, B=B, Hq=Hq, Hkv=Hkv, n=n), ews=z.paged_evict_workspace(cache, table, budget),
                 O=torch.zeros((B, Hq, n, d), dtype=torch.bfloat16, device=DEV), lse=torch.zeros((B, Hq, n), device=DEV), budget=budget)
        return x

    def seen(x):
        return [x[name].clone() for name in ("length", "weight", "tokens", "O", "lse")] + [x["cache"].K.clone(), x["cache"].V.clone()]

    def feed(x, i):
        x["Q"].copy_(Qs[i])
        x["K"].copy_(Ks[i])
        x["V"].copy_(Ks[-1 - i])

    want, x = [], state()
    for i in range(5):
        feed(x, i)
        steps(s, **x)
        torch.cuda.synchronize()
        want.append(seen(x))
    # another stream
    y, side = state(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for i in range(5):
            feed(y, i)
            steps(s, **y)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(seen(y), want[-1]))
    # two graphs with buffers of their own, replayed in turn
    pair = [state(), state()]
    graphs = []
    for y in pair:
        feed(y, 0)
        kept = {name: y[name].clone() for name in ("length", "weight", "tokens")}
        pools = y["cache"].K.clone(), y["cache"].V.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            steps(s, **y)
        for name, t in kept.items():
            y[name].copy_(t)
        y["cache"].K.copy_(pools[0])
        y["cache"].V.copy_(pools[1])
        graphs.append(graph)
    for i in range(5):
        for y, graph in zip(pair, graphs):
            feed(y, i)
            graph.replay()
            torch.cuda.synchronize()
            busy = torch.randn(1000, device=DEV).sum()
            assert math.isfinite(float(busy))
            assert all(torch.equal(a, b) for a, b in zip(seen(y), want[i])), f"replay {i}"


@pytest.mark.gpu
def test_calls_of_the_extension_module_are_the_general_ones(monkeypatch):
    """The three calls through _pycall and through ctypes: the same bits; and tensors that it does not take are refused all the same."""
    from paper_2410_08584_amd import binding
    s = Setting(4, 8, 4, 20, 64, "bf16", 16, [20, 90, 300], [20, 3, 0], (0, 3, 4), (40, 77), order="token", seed=41)
    taken = []

    class Watched:
        def __init__(self, inner):
            self.inner = inner

        def __getattr__(self, name):
            def call(*args):
                taken.append((name, getattr(self.inner, name)(*args)))
                return taken[-1][1]
            return call

    table, a = s.table.to(DEV), s.args()

    def everything():
        cache, length = s.cache(), s.ints(s.lens)
        O, lse = torch.zeros((s.B, s.Hq, s.n, s.d), dtype=s.dtype, device=DEV), torch.zeros((s.B, s.Hq, s.n), device=DEV)
        z.zipvl_chunk_attn_paged(s.Q, cache, table, length, s.scale, O=O, lse=lse, ws=z.chunk_paged_workspace(cache, table, a["prefix_table"], B=s.B, Hq=s.Hq, Hkv=s.Hkv, n=s.n), **a)
        weight = torch.zeros((s.B * s.Hkv, s.table.shape[1] * s.page), device=DEV)
        z.zipvl_paged_weigh(s.Q, cache, table, length, lse, s.scale, k=a["k"], before=weight, weight=weight)
        tokens = torch.full(weight.shape, -1, dtype=torch.int32, device=DEV)
        out = dict(length_out=torch.zeros_like(length), weight_out=torch.zeros_like(weight), tokens_out=torch.zeros_like(tokens))
        z.zipvl_paged_evict(cache, table, length, weight, 60, tokens=tokens, sinks=2, recent=5, ws=z.paged_evict_workspace(cache, table, 60), **out)
        return O, lse, weight, *out.values(), cache.K, cache.V

    with monkeypatch.context() as m:
        m.setattr(binding, "_native", Watched(binding._native))
        fast = everything()
        assert taken == [("chunk_attn_paged", 0), ("paged_weigh", 0), ("paged_evict", 0)]
        cache, length, lse = s.cache(), s.ints(s.lens), torch.zeros((s.B, s.Hq, s.n), device=DEV)
        weight = torch.zeros((s.B * s.Hkv, s.table.shape[1] * s.page), device=DEV)
        for call in (lambda: z.zipvl_chunk_attn_paged(s.Q, cache, table, length.cpu(), s.scale, O=torch.zeros_like(s.Q), lse=lse, **a),
                     lambda: z.zipvl_paged_weigh(s.Q, cache, table, length, lse.double(), s.scale, weight=weight),
                     lambda: z.zipvl_paged_evict(cache, table, length, weight[:, :-1], 60)):
            with pytest.raises(z.ZipvlError):
                call()
    with monkeypatch.context() as m:
        m.setattr(binding, "_native", binding._NoExtension())
        general = everything()
    assert all(torch.equal(x, y) for x, y in zip(fast, general))


@pytest.mark.gpu
@pytest.mark.parametrize("B,Hq,Hkv,n,d,dtype,lens,groups,pre", [(6, 28, 4, 9, 128, "bf16", [900, 9, 40], (0, 6), (1500,)), (2, 8, 8, 300, 64, "f32", [2000, 300], (), ()),
                                                                (7, 4, 2, 5, 64, "bf16", [5000, 5], (), ()), (5, 2, 1, 40, 128, "f32", [40, 100], (1, 3, 5), (700, 64))])
def test_workspaces_are_kept_to(B, Hq, Hkv, n, d, dtype, lens, groups, pre):
    """Nothing behind the bytes that were asked for is written, and what they held does not matter."""
    s = Setting(B, Hq, Hkv, n, d, dtype, 16, lens, None, groups, pre, seed=42)
    cache, table, a = s.cache(), s.table.to(DEV), s.args()

    def guarded(ws):
        x = torch.full((ws.numel() + 4096,), 0xFF, dtype=torch.uint8, device=DEV)
        return x[:ws.numel()], x[ws.numel():]

    ws, guard = guarded(z.chunk_paged_workspace(cache, table, a["prefix_table"], B=B, Hq=Hq, Hkv=Hkv, n=n))
    O, lse = chunk(s, cache, ws=ws)
    assert (guard == 0xFF).all()
    assert_chunk(s, O, lse)
    weight = torch.rand((B * Hkv, s.table.shape[1] * 16), device=DEV)
    ws, guard = guarded(z.paged_evict_workspace(cache, table, 100))
    length = s.ints(s.lens)
    z.zipvl_paged_evict(cache, table, length, weight, 100, ws=ws)
    assert (guard == 0xFF).all() and length.tolist() == [min(x, 100) for x in s.lens]


# ---------------------------------------------------------------- refusals, on the CPU
@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(z.library_path()):
        from paper_2410_08584_amd.build import build_library
        build_library(verbose=False)
    return z.load_library()


FAKE, ODD = 0x100000, 0x100004


def dims(B=2, Hq=4, Hkv=2, n=8, d=64, dtype=1, q=None):
    from paper_2410_08584_amd.binding import Dims
    dm = Dims()
    dm.B, dm.Hq, dm.Hkv, dm.n, dm.d, dm.dtype = B, Hq, Hkv, n, d, dtype
    dm.q_strides = (C.c_int64 * 3)(*(q or (Hq * n * d, n * d, d)))
    return dm


def pages(K=FAKE, V=FAKE, num=10, page=16):
    return z.Pages(K, V, num, page)


def test_chunk_attn_paged_refuses(lib):
    def call(dm=None, pg=None, Q=FAKE, table=FAKE, width=4, length=FAKE, k=None, ptab=None, pwidth=0, plen=None, begin=None, groups=0, scale=0.1, O=0x900000, out=None,
             lse=None, ws=FAKE, nbytes=1 << 40):
        return lib.zipvl_chunk_attn_paged(Q, C.byref(pg or pages()), table, width, length, k, ptab, pwidth, plen, begin, groups, C.byref(dm or dims()), scale, O,
                                          C.byref(out) if out else None, lse, ws, nbytes, None)
    assert call(dims(Hq=5)) == -2 and call(dims(d=96)) == -2 and call(dims(dtype=3)) == -5 and call(dims(n=0)) == -1 and call(dims(B=0)) == -1
    assert call(dims(Hq=4096, Hkv=1, n=1 << 18, B=1)) == -2 and "2^30" in z.zipvl_last_error()
    assert call(dims(B=1 << 12, Hq=2, Hkv=1, n=1 << 18)) == -2
    assert call(dims(q=(512, 128, 60))) == -3 and call(dims(q=(512, 128, 56))) == -1 and call(dims(q=(-512, 128, 64))) == -1
    assert call(pg=pages(K=None)) == -1 and call(pg=pages(K=ODD)) == -3 and call(pg=pages(num=0)) == -1 and call(pg=pages(page=48)) == -2 and call(pg=pages(page=8)) == -2
    assert call(table=None) == -1 and call(width=0) == -1 and call(width=1 << 21) == -2 and call(table=0x100001) == -3
    assert call(Q=None) == -1 and call(Q=ODD) == -3 and call(O=None) == -1 and call(O=ODD) == -3 and call(O=FAKE) == -1
    assert call(length=None) == -1 and call(length=0x100002) == -3 and call(k=0x100001) == -3 and call(lse=0x100002) == -3
    assert call(groups=-1) == -1 and call(groups=3) == -1 and call(groups=1) == -1
    assert call(groups=1, ptab=FAKE, pwidth=0, plen=FAKE, begin=FAKE) == -1 and call(groups=1, ptab=FAKE, pwidth=2, plen=None, begin=FAKE) == -1
    assert call(groups=1, ptab=FAKE, pwidth=2, plen=0x100001, begin=FAKE) == -3
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert call(scale=scale) == -1
    assert call(out=dims(q=(512, 0, 64))) == -1 and "overlap" in z.zipvl_last_error()
    assert call(out=dims(q=(512, 128, 60))) == -3
    need = z.workspace_bytes(z.OP_CHUNK_PAGED, dims(), 4096 * 16)
    assert need > 0 and call(width=4096, ws=None) == -4 and call(width=4096, nbytes=need - 1) == -4 and call(width=4096, ws=ODD) == -3
    assert z.workspace_bytes(z.OP_CHUNK_PAGED, dims(), -1) == 0 and "negative" in z.zipvl_last_error()


def test_paged_weigh_refuses(lib):
    def call(dm=None, pg=None, Q=FAKE, table=FAKE, width=4, length=FAKE, k=None, lse=FAKE, pitch=8, scale=0.1, before=None, weight=0x900000):
        return lib.zipvl_paged_weigh(Q, C.byref(pg or pages()), table, width, length, k, lse, pitch, C.byref(dm or dims()), scale, before, weight, None)
    assert call(dims(Hq=5)) == -2 and call(dims(d=96)) == -2 and call(dims(dtype=3)) == -5 and call(dims(n=0)) == -1
    assert call(pg=pages(K=None)) == -1 and call(pg=pages(page=48)) == -2 and call(table=None) == -1 and call(width=0) == -1
    assert call(Q=None) == -1 and call(Q=ODD) == -3 and call(length=None) == -1 and call(lse=None) == -1 and call(weight=None) == -1
    assert call(lse=0x100001) == -3 and call(weight=0x900002) == -3 and call(before=0x900002) == -3 and call(k=0x100001) == -3
    assert call(pitch=7) == -1 and call(pitch=-8) == -1 and call(scale=0.0) == -1
    size = 4 * 4 * 16 * 4                                     # units, pages, rows, bytes
    assert call(before=0x900000 + size - 4) == -1 and "overlaps" in z.zipvl_last_error() and call(before=0x900000 - size + 4) == -1
    assert call(lse=0x900000 + size - 4) == -1 and call(length=0x900000) == -1 and call(k=0x900000) == -1 and call(table=0x900000 + 16) == -1


def test_paged_evict_refuses(lib):
    far = [0x1000000 * (x + 1) for x in range(8)]

    def call(dm=None, pg=None, table=far[0], width=4, length=far[1], k=None, weight=far[2], tokens=far[3], budget=10, sinks=0, recent=0, length_out=far[4], weight_out=far[5],
             tokens_out=far[6], ws=far[7], nbytes=1 << 40):
        return lib.zipvl_paged_evict(C.byref(pg or pages()), table, width, C.byref(dm or dims()), length, k, weight, tokens, budget, sinks, recent, length_out, weight_out,
                                     tokens_out, ws, nbytes, None)
    assert call(dims(d=96)) == -2 and call(dims(dtype=3)) == -5 and call(dims(B=0)) == -1 and call(dims(B=65536, Hkv=1)) == -2
    assert call(pg=pages(V=None)) == -1 and call(pg=pages(page=48)) == -2 and call(table=None) == -1 and call(width=0) == -1 and call(width=1 << 21) == -2
    for name in ("length", "weight", "length_out", "weight_out"):
        assert call(**{name: None}) == -1
    assert call(tokens=None) == -1 and call(tokens_out=None) == -1
    assert call(budget=-1) == -1 and call(sinks=-1) == -1 and call(recent=-1) == -1
    for name in ("length", "weight", "tokens", "k", "length_out", "weight_out", "tokens_out"):
        assert call(**{name: 0x5000002}) == -3
    for name in ("weight", "tokens", "weight_out", "tokens_out"):        # read and written by four rows
        assert call(**{name: 0x5000008}) == -3
    size = 4 * 4 * 16 * 4
    assert call(weight_out=far[2] + 16) == -1 and "overlaps" in z.zipvl_last_error() and call(tokens_out=far[2]) == -1 and call(weight_out=far[3] - size + 16) == -1
    assert call(length_out=far[2]) == -1 and call(length_out=far[0]) == -1 and call(weight_out=far[6] + 16) == -1 and "two outputs" in z.zipvl_last_error()
    assert call(k=far[1], length=far[1], length_out=far[1]) == -1
    need = z.workspace_bytes(z.OP_PAGED_EVICT, dims(n=64), 10)
    assert need >= 4 * 10 * 20 and call(ws=None) == -4 and call(nbytes=need - 1) == -4 and call(ws=far[7] + 4) == -3


def test_binding_refuses_what_does_not_fit():
    cache = z.PagedCache(torch.zeros((6, 16, 64)), torch.zeros((6, 16, 64)))
    Q, table, length = torch.zeros((2, 4, 3, 64)), torch.zeros((4, 3), dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    lse, weight = torch.zeros((2, 4, 3)), torch.zeros((4, 48))

    def refuses(f, *a, code=None, **k):
        with pytest.raises(z.ZipvlError) as e:
            f(*a, **k)
        assert code is None or e.value.code == code, e.value
    c = z.zipvl_chunk_attn_paged
    refuses(c, Q[0], cache, table, length, 0.1, code=-2)
    refuses(c, Q.to(torch.bfloat16), cache, table, length, 0.1, code=-5)
    refuses(c, torch.zeros((2, 4, 3, 128)), cache, table, length, 0.1, code=-2)
    refuses(c, Q, cache, table[:3], length, 0.1, code=-2)
    refuses(c, Q, cache, table[:, 0], length, 0.1, code=-2)
    refuses(c, Q, cache, table.long(), length, 0.1, code=-5)
    refuses(c, Q, cache, table, length[:3], 0.1, code=-2)
    refuses(c, Q, cache, table, length, 0.1, k=length[:2], code=-2)
    refuses(c, Q, cache, table, length, 0.1, prefix_table=table[:2], code=-1)
    refuses(c, Q, cache, table, length, 0.1, prefix_table=table[:2], prefix_len=length[:2], group_begin=length[:1], code=-2)
    refuses(c, Q, cache, table, length, 0.1, prefix_table=table[:3], prefix_len=length[:2], group_begin=length[:2], code=-2)
    refuses(c, Q, cache, table, length, 0.1, O=torch.zeros((2, 4, 3, 32)), code=-2)
    refuses(c, Q, cache, table, length, 0.1, O=Q.double(), code=-5)
    refuses(c, Q, cache, table, length, 0.1, lse=lse[:, :, :2], code=-2)
    refuses(c, Q, cache, table, length, 0.1, lse=torch.zeros((2, 3, 4)).transpose(1, 2), code=-1)
    refuses(c, Q, cache, table, length, 0.1, code=-1)          # not on a GPU
    w = z.zipvl_paged_weigh
    refuses(w, Q, cache, table, length, lse[:, :, :2], 0.1, code=-2)
    refuses(w, Q, cache, table, length, lse.double(), 0.1, code=-5)
    refuses(w, Q, cache, table, length, torch.zeros((2, 3, 4)).transpose(1, 2), 0.1, code=-1)
    refuses(w, Q, cache, table, length, torch.zeros((4, 2, 3)).transpose(0, 1), 0.1, code=-1)
    refuses(w, Q, cache, table, length, lse, 0.1, weight=weight[:, :47], code=-2)
    refuses(w, Q, cache, table, length, lse, 0.1, before=weight.double(), code=-5)
    refuses(w, Q, cache, table, length, lse, 0.1, code=-1)     # not on a GPU
    e = z.zipvl_paged_evict
    refuses(e, cache, table[0], length, weight, 10, code=-2)
    refuses(e, cache, table, length[:3], weight, 10, code=-2)
    refuses(e, cache, table, length, weight[:, :47], 10, code=-2)
    refuses(e, cache, table, length, weight.double(), 10, code=-5)
    refuses(e, cache, table, length, weight, 10, tokens=weight, code=-5)
    refuses(e, cache, table, length, weight, 10, tokens_out=weight, code=-1)
    refuses(e, cache, table, length, weight, -1, code=-1)
    refuses(e, cache, table, length, weight, 2 ** 31, code=-1)
    refuses(e, cache, table, length, weight, 10, recent=-1, code=-1)
    refuses(e, cache, table, length, weight, 10, k=length[:2], code=-2)
    refuses(e, cache, table, length, weight, 10, code=-1)      # not on a GPU
