"""Rotary positions, rows into paged caches and decode attention over pages with shared prefixes, against plain forms in 64 bits.

Tolerances.  u = 2^-24 is the rounding of fp32, h(t) = finfo(t).eps / 2 that of an output.
  rotation   sine and cosine are within 3.5 u of the true ones (one rounding each of the angle's fraction, of its factor and of the result, the
             cosine's square doubling the first two), so (x, y) comes out within 3.5 u (|x| + |y|), two roundings of products and sums within
             2 u (|x| + |y|): 6 u (|x| + |y|) + h |result|.
  attention  a logit is a sum of d products in chains of at most 32 additions: off by 32 u scale sum|q k|, and by u of itself in the exponent; a weight
             carries that as a factor, once in the numerator and once in the denominator; sums over L rows go in chains of L / 16 + 64 additions;
             bf16 weights keep 16 bits.  Relative to A = sum of weight |v|: T = 2 (34 u max(scale sum|q k|) + (L / 16 + 64) u + [bf16] 2^-16).
             Output: T A + h |result|.
"""
import ctypes as C
import math

import pytest
import torch

import paper_2410_08584_amd as z

DEV = "cuda:0"
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def say(msg):
    print(msg, flush=True)


# ---------------------------------------------------------------- plain forms, 64 bits, on the CPU
def rotated(x, pos, freqs, axes, layout, inverse=False):
    """x [B,H,n,d], pos [axes,B,n] -> (result, |x| + |y| of every element's pair; 0 for channels without a pair)"""
    out, size = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64)
    pairs = len(freqs)
    for i in range(pairs):
        a, b = (i, i + pairs) if layout == z.ROPE_HALVES else (2 * i, 2 * i + 1)
        t = pos[axes[i]].double() * freqs[i] * (-1 if inverse else 1)
        c, s = torch.cos(t)[:, None], torch.sin(t)[:, None]
        xa, xb = x[..., a].double(), x[..., b].double()
        out[..., a], out[..., b] = xa * c - xb * s, xa * s + xb * c
        size[..., a] = size[..., b] = xa.abs() + xb.abs()
    return out, size


def assert_rotated(got, x, pos, freqs, axes, layout, inverse=False):
    ref, size = rotated(x.cpu(), pos.cpu(), freqs, axes, layout, inverse)
    err = (got.cpu().double() - ref).abs()
    tol = 6 * U * size + half_step(got.dtype) * ref.abs() * (size > 0)
    assert (err <= tol).all(), f"worst {(err - tol).max().item():.3e} over"


def attention(q, K, V, scale):
    """q [G,d] against K, V [L,d] -> (o, bound without the output's own rounding)"""
    q, K, V = q.double(), K.double(), V.double()
    L = K.shape[0]
    if L == 0:
        return torch.zeros_like(q), torch.zeros_like(q)
    w = torch.softmax(q @ K.T * scale, dim=1)
    big = (q.abs() @ K.abs().T).max() * scale
    return w @ V, (2 * (34 * U * big + (L / 16 + 64) * U)) * (w @ V.abs())


def assert_attention(got, ref, bound, weights):
    dtype = got.dtype
    err = (got.cpu().double() - ref).abs()
    tol = bound + half_step(dtype) * ref.abs() + (2 * 2.0 ** -16 * weights if dtype == torch.bfloat16 else 0)
    over = (err - tol).max().item()
    assert over <= 0, f"worst {over:.3e} over"


# ---------------------------------------------------------------- rotation
def frequencies(pairs, theta=10000.0):
    return [theta ** (-i / pairs) for i in range(pairs)]


def axes_of(pairs, axes):
    return [i * axes // pairs for i in range(pairs)]


ROTATE = [  # B, Hq, Hkv, n, d, dtype, pairs, axes, layout, inverse, order
    (1, 4, 4, 1, 64, "f32", 32, 1, z.ROPE_HALVES, False, "head"),
    (2, 4, 2, 33, 128, "bf16", 64, 3, z.ROPE_HALVES, False, "token"),
    (3, 28, 4, 17, 128, "bf16", 64, 1, z.ROPE_NEIGHBOURS, True, "head"),
    (2, 6, 3, 100, 64, "bf16", 8, 2, z.ROPE_HALVES, False, "head"),
    (1, 5, 1, 257, 128, "f32", 24, 4, z.ROPE_NEIGHBOURS, False, "token"),
    (5, 8, 8, 65, 64, "f32", 16, 2, z.ROPE_NEIGHBOURS, True, "token"),
    (70, 2, 1, 1, 128, "f32", 64, 3, z.ROPE_HALVES, False, "head"),
    (1, 32, 32, 700, 128, "bf16", 32, 2, z.ROPE_HALVES, True, "head"),
    (2, 3, 3, 5000, 64, "bf16", 32, 3, z.ROPE_HALVES, False, "token"),
]


def layer(B, Hq, Hkv, n, d, dtype, order, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((B, Hq + 2 * Hkv, n, d), generator=g).to(DT[dtype]).to(DEV)
    if order == "token":
        x = x.transpose(1, 2).contiguous().transpose(1, 2)
    return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]


def positions(axes, B, n, seed, low=-5, high=70000):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(low, high, (axes, B, n), generator=g, dtype=torch.int64).to(torch.int32).to(DEV)


@pytest.mark.gpu
@pytest.mark.parametrize("case", ROTATE, ids=lambda c: f"B{c[0]}n{c[3]}d{c[4]}{c[5]}p{c[6]}x{c[7]}l{c[8]}{'inv' if c[9] else ''}{c[10]}")
def test_rotate(case):
    B, Hq, Hkv, n, d, dtype, pairs, axes, layout, inverse, order = case
    say(f"rotate {case}")
    Q, K, _ = layer(B, Hq, Hkv, n, d, dtype, order, 1)
    pos = positions(axes, B, n, 2)
    f, a = frequencies(pairs), axes_of(pairs, axes)
    rope = z.Rope(f, a, layout)
    flags = z.ROTATE_INVERSE if inverse else 0
    Qo, Ko = z.zipvl_rotate(Q, K, pos, rope, flags)
    assert_rotated(Qo, Q, pos, f, a, layout, inverse)
    assert_rotated(Ko, K, pos, f, a, layout, inverse)
    # one tensor alone, and in the place of the input: the same bits; what stands between the rows of a view is left alone
    only, none = z.zipvl_rotate(None, K, pos, rope, flags)
    assert only is None and torch.equal(none, Ko)
    whole = torch.full((B, n, Hq + 3, d), 7.0, dtype=Q.dtype, device=DEV)
    view = whole[:, :, 1:1 + Hq].transpose(1, 2)
    view.copy_(Q)
    z.zipvl_rotate(view, None, pos, rope, flags, Qo=view)
    assert torch.equal(view, Qo)
    assert bool((whole[:, :, 0] == 7).all()) and bool((whole[:, :, 1 + Hq:] == 7).all())


@pytest.mark.gpu
@pytest.mark.parametrize("low,high", [(-2 ** 31, 2 ** 31 - 1), (2 ** 24, 2 ** 24 + 100), (0, 1)])
def test_rotate_far_positions(low, high):
    """Whole turns are dropped exactly: positions at the ends of int32, beyond 2^24, and zero (which copies)."""
    B, H, n, d, pairs = 2, 3, 64, 128, 64
    K, _, _ = layer(B, H, H, n, d, "f32", "head", 3)
    pos = positions(1, B, n, 4, low, high)
    pos[0, 0, :3] = torch.tensor([low, low, high - 1 if high == 1 else high - 1], dtype=torch.int64).to(torch.int32)
    f = [6.28, -1.0] + frequencies(pairs)[2:]
    _, Ko = z.zipvl_rotate(None, K, pos, z.Rope(f))
    # the plain form's own angle, |pos| freq, is rounded at 2^-53 of 2^31 * 6.28: 1.5e-6 of a radian; taken in whole turns by exact fractions instead
    from fractions import Fraction
    two_pi = Fraction(314159265358979323846264338327950288419716939937510582097494459, 10 ** 62) * 2
    p = pos.cpu()[0]
    angle = torch.empty((B, n, pairs), dtype=torch.float64)
    for b in range(B):
        for t in range(n):
            for i in range(pairs):
                turns = Fraction(f[i]) * int(p[b, t]) / two_pi
                angle[b, t, i] = float((turns - math.floor(turns)) * two_pi)
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    x = K.cpu().double()
    xa, xb = x[..., :pairs], x[..., pairs:]
    ref, size = torch.cat([xa * c - xb * s, xa * s + xb * c], dim=-1), (xa.abs() + xb.abs()).repeat(1, 1, 1, 2)
    # beyond 2^24 the angle itself is off by up to 1e-9 a position's 2^-24th part: 2^31 / 2^24 * 1e-9
    err, tol = (Ko.cpu().double() - ref).abs(), (6 * U + 1.3e-7) * size + half_step(torch.float32) * ref.abs()
    assert (err <= tol).all(), (err - tol).max().item()
    if high == 1:
        assert torch.equal(Ko, K)


@pytest.mark.gpu
@pytest.mark.parametrize("inverse", [False, True])
def test_rotate_at_the_ends_of_int32(inverse):
    """The fraction of a turn is off by 3.7e-9 radians at most, at any position: turns a position truncated at 3 2^-64 (times 2^31: 2.2e-9) and 32 bits kept (1.5e-9)."""
    from fractions import Fraction
    say(f"rotate at the ends inverse={inverse}")
    n, d, pairs = 40, 128, 64
    K, _, _ = layer(1, 1, 1, n, d, "f32", "head", 8)
    pos = positions(1, 1, n, 9, -2 ** 31, 2 ** 31)
    pos[0, 0, :12] = torch.tensor([-2 ** 31, 2 ** 31 - 1, -2 ** 31 + 1, 2 ** 31 - 2, 2 ** 30, -2 ** 30, 2 ** 24 + 1, 0xFFFF, -1, 0, 1, 2 ** 30 - 1])
    f = [2 * math.pi, -2 * math.pi, 6.28, -6.2, 5.0, 4.0, 3.9999, -2.0, 1e-300, -1e-12, 0.0] + frequencies(pairs)[11:]
    _, Ko = z.zipvl_rotate(None, K, pos, z.Rope(f), z.ROTATE_INVERSE if inverse else 0)
    two_pi = Fraction(314159265358979323846264338327950288419716939937510582097494459, 10 ** 62) * 2
    angle = torch.empty((n, pairs), dtype=torch.float64)
    for t in range(n):
        for i in range(pairs):
            turns = Fraction(f[i]) * int(pos[0, 0, t]) / two_pi
            angle[t, i] = float((turns - math.floor(turns)) * two_pi) * (-1 if inverse else 1)
    c, s = torch.cos(angle), torch.sin(angle)
    x = K.cpu().double()[0, 0]
    xa, xb = x[:, :pairs], x[:, pairs:]
    ref, size = torch.cat([xa * c - xb * s, xa * s + xb * c], dim=-1), (xa.abs() + xb.abs()).repeat(1, 2)
    err, tol = (Ko.cpu().double()[0, 0] - ref).abs(), (6 * U + 3.7e-9) * size + half_step(torch.float32) * ref.abs()
    assert (err <= tol).all(), (err - tol).max().item()


@pytest.mark.gpu
@pytest.mark.parametrize("layout", [z.ROPE_HALVES, z.ROPE_NEIGHBOURS])
def test_the_inverse_rotation_is_the_gradient(layout):
    """d/dx of sum(w * rotate(x)) is the inverse rotation of w: against differences of the kernel itself (rotation is linear: any step will do), and
    against autograd of the plain form."""
    B, H, n, d, pairs = 1, 2, 9, 64, 24
    K, _, w = layer(B, H, H, n, d, "f32", "head", 5)
    pos, f = positions(2, B, n, 6), frequencies(pairs)
    a = axes_of(pairs, 2)
    rope = z.Rope(f, a, layout)
    grad = z.zipvl_rotate(None, w, pos, rope, z.ROTATE_INVERSE)[1].cpu().double()
    x = K.cpu().double().requires_grad_()
    first, second = (torch.arange(pairs), torch.arange(pairs) + pairs) if layout == z.ROPE_HALVES else (2 * torch.arange(pairs), 2 * torch.arange(pairs) + 1)
    t = torch.stack([pos.cpu()[a[i]].double() * f[i] for i in range(pairs)], dim=-1)[:, None]
    loss = (w.cpu().double()[..., first] * (x[..., first] * torch.cos(t) - x[..., second] * torch.sin(t))).sum()
    loss = loss + (w.cpu().double()[..., second] * (x[..., first] * torch.sin(t) + x[..., second] * torch.cos(t))).sum()
    loss = loss + (w.cpu().double()[..., 2 * pairs:] * x[..., 2 * pairs:]).sum()
    loss.backward()
    size = rotated(w.cpu(), pos.cpu(), f, a, layout, True)[1]
    assert ((grad - x.grad).abs() <= 6 * U * size + half_step(torch.float32) * x.grad.abs() * (size > 0)).all()
    base = z.zipvl_rotate(None, torch.zeros_like(K), pos, rope)[1]
    for channel in (0, 1, pairs - 1, pairs, 2 * pairs - 1, d - 1):
        step = torch.zeros_like(K)
        step[..., channel] = 1.0
        slope = ((z.zipvl_rotate(None, step, pos, rope)[1] - base).cpu().double() * w.cpu().double()).sum(dim=-1)
        # two sums of at most two products of w with a sine or cosine, each within 6 u
        assert ((slope - grad[..., channel]).abs() <= 14 * U * (size[..., channel] + w.cpu().double()[..., channel].abs())).all()


# ---------------------------------------------------------------- rows into pages
def random_table(units, width, num_pages, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randperm(num_pages, generator=g)[:units * width].view(units, width).to(torch.int32).to(DEV)


def pools(num_pages, page, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return z.PagedCache(*(torch.randn((num_pages, page, d), generator=g).to(DT[dtype]).to(DEV) for _ in range(2)))


APPEND = [  # B, Hq (0: no queries), Hkv, n, d, dtype, page, pairs, axes, k, starts, idx, order
    (3, 28, 4, 1, 128, "bf16", 64, 64, 3, None, [0, 63, 64], False, "head"),
    (2, 8, 2, 40, 64, "bf16", 16, 32, 1, [[40, 0], [17, 16]], [5, 16], False, "token"),
    (4, 4, 4, 333, 64, "f32", 32, 16, 2, "batch", [0, 31, 32, 33], False, "head"),
    (1, 0, 3, 700, 128, "bf16", 128, 0, 0, [[700, 1, 129]], [0], True, "head"),
    (2, 0, 2, 257, 128, "f32", 256, 64, 3, [[100, 257], [0, 255]], [250, 1], True, "token"),
    (2, 0, 2, 200, 64, "bf16", 16, 32, 2, "batch", [3, 0], True, "head"),
    (2, 0, 5, 90, 128, "bf16", 16, 0, 0, None, [7, 100], False, "token"),
    (65, 2, 1, 1, 64, "f32", 16, 24, 1, "batch", [1], False, "head"),
    (2, 0, 2, 50, 128, "bf16", 64, 64, 1, [[-3, 51], [10 ** 6, 50]], [0, 1], False, "head"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("case", APPEND, ids=lambda c: f"B{c[0]}Hq{c[1]}Hkv{c[2]}n{c[3]}d{c[4]}{c[5]}page{c[6]}p{c[7]}{'idx' if c[11] else ''}{c[12]}")
def test_paged_append(case, in_place):
    B, Hq, Hkv, n, d, dtype, page, pairs, axes, k, starts, with_idx, order = case
    say(f"paged_append {case} in_place={in_place}")
    units = B * Hkv
    Q, K, V = layer(B, max(Hq, 1), Hkv, n, d, dtype, order, 7)
    g = torch.Generator().manual_seed(8)
    per_batch = k == "batch"
    if per_batch:
        k = torch.randint(0, n + 1, (B,), generator=g)
    elif k is not None:
        k = torch.tensor(k).reshape(-1)
    start = torch.tensor([starts[u % len(starts)] for u in range(units)])
    width = -(-(max(starts) + n) // page)
    cache = pools(units * width + 2, page, d, dtype, 9)
    table = random_table(units, width, cache.num_pages, 10)
    idx = None
    if with_idx:
        idx = torch.stack([torch.randperm(n, generator=g).sort().values if i % 2 else torch.randperm(n, generator=g) for i in range(len(k))]).to(torch.int32)
    pos = positions(axes, B, n, 11) if pairs else None
    f, a = frequencies(pairs) if pairs else [], axes_of(pairs, axes) if pairs else []
    rope = z.Rope(f, a) if pairs else None
    want_K, want_V = cache.K.clone().cpu(), cache.V.clone().cpu()
    size_K = torch.zeros(want_K.shape, dtype=torch.float64)
    want_K64 = want_K.double()
    Kr, size = rotated(K.cpu(), pos.cpu(), f, a, z.ROPE_HALVES) if pairs else (K.cpu().double(), torch.zeros(K.shape, dtype=torch.float64))
    want_len, counts = [], []
    for u in range(units):
        b, h = divmod(u, Hkv)
        m = n if k is None else min(max(int(k[b if per_batch else u]), 0), n)
        counts.append(m)
        for i in range(m):
            t = int(idx[b if per_batch else u, i]) if with_idx else i
            r = int(start[u]) + i
            at = (int(table[u, r // page]), r % page)
            want_K64[at], size_K[at], want_V[at] = Kr[b, h, t], size[b, h, t], V[b, h, t].cpu()
        want_len.append(int(start[u]) + m)
    start_d = start.to(torch.int32).to(DEV)
    length = start_d if in_place else torch.full((units,), -9, dtype=torch.int32, device=DEV)
    Qo = torch.full((B, Hq, n, d), 3.0, dtype=DT[dtype], device=DEV) if Hq else None
    got, _ = z.zipvl_paged_append(K, V, cache, table, start_d, idx=None if idx is None else idx.to(DEV), k=None if k is None else k.to(torch.int32).to(DEV),
                                  pos=pos, rope=rope, Q=Q if Hq else None, Qo=Qo, length=None if in_place else length,
                                  flags=z.T_PER_BATCH if per_batch else 0)
    torch.cuda.synchronize()
    assert got is length and length.tolist() == want_len
    if not in_place:
        assert torch.equal(start_d.cpu(), start.to(torch.int32))
    assert torch.equal(cache.V.cpu(), want_V)
    err = (cache.K.cpu().double() - want_K64).abs()
    assert (err <= 6 * U * size_K + half_step(DT[dtype]) * want_K64.abs() * (size_K > 0)).all()         # unrotated and untouched rows: bit copies
    if Hq:
        Qr, qsize = rotated(Q.cpu(), pos.cpu(), f, a, z.ROPE_HALVES)
        for b in range(B):
            for h in range(Hq):
                m = counts[b * Hkv + h // (Hq // Hkv)]
                err = (Qo[b, h, :m].cpu().double() - Qr[b, h, :m]).abs()
                assert (err <= 6 * U * qsize[b, h, :m] + half_step(DT[dtype]) * Qr[b, h, :m].abs() * (qsize[b, h, :m] > 0)).all()
                assert bool((Qo[b, h, m:] == 3).all())


@pytest.mark.gpu
@pytest.mark.parametrize("layout", [z.ROPE_HALVES, z.ROPE_NEIGHBOURS])
@pytest.mark.parametrize("B,Hq,Hkv,n,d,dtype,pairs,k", [(3, 8, 2, 1, 128, "bf16", 64, None), (2, 6, 3, 37, 64, "f32", 24, [[37, 5, 0], [1, 36, 17]]), (4, 28, 4, 130, 128, "bf16", 16, None),
                                                        (3, 4, 4, 65, 128, "f32", 64, "batch")])
def test_paged_append_with_queries_in_place(layout, B, Hq, Hkv, n, d, dtype, pairs, k):
    """Qo in the place of Q, pairs of both layouts: the rows that a head's unit brings are turned, the others stay."""
    say(f"paged_append in place B={B} n={n} {dtype} layout={layout} k={k}")
    page, units, axes = 32, B * Hkv, 2
    Q, K, V = (x.contiguous() for x in layer(B, Hq, Hkv, n, d, dtype, "head", 14))
    per_batch = k == "batch"
    counts = [n] * units if k is None else [(7 + 29 * b) % (n + 1) for b in range(B) for _ in range(Hkv)] if per_batch else sum(k, [])
    k_d = None if k is None else torch.tensor(counts[::Hkv] if per_batch else counts, dtype=torch.int32, device=DEV)
    pos, f, a = positions(axes, B, n, 15), frequencies(pairs), axes_of(pairs, axes)
    width = -(-(n + 20) // page)
    cache, table = pools(units * width, page, d, dtype, 16), random_table(units, width, units * width, 17)
    start = torch.tensor([u * 5 % 21 for u in range(units)], dtype=torch.int32, device=DEV)
    want, at = Q.clone(), Q
    length, got = z.zipvl_paged_append(K, V, cache, table, start, k=k_d, pos=pos, rope=z.Rope(f, a, layout), Q=at, Qo=at, length=torch.empty_like(start),
                                       flags=z.T_PER_BATCH if per_batch else 0)
    assert got is at and length.tolist() == [int(start[u]) + counts[u] for u in range(units)]
    for u in range(units):
        b, g, m = u // Hkv, u % Hkv, counts[u]
        heads = slice(g * (Hq // Hkv), (g + 1) * (Hq // Hkv))
        assert torch.equal(at[b, heads, m:], want[b, heads, m:])
        if m:
            assert_rotated(at[b:b + 1, heads, :m], want[b:b + 1, heads, :m], pos[:, b:b + 1, :m], f, a, layout)
            rows = cache.K[table[u].long()].view(-1, d)[int(start[u]):int(start[u]) + m]
            assert_rotated(rows[None, None], K[b:b + 1, g:g + 1, :m], pos[:, b:b + 1, :m], f, a, layout)
            assert torch.equal(cache.V[table[u].long()].view(-1, d)[int(start[u]):int(start[u]) + m], V[b, g, :m])


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 70])
def test_paged_append_where_pages_end_or_are_missing(n):
    """Rows behind the table, and rows whose page is none, are not written; lengths stop at the table's end; starts outside are clamped."""
    B, Hkv, d, page, width = 2, 2, 64, 16, 4
    _, K, V = layer(B, 1, Hkv, n, d, "bf16", "head", 12)
    cache = pools(20, page, d, "bf16", 13)
    table = torch.tensor([[1, 2, 3, 4], [5, -1, 7, 8], [9, 20, 2 ** 31 - 1, -2 ** 31], [13, 14, 15, 16]], dtype=torch.int32, device=DEV)
    start = torch.tensor([60, 14, 0, -7], dtype=torch.int32, device=DEV)
    want_K, want_V = cache.K.clone(), cache.V.clone()
    want_len = []
    for u in range(4):
        s = min(max(int(start[u]), 0), width * page)
        for i in range(n):
            r = s + i
            if r >= width * page or not 0 <= int(table[u, r // page]) < 20:
                continue
            want_K[int(table[u, r // page]), r % page] = K[u // 2, u % 2, i]
            want_V[int(table[u, r // page]), r % page] = V[u // 2, u % 2, i]
        want_len.append(min(s + n, width * page))
    length, _ = z.zipvl_paged_append(K, V, cache, table, start, length=torch.zeros_like(start))
    assert length.tolist() == want_len
    assert torch.equal(cache.K, want_K) and torch.equal(cache.V, want_V)
    full = torch.full((4,), width * page, dtype=torch.int32, device=DEV)
    z.zipvl_paged_append(K, V, cache, table, full)                      # full caches are left as they are
    assert full.tolist() == [width * page] * 4
    assert torch.equal(cache.K, want_K) and torch.equal(cache.V, want_V)


@pytest.mark.gpu
def test_paged_append_of_more_heads_than_a_grid_has_rows():
    heads, n, d = 40000, 64, 64
    K = torch.arange(heads * n, dtype=torch.int32, device=DEV).view(1, heads, n, 1).expand(1, heads, n, 8).contiguous().view(torch.bfloat16).repeat(1, 1, 1, 4)
    V = K.flip(1)
    cache = z.PagedCache(*(torch.zeros((heads, n, d), dtype=torch.bfloat16, device=DEV) for _ in range(2)))
    table = torch.arange(heads - 1, -1, -1, dtype=torch.int32, device=DEV).view(heads, 1)
    length, _ = z.zipvl_paged_append(K, V, cache, table, torch.zeros(heads, dtype=torch.int32, device=DEV))
    assert torch.equal(cache.K.view(torch.int16), K[0].flip(0).view(torch.int16)) and torch.equal(cache.V.view(torch.int16), V[0].flip(0).view(torch.int16))
    assert (length == n).all()


def needs_memory(gib):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib * 2 ** 30:
        pytest.skip(f"{gib} GiB of free GPU memory are needed")


@pytest.mark.gpu
def test_paged_append_of_more_tokens_than_one_grid_has_threads():
    """33 x 2^24 tokens, of which every sequence brings the first few: those of the last are tokens beyond 2^29."""
    needs_memory(16)
    B, n, d, page, c = 33, 1 << 24, 128, 16, 5
    K = torch.zeros((1, 1, n, d), dtype=torch.bfloat16, device=DEV)
    K[0, 0, :c] = torch.randn((c, d), generator=torch.Generator().manual_seed(91)).to(DEV)
    wide = K.expand(B, 1, n, d)
    pos = torch.zeros((1, B, n), dtype=torch.int32, device=DEV)
    pos[0, :, :c] = positions(1, B, c, 92)[0]
    f = frequencies(64)
    cache = pools(B, page, d, "bf16", 93)
    table = torch.arange(B - 1, -1, -1, dtype=torch.int32, device=DEV).view(B, 1)
    before = cache.K.clone()
    length, _ = z.zipvl_paged_append(wide, wide, cache, table, torch.zeros((B,), dtype=torch.int32, device=DEV),
                                     k=torch.full((B,), c, dtype=torch.int32, device=DEV), pos=pos, rope=z.Rope(f))
    assert (length == c).all()
    assert_rotated(cache.K.flip(0)[:, None, :c], K[:, :, :c].expand(B, 1, c, d), pos[:, :, :c], f, [0] * 64, z.ROPE_HALVES)
    assert torch.equal(cache.V[:, :c], K[0, :, :c].expand(B, c, d)) and torch.equal(cache.K[:, c:], before[:, c:])


@pytest.mark.gpu
def test_rotate_more_tokens_than_one_grid_has_threads():
    needs_memory(160)
    B, n, d = 33, 1 << 24, 128
    K = torch.zeros((B, 1, n, d), dtype=torch.bfloat16, device=DEV)
    pos = torch.zeros((1, B, n), dtype=torch.int32, device=DEV)
    spots = [(0, 0), (15, n - 5), (16, 0), (31, n - 5), (32, 0), (32, n // 2 + 3), (32, n - 5)]
    rows = torch.randn((len(spots), 1, 5, d), generator=torch.Generator().manual_seed(94)).to(torch.bfloat16).to(DEV)
    at = positions(1, len(spots), 5, 95)
    for i, (b, t) in enumerate(spots):
        K[b, 0, t:t + 5], pos[0, b, t:t + 5] = rows[i, 0], at[0, i]
    f = frequencies(64)
    z.zipvl_rotate(None, K, pos, z.Rope(f), Ko=K)
    got = torch.stack([K[b, :, t:t + 5] for b, t in spots])
    assert_rotated(got, rows, at, f, [0] * 64, z.ROPE_HALVES)


# ---------------------------------------------------------------- attention over pages
class Batch:
    """A batch in pages whose unused rows and unused pages hold NaN, and its plain result."""

    def __init__(self, B, Hq, Hkv, d, dtype, page, lens, groups=(), prefix=(), seed=0, gain=1.0, begin=None, wide=0, spike=0.0):
        g = torch.Generator().manual_seed(seed)
        G = Hq // Hkv
        self.B, self.Hq, self.Hkv, self.d, self.scale, self.dtype = B, Hq, Hkv, d, 1.0 / math.sqrt(d), DT[dtype]
        self.lens = [lens[u % len(lens)] for u in range(B * Hkv)]
        P = len(groups)
        self.begin = list(begin) if begin is not None else ([sum(groups[:p]) for p in range(P + 1)] if P else None)
        self.prefix = [prefix[u % len(prefix)] for u in range(P * Hkv)] if P else []
        width, pwidth = max(1, -(-max(self.lens) // page)) + wide, max(1, -(-max(self.prefix, default=0) // page)) + wide
        used = [-(-x // page) for x in self.lens + self.prefix]
        num = sum(used) + 3
        order = torch.randperm(num, generator=g)
        K = torch.full((num, page, d), math.nan)
        V = torch.full((num, page, d), math.nan)
        tables, rows, at = [], [], 0
        for u, length in enumerate(self.lens + self.prefix):
            own = u < len(self.lens)
            pages = order[at:at + used[u]]
            at += used[u]
            k, v = torch.randn((length, d), generator=g) * gain, torch.randn((length, d), generator=g)
            if spike and length:
                k[int(torch.randint(0, length, (1,), generator=g))] *= spike
            k, v = k.to(self.dtype), v.to(self.dtype)
            for j, p in enumerate(pages.tolist()):
                part = slice(j * page, min(length, (j + 1) * page))
                K[p, :part.stop - part.start], V[p, :part.stop - part.start] = k[part].float(), v[part].float()
            rows.append((k, v))
            w = width if own else pwidth
            tables.append(torch.cat([pages, torch.randint(-5, num + 5, (w - len(pages),), generator=g)]))
        self.rows, self.prefix_rows = rows[:len(self.lens)], rows[len(self.lens):]
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
        self.table = torch.stack(tables[:len(self.lens)]).to(torch.int32).to(DEV)
        self.prefix_table = torch.stack(tables[len(self.lens):]).to(torch.int32).to(DEV) if P else None
        self.length, self.prefix_len, self.group_begin = ints(self.lens), ints(self.prefix) if P else None, ints(self.begin) if P else None
        self.cache = z.PagedCache(K.to(self.dtype).to(DEV), V.to(self.dtype).to(DEV))
        self.q = torch.randn((B * Hq, d), generator=g).to(self.dtype).to(DEV)
        self.P = P

    def group(self, b):
        return next((p for p in range(self.P) if self.begin[p] <= b < self.begin[p + 1]), None)

    def run(self, **kw):
        return z.zipvl_decode_attn_paged(self.q, self.cache, self.table, self.length, self.scale, B=self.B, Hq=self.Hq, Hkv=self.Hkv,
                                         prefix_table=self.prefix_table, prefix_len=self.prefix_len, group_begin=self.group_begin, **kw)

    def check(self, o, which=None):
        G = self.Hq // self.Hkv
        for b in range(self.B) if which is None else which:
            for h in range(self.Hkv):
                k, v = self.rows[b * self.Hkv + h]
                p = self.group(b)
                if p is not None:
                    k, v = (torch.cat([x, y]) for x, y in zip(self.prefix_rows[p * self.Hkv + h], (k, v)))
                heads = slice(b * self.Hq + h * G, b * self.Hq + (h + 1) * G)
                q = self.q[heads].cpu()
                ref, bound = attention(q, k, v, self.scale)
                size = torch.softmax(q.double() @ k.double().T * self.scale, dim=1) @ v.double().abs() if k.shape[0] else torch.zeros_like(ref)
                assert_attention(o[heads], ref, bound, size)


DECODE = [  # B, Hq, Hkv, d, dtype, page, lens, groups, prefix
    (1, 1, 1, 64, "f32", 16, [1], (), ()),
    (2, 4, 4, 128, "bf16", 16, [0, 1, 15, 16, 17, 31, 32, 33], (), ()),
    (3, 28, 4, 128, "bf16", 64, [63, 64, 65, 200, 0, 7], (), ()),
    (2, 8, 2, 64, "bf16", 32, [5, 700, 33, 129], (), ()),
    (2, 32, 1, 128, "f32", 16, [100, 3], (), ()),
    (2, 32, 1, 64, "bf16", 256, [300, 255], (), ()),
    (2, 4, 4, 64, "f32", 16, [40, 3, 16, 0], (2,), [576, 575, 17, 1]),
    (8, 28, 4, 128, "bf16", 64, [30, 0, 64, 150], (8,), [1000, 640, 700, 65]),
    (5, 6, 2, 128, "f32", 128, [10, 300, 0], (1, 4), [400, 0, 129, 128]),
    (17, 8, 8, 64, "bf16", 16, [9, 40], (3, 0, 13, 1), [333, 90, 15]),
    (40, 16, 2, 128, "bf16", 32, [20, 5, 70], (33, 7), [500, 260]),
    (33, 4, 1, 64, "f32", 16, [12, 0], (33,), [200]),
    (70, 2, 2, 128, "bf16", 16, [3], (70,), [90]),
    (3, 14, 2, 128, "bf16", 128, [0], (2, 1), [1, 257]),
    (2, 4, 4, 64, "bf16", 16, [0], (2,), [0]),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", DECODE, ids=lambda c: f"B{c[0]}Hq{c[1]}Hkv{c[2]}d{c[3]}{c[4]}page{c[5]}P{len(c[7])}")
def test_decode_attn_paged(case):
    say(f"decode_attn_paged {case}")
    batch = Batch(*case, seed=21)
    o = batch.run()
    batch.check(o)
    # wider tables (other splits), an output and a workspace of the caller's that held something else
    wide = Batch(*case, seed=21, wide=40)
    ws = z.decode_paged_workspace(wide.cache, wide.table, wide.prefix_table, B=wide.B, Hq=wide.Hq, Hkv=wide.Hkv).fill_(255)
    out = torch.full((wide.B * wide.Hq, wide.d), math.nan, dtype=wide.dtype, device=DEV)
    assert wide.run(o=out, ws=ws) is out
    wide.check(out)
    again = wide.run(ws=ws)
    assert torch.equal(out, again)                                       # the order of all sums is fixed


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("groups", [(), (6,), (2, 4)])
def test_decode_attn_paged_long(dtype, d, groups):
    """Lengths that are cut into many parts, unequal within the batch."""
    say(f"decode_attn_paged long {dtype} {d} {groups}")
    batch = Batch(6, 14, 2, d, dtype, 64, [5000, 40, 0, 1, 2049, 300, 16, 17, 9000, 128, 64, 1000], groups, [7000, 3001, 4097, 1] if groups else [], seed=22)
    batch.check(batch.run())


@pytest.mark.gpu
@pytest.mark.parametrize("case", [  # B, Hq, Hkv, d, dtype, page, lens, groups, prefix: more items than workgroups of their own
    (40, 16, 8, 64, "bf16", 16, [5, 40, 0, 33, 700, 64, 1], (17, 3, 20), [600, 0, 333, 1200]),
    (33, 24, 8, 128, "bf16", 64, [90, 3, 0, 1500], (33,), [2000, 100]),
    (80, 8, 4, 128, "f32", 32, [10, 0, 200, 31], (75, 5), [900, 33, 500]),
    (130, 4, 2, 64, "f32", 16, [64, 7], (), []),
    (45, 128, 8, 64, "bf16", 16, [20, 100], (30, 15), [300, 17]),
    (35, 160, 8, 128, "bf16", 128, [33, 0, 260], (35,), [700]),
    (200, 2, 2, 64, "bf16", 16, [3], tuple([1] * 150), [40, 16, 0]),
], ids=lambda c: f"B{c[0]}Hq{c[1]}Hkv{c[2]}d{c[3]}{c[4]}P{len(c[7])}")
def test_decode_attn_paged_of_many_items(case):
    say(f"decode_attn_paged many {case[:6]}")
    batch = Batch(*case, seed=28)
    o = batch.run()
    batch.check(o, which=list(range(0, batch.B, 3)) + [batch.B - 1])
    assert torch.equal(o, batch.run())


@pytest.mark.gpu
@pytest.mark.parametrize("case", DECODE + [(6, 14, 2, 128, "f32", 64, [5000, 40, 0, 1, 2049], (2, 4), [7000, 3001, 1]), (6, 32, 1, 64, "bf16", 16, [9000, 40, 300], (6,), [3000])],
                         ids=lambda c: f"B{c[0]}Hq{c[1]}Hkv{c[2]}d{c[3]}{c[4]}page{c[5]}P{len(c[7])}")
def test_decode_attn_paged_stays_in_its_workspace(case):
    """A workspace of exactly the bytes that the tables need: what follows it is left alone, and the output is the same as with one of wider tables."""
    say(f"decode_attn_paged workspace {case}")
    batch = Batch(*case, seed=34)
    dm = z.dims_of(None, None, None, B=batch.B, Hq=batch.Hq, Hkv=batch.Hkv, n=batch.table.shape[1] * case[5], d=batch.d, dtype=1 if case[4] == "bf16" else 0)
    need = z.workspace_bytes(z.OP_DECODE_PAGED, dm, batch.prefix_table.shape[1] * case[5] if batch.P else 0)
    room = torch.full((need + (1 << 20),), 0xA5, dtype=torch.uint8, device=DEV)
    o = batch.run(ws=room[:need])
    batch.check(o)
    assert bool((room[need:] == 0xA5).all())
    with pytest.raises(z.ZipvlError, match="workspace"):
        batch.run(ws=room[:need - 1])


@pytest.mark.gpu
@pytest.mark.parametrize("lens", [[1, 0, 16, 17], [0], [0, 0, 0, 0, 0, 0, 5]])
def test_decode_attn_paged_of_thousands_of_units(lens):
    """More units than are looked at in LDS, most of them short or empty, one long."""
    say(f"decode_attn_paged thousands {lens}")
    B, Hq, Hkv = 700, 8, 8
    lens = (lens * (B * Hkv))[:B * Hkv]
    lens[3333] = 900
    batch = Batch(B, Hq, Hkv, 64, "bf16", 16, lens, (300, 0, 400), [33], seed=29)
    batch.check(batch.run(), which=[0, 1, 2, 150, 299, 300, 301, 416, 417, 500, 698, 699])


@pytest.mark.gpu
@pytest.mark.parametrize("case", [  # B, Hq, Hkv, d, dtype, page, lens, groups, prefix: items longer than many workgroups' pieces, and pieces of one item
    (64, 8, 8, 64, "bf16", 64, [3, 40, 0, 64, 31] * 20 + [30000] + [17, 1, 0] * 137, (), ()),
    (2, 16, 2, 128, "f32", 32, [6000, 1, 0, 90], (2,), [20000, 33]),
    (1, 8, 2, 128, "bf16", 16, [33, 40000], (1,), [17000, 700]),
    (20, 16, 8, 128, "bf16", 64, [4000, 2500, 5100, 10, 3000, 4500, 0], (20,), [3000, 500]),
    (20, 16, 8, 64, "bf16", 64, [9000, 2500, 5100, 12000, 3000], (9, 2), [3000, 5000]),
    (2, 64, 2, 64, "f32", 32, [19000, 5000, 0, 700], (), ()),
    (30, 4, 2, 128, "f32", 128, [2000, 3000, 900, 4000], (16, 14), [5000]),
], ids=lambda c: f"B{c[0]}Hq{c[1]}Hkv{c[2]}d{c[3]}{c[4]}P{len(c[7])}")
def test_decode_attn_paged_of_long_items(case):
    say(f"decode_attn_paged long items {case[:6]}")
    batch = Batch(*case, seed=31)
    o = batch.run()
    batch.check(o, which=sorted({0, 1 % batch.B, batch.B // 5, batch.B - 2 if batch.B > 1 else 0, batch.B - 1}))
    assert torch.equal(o, batch.run())


@pytest.mark.gpu
@pytest.mark.parametrize("case", [  # B, Hq, Hkv, d, dtype, page, lens, groups, prefix: many rows, one or two of whose items have most of the parts
    (64, 32, 1, 128, "bf16", 64, [3, 40, 0, 70] * 8 + [40000] + [5] * 31, (), ()),
    (53, 31, 1, 64, "bf16", 32, [2] * 50 + [30000, 0, 9000], (), ()),
    (70, 24, 2, 128, "f32", 16, [1, 7] * 69 + [9000, 12000], (40, 2, 28), [17, 5000, 0, 300, 40, 8]),
], ids=lambda c: f"B{c[0]}Hq{c[1]}Hkv{c[2]}d{c[3]}{c[4]}P{len(c[7])}")
def test_decode_attn_paged_of_many_rows_one_of_them_long(case):
    say(f"decode_attn_paged many rows {case[:6]}")
    batch = Batch(*case, seed=35)
    o = batch.run()
    batch.check(o, which=sorted({0, 1, 2, 31, 32, 33, 40, 41, 42, batch.B - 3, batch.B - 2, batch.B - 1}))
    assert torch.equal(o, batch.run())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("gain,spike", [(20.0, 0.0), (1.0, 40.0), (1e-3, 0.0)])
def test_decode_attn_paged_where_one_row_has_all_the_weight(dtype, d, gain, spike):
    """Logits up to some hundreds, of both signs; running maxima that are exceeded late."""
    say(f"decode_attn_paged gain {gain} spike {spike} {dtype}")
    batch = Batch(4, 8, 2, d, dtype, 32, [700, 33, 90, 2000], (3, 1), [900, 300], seed=23, gain=gain, spike=spike)
    batch.check(batch.run())


@pytest.mark.gpu
@pytest.mark.parametrize("B,Hq,Hkv,groups", [(64, 2, 1, ()), (64, 32, 1, ()), (20, 40, 40, (20,))], ids=["16 columns", "32 columns", "a block of a prefix"])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_attn_paged_keeps_all_bits_of_bf16_weights(B, Hq, Hkv, groups, d):
    """Two rows of weights 1 and w = exp(-a), 0 < a < 0.7, whose values nearly cancel: (w r - v) / (1 + w) with v = w r rounded to bf16.  w is off by 4 u (the scale,
    the exponent, its power of two: u, u, 2 u), r <= 2 makes 8 u of that, at most six roundings of sums up to 2 are 12 u, and the sum of weights is 1.5 and more:
    14 u, and half a step of the result.  A weight of 16 bits is off by up to 2^-18, which is 64 u."""
    say(f"decode_attn_paged weights B={B} Hq={Hq} Hkv={Hkv} d={d}")
    g = torch.Generator().manual_seed(41)
    P, page = len(groups), 16
    units = P * Hkv if P else B * Hkv
    a = (0.02 + 0.67 * torch.rand((units,), generator=g)).to(torch.bfloat16)
    w = torch.exp(-a.double())
    r = (1 + torch.rand((units, d), generator=g)).to(torch.bfloat16)
    v = (w[:, None] * r.double()).to(torch.bfloat16)
    K, V = (torch.zeros((units, page, d), dtype=torch.bfloat16) for _ in range(2))
    K[:, 1, 0], V[:, 0], V[:, 1] = -a, -v, r
    q = torch.zeros((B * Hq, d), dtype=torch.bfloat16)
    q[:, 0] = 1.0
    pages = torch.arange(units, dtype=torch.int32, device=DEV).view(units, 1)
    two = torch.full((units,), 2, dtype=torch.int32, device=DEV)
    prefix = dict(prefix_table=pages, prefix_len=two, group_begin=torch.tensor([0, B], dtype=torch.int32, device=DEV)) if P else {}
    table, length = (torch.zeros((B * Hkv, 1), dtype=torch.int32, device=DEV), torch.zeros((B * Hkv,), dtype=torch.int32, device=DEV)) if P else (pages, two)
    o = z.zipvl_decode_attn_paged(q.to(DEV), z.PagedCache(K.to(DEV), V.to(DEV)), table, length, 1.0, B=B, Hq=Hq, Hkv=Hkv, **prefix).cpu().double()
    ref = ((w[:, None] * r.double() - v.double()) / (1 + w[:, None])).view(-1, Hkv, 1, d).expand(B, Hkv, Hq // Hkv, d).reshape(B * Hq, d)
    err, tol = (o - ref).abs(), 14 * U + half_step(torch.bfloat16) * ref.abs()
    assert (err <= tol).all(), f"worst {(err - tol).max().item():.3e} over"


@pytest.mark.gpu
@pytest.mark.parametrize("case", [  # B, Hq, Hkv, d, dtype, page, lens, groups, prefix
    (3, 28, 4, 128, "bf16", 16, [1, 17, 33, 700], (), ()),
    (2, 8, 4, 64, "bf16", 64, [5, 48, 100, 2000], (), ()),
    (2, 64, 2, 64, "bf16", 32, [40, 333], (), ()),
    (5, 40, 2, 128, "bf16", 32, [0], (5,), [50, 900]),
    (4, 4, 4, 64, "bf16", 16, [3, 20], (3,), [70, 33]),
    (3, 8, 2, 128, "f32", 16, [1, 17, 33, 500], (), ()),
    (5, 40, 2, 64, "f32", 32, [0], (5,), [50, 400]),
], ids=lambda c: f"B{c[0]}Hq{c[1]}Hkv{c[2]}d{c[3]}{c[4]}P{len(c[7])}")
def test_decode_attn_paged_with_infinities(case):
    """Of every sequence, or prefix, one row of V has an infinity (the first, the last, a middle one, or the first of the last tile of 32, which others stand in for): its channel
    is infinite, of its sign, for all heads that see it, and the other channels are as without it.  One key is infinite against queries of the other sign: it weighs nothing."""
    say(f"decode_attn_paged infinities {case}")
    batch = Batch(*case, seed=33)
    page, inf = case[5], math.inf
    batch.q = batch.q.abs()
    sign, at = {}, 0
    units = [(batch.table[u], batch.rows, u) for u in range(len(batch.rows))] + [(batch.prefix_table[u], batch.prefix_rows, u) for u in range(len(batch.prefix_rows))]
    for table, rows, u in units:
        k, v = rows[u]
        n = k.shape[0]
        if n == 0:
            continue
        row = [0, n - 1, n // 2, (n - 1) // 32 * 32][at % 4]
        channel, value = at % batch.d, inf if at % 3 else -inf
        at += 1
        batch.cache.V[int(table[row // page]), row % page, channel] = value
        v[row, channel] = 0.0
        sign[id(rows), u] = channel, value
        if n > 40:                                                       # another row's key; as a row of the plain form it goes
            gone = row + 1 if row + 1 < n else row - 1
            batch.cache.K[int(table[gone // page]), gone % page, 1] = -inf
            keep = torch.arange(n) != gone
            rows[u] = k[keep], v[keep]
    o = batch.run()
    expected, G = {}, batch.Hq // batch.Hkv
    for b in range(batch.B):
        for h in range(batch.Hkv):
            heads = slice(b * batch.Hq + h * G, b * batch.Hq + (h + 1) * G)
            p = batch.group(b)
            seen = [sign.get((id(batch.rows), b * batch.Hkv + h))] + ([sign.get((id(batch.prefix_rows), p * batch.Hkv + h))] if p is not None else [])
            for channel, value in filter(None, seen):
                assert bool((o[heads, channel] == value).all()), (b, h, channel, value)
                expected[b, h, channel] = heads
    for (b, h, channel), heads in expected.items():                      # the other channels: with the infinite ones taken from the plain form
        k, v = batch.rows[b * batch.Hkv + h]
        p = batch.group(b)
        if p is not None:
            k, v = (torch.cat([x, y]) for x, y in zip(batch.prefix_rows[p * batch.Hkv + h], (k, v)))
        o[heads, channel] = attention(batch.q[heads].cpu(), k, v, batch.scale)[0][:, channel].to(o.dtype).to(DEV)
    batch.check(o)


@pytest.mark.gpu
def test_decode_attn_paged_without_a_group_and_in_any_partition():
    """Batch elements in front of, between and behind the groups have no prefix; bounds outside the batch are clamped."""
    for begin, groups in (([2, 4, 5], (2, 1)), ([1, 1, 3], (0, 2)), ([-4, 3, 100], (3, 3))):
        batch = Batch(6, 8, 4, 64, "bf16", 16, [20, 0, 50], groups, [100, 31], seed=24, begin=begin)
        batch.check(batch.run())


@pytest.mark.gpu
@pytest.mark.parametrize("junk", [0x00, 0x3F, 0x7F, 0xC0, 0xFF])
def test_decode_attn_paged_of_groups_that_fall(junk):
    """Groups that fall may overlap: whatever the workspace holds then, nothing outside it is read, and the next call, with groups that ascend, is right."""
    say(f"decode_attn_paged groups that fall, workspace of {junk:#x}")
    batch = Batch(40, 8, 4, 64, "bf16", 16, [20, 0, 50], (25, 15), [100, 31], seed=27)
    ws = z.decode_paged_workspace(batch.cache, batch.table, batch.prefix_table, B=batch.B, Hq=batch.Hq, Hkv=batch.Hkv).fill_(junk)
    begin = batch.group_begin.clone()
    for falling in ([0, 40, 0], [40, 0, 40], [2 ** 31 - 1, -2 ** 31, 7]):
        batch.group_begin.copy_(torch.tensor(falling))
        batch.run(ws=ws)
    batch.group_begin.copy_(begin)
    batch.check(batch.run(ws=ws))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_attn_paged_skips_rows_without_a_page_and_clamps_lengths(dtype):
    batch = Batch(2, 4, 2, 64, dtype, 16, [64, 64, 64, 64], (2,), [48, 48], seed=25)
    num = batch.cache.num_pages
    for u, (table, rows) in enumerate([(batch.table[1], batch.rows), (batch.prefix_table[0], batch.prefix_rows)]):
        table[1] = [-1, num][u]
        which = [1, 0][u]
        k, v = rows[which]
        keep = torch.cat([torch.arange(16), torch.arange(32, k.shape[0])])
        rows[which] = (k[keep], v[keep])
    batch.length.copy_(torch.tensor([1000, 64, -3, 2 ** 31 - 1], dtype=torch.int32))
    batch.rows[2] = tuple(x[:0] for x in batch.rows[2])
    batch.check(batch.run())
    batch.table.fill_(num + 7)                                           # nothing of their own is left
    batch.prefix_table.fill_(-1)
    assert not batch.run().any()


@pytest.mark.gpu
def test_decode_attn_paged_over_more_than_4_gib():
    """Pages whose bytes are beyond 32-bit offsets, for both directions (2 x 4.3 GiB of pages)."""
    say("decode_attn_paged 4 GiB")
    d, page, num = 128, 256, (1 << 32) // (256 * 128 * 2) + 1500
    cache = z.PagedCache.empty(num, page, d, torch.bfloat16, DEV)
    B, Hkv, n = 2, 2, 600
    _, K, V = layer(B, 4, Hkv, n, d, "bf16", "head", 26)
    table = (num - 1 - torch.arange(12).view(4, 3) * 100).to(torch.int32).to(DEV)
    length, _ = z.zipvl_paged_append(K, V, cache, table, torch.zeros((4,), dtype=torch.int32, device=DEV), length=torch.empty((4,), dtype=torch.int32, device=DEV))
    for u in range(4):
        got = cache.K[table[u].long()].view(-1, d)[:n]
        assert torch.equal(got, K[u // 2, u % 2])
    q = torch.randn((B * 4, d), generator=torch.Generator().manual_seed(27)).to(torch.bfloat16).to(DEV)
    o = z.zipvl_decode_attn_paged(q, cache, table, length, 0.1, B=B, Hq=4, Hkv=Hkv)
    for u in range(4):
        heads = slice(2 * u, 2 * u + 2)
        k, v = K[u // 2, u % 2].cpu(), V[u // 2, u % 2].cpu()
        ref, bound = attention(q[heads].cpu(), k, v, 0.1)
        assert_attention(o[heads], ref, bound, torch.softmax(q[heads].cpu().double() @ k.double().T * 0.1, dim=1) @ v.double().abs())


# ---------------------------------------------------------------- together
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,Hq,Hkv", [("bf16", 128, 8, 2), ("f32", 64, 4, 4)])
def test_questions_about_one_image(dtype, d, Hq, Hkv):
    """An image is prefilled once: rotated, scored, thinned, its kept rows put into pages as a prefix.  Three questions of unequal lengths then start their
    own pages and take two decode steps each.  The outputs of both steps against attention in 64 bits over the kept rows and the conversation's own."""
    say(f"questions about one image {dtype}")
    n, page, B = 300, 32, 3
    scale = 1.0 / math.sqrt(d)
    f, a = frequencies(d // 2), axes_of(d // 2, 3)
    rope = z.Rope(f, a)
    Q, K, V = layer(1, Hq, Hkv, n, d, dtype, "token", 31)
    K = (K + 3.0 * (torch.rand((1, Hkv, n, 1), generator=torch.Generator().manual_seed(32)) < 0.1).to(DEV) * Q[:, :Hkv].mean(dim=2, keepdim=True)).to(DT[dtype])
    pos = positions(3, 1, n, 33, 0, 40)
    Qr, Kr = z.zipvl_rotate(Q, K, pos, rope)
    mass, rank = z.zipvl_score(Qr, Kr, list(range(n - 64, n)), scale)
    idx, k = z.zipvl_select(mass, rank, 0.9)
    width = -(-n // page)
    cache = pools(3 + Hkv * width + B * Hkv * 3, page, d, dtype, 34)
    order = random_table(1, cache.num_pages, cache.num_pages, 35)[0]
    prefix_table, table = order[:Hkv * width].view(Hkv, width), order[Hkv * width:Hkv * width + B * Hkv * 3].view(B * Hkv, 3)
    prefix_len, _ = z.zipvl_paged_append(Kr, V, cache, prefix_table, torch.zeros((Hkv,), dtype=torch.int32, device=DEV), idx=idx, k=k,
                                         length=torch.empty((Hkv,), dtype=torch.int32, device=DEV))
    begin = torch.tensor([0, B], dtype=torch.int32, device=DEV)
    # the questions, padded to the longest
    lens = torch.tensor([17, 40, 1], dtype=torch.int32, device=DEV)
    _, Kq, Vq = layer(B, Hq, Hkv, 40, d, dtype, "head", 36)
    posq = (50 + torch.arange(40, device=DEV, dtype=torch.int32)).expand(3, B, 40).contiguous()
    length = torch.zeros((B * Hkv,), dtype=torch.int32, device=DEV)
    z.zipvl_paged_append(Kq, Vq, cache, table, length, k=lens, pos=posq, rope=rope, flags=z.T_PER_BATCH)
    tol_k = lambda x, size: 6 * U * size + half_step(DT[dtype]) * x.abs()
    own = []
    Kq64 = rotated(Kq.cpu(), posq.cpu(), f, a, z.ROPE_HALVES)
    for u in range(B * Hkv):
        b, h = divmod(u, Hkv)
        m = int(lens[b])
        got = cache.K[table[u].long()].view(-1, d)[:m].cpu()
        assert ((got.double() - Kq64[0][b, h, :m]).abs() <= tol_k(Kq64[0][b, h, :m], Kq64[1][b, h, :m])).all()
        own.append([got, Vq[b, h, :m].cpu()])                            # as stored: what the attention is defined on
    kept = [Kr[0, h, idx[h, :int(k[h])].long()].cpu() for h in range(Hkv)], [V[0, h, idx[h, :int(k[h])].long()].cpu() for h in range(Hkv)]
    assert prefix_len.tolist() == k.tolist() and int(k.max()) < n
    for step in range(2):
        q, kn, vn = layer(B, Hq, Hkv, 1, d, dtype, "token", 40 + step)
        at = (50 + lens + step).view(1, B, 1).expand(3, B, 1).contiguous()
        length, qr = z.zipvl_paged_append(kn, vn, cache, table, length, pos=at, rope=rope, Q=q)
        o = z.zipvl_decode_attn_paged(qr, cache, table, length, scale, B=B, Hq=Hq, Hkv=Hkv, prefix_table=prefix_table, prefix_len=prefix_len, group_begin=begin)
        assert_rotated(qr, q, at, f, a, z.ROPE_HALVES)
        kn64, size = rotated(kn.cpu(), at.cpu(), f, a, z.ROPE_HALVES)
        for u in range(B * Hkv):
            b, h = divmod(u, Hkv)
            m = int(lens[b]) + step
            row = cache.K[int(table[u, m // page]), m % page].cpu()
            assert ((row.double() - kn64[b, h, 0]).abs() <= tol_k(kn64[b, h, 0], size[b, h, 0])).all()
            own[u] = [torch.cat([own[u][0], row[None]]), torch.cat([own[u][1], vn[b, h].cpu()])]
            G = Hq // Hkv
            heads = slice(b * Hq + h * G, b * Hq + (h + 1) * G)
            kk, vv = torch.cat([kept[0][h], own[u][0]]), torch.cat([kept[1][h], own[u][1]])
            qq = qr.view(B * Hq, d)[heads].cpu()
            ref, bound = attention(qq, kk, vv, scale)
            assert_attention(o[heads], ref, bound, torch.softmax(qq.double() @ kk.double().T * scale, dim=1) @ vv.double().abs())


@pytest.mark.gpu
def test_decode_steps_as_a_graph_and_on_another_stream():
    """A captured step (append with rotation, then attention) advances lengths on the device: every replay against the eager step from the same state."""
    say("graph of paged decode steps")
    B, Hq, Hkv, d, page = 5, 8, 2, 128, 16
    batch = Batch(B, Hq, Hkv, d, "bf16", page, [30, 31, 32, 90, 1, 15, 16, 17, 60, 0], (4, 1), [200, 333], seed=51)
    rope = z.Rope.of_sections((16, 24, 24))
    width = 12
    order = torch.randperm(B * Hkv * width + 1, generator=torch.Generator().manual_seed(52)).to(torch.int32)
    base = batch.cache.num_pages
    grown = [torch.cat([x, torch.zeros((B * Hkv * width + 1, page, d), dtype=x.dtype, device=DEV)]) for x in (batch.cache.K, batch.cache.V)]
    table = (base + order[:B * Hkv * width].view(B * Hkv, width)).to(DEV)
    for u in range(B * Hkv):                                             # full pages stay where they are, the rest has pages to grow into
        whole = batch.lens[u] // page
        table[u, :whole] = batch.table[u, :whole]
        if batch.lens[u] % page:
            for x in grown:
                x[int(table[u, whole])] = x[int(batch.table[u, whole])]
    q, kn, vn = layer(B, Hq, Hkv, 1, d, "bf16", "head", 53)
    pos = positions(3, B, 1, 54)

    def make():
        cache = z.PagedCache(*(x.clone() for x in grown))
        return dict(cache=cache, length=batch.length.clone(), pos=pos.clone(), Qo=torch.empty((B, Hq, 1, d), dtype=torch.bfloat16, device=DEV),
                    o=torch.empty((B * Hq, d), dtype=torch.bfloat16, device=DEV),
                    ws=z.decode_paged_workspace(cache, table, batch.prefix_table, B=B, Hq=Hq, Hkv=Hkv))

    def step(s):
        z.zipvl_paged_append(kn, vn, s["cache"], table, s["length"], pos=s["pos"], rope=rope, Q=q, Qo=s["Qo"])
        z.zipvl_decode_attn_paged(s["Qo"], s["cache"], table, s["length"], batch.scale, B=B, Hq=Hq, Hkv=Hkv, prefix_table=batch.prefix_table,
                                  prefix_len=batch.prefix_len, group_begin=batch.group_begin, o=s["o"], ws=s["ws"])
        s["pos"] += 1

    eager, captured, other = make(), make(), make()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    warm = make()
    with torch.cuda.stream(side):
        step(warm)
        for _ in range(4):
            step(other)                                                  # torch's current stream is the one that is used
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured)
    for i in range(4):
        step(eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(captured["o"], eager["o"]) and torch.equal(captured["length"], eager["length"])
        assert torch.equal(captured["length"].cpu(), batch.length.cpu() + i + 1)
    for s in (captured, other):
        assert torch.equal(s["o"], eager["o"])
        assert s["cache"].K.view(torch.int16).equal(eager["cache"].K.view(torch.int16)) and s["cache"].V.view(torch.int16).equal(eager["cache"].V.view(torch.int16))


@pytest.mark.gpu
def test_calls_of_the_extension_module_are_the_general_ones(monkeypatch):
    """Positions and pages through _pycall and through ctypes: the same bits; and tensors that it does not take are refused all the same."""
    from paper_2410_08584_amd import binding
    B, Hq, Hkv, n, d, page = 3, 8, 4, 20, 64, 16
    rope = z.Rope.of_sections((8, 12, 12))
    Q, K, V = layer(B, Hq, Hkv, n, d, "bf16", "token", 61)
    pos = positions(3, B, n, 62)
    batch = Batch(B, Hq, Hkv, d, "bf16", page, [3, 50, 16], (2, 1), [40, 77], seed=63)
    taken = []

    class Watched:
        def __init__(self, inner):
            self.inner = inner

        def __getattr__(self, name):
            def call(*args):
                rc = getattr(self.inner, name)(*args)
                taken.append((name, rc))
                return rc
            return call

    def everything():
        Qo, Ko = torch.zeros((B, Hq, n, d), dtype=Q.dtype, device=DEV), torch.zeros((B, Hkv, n, d), dtype=Q.dtype, device=DEV)
        z.zipvl_rotate(Q, K, pos, rope, z.ROTATE_INVERSE, Qo=Qo, Ko=Ko)
        cache = pools(60, page, d, "bf16", 64)
        table = random_table(B * Hkv, 4, 60, 65)
        start = torch.arange(B * Hkv, dtype=torch.int32, device=DEV)
        k = torch.tensor([20, 3, 0], dtype=torch.int32, device=DEV)
        Qa = torch.zeros((B, Hq, n, d), dtype=Q.dtype, device=DEV)
        z.zipvl_paged_append(K, V, cache, table, start, k=k, pos=pos, rope=rope, Q=Q, Qo=Qa, flags=z.T_PER_BATCH)
        o = torch.zeros((B * Hq, d), dtype=Q.dtype, device=DEV)
        batch.run(o=o, ws=z.decode_paged_workspace(batch.cache, batch.table, batch.prefix_table, B=B, Hq=Hq, Hkv=Hkv))
        return Qo, Ko, cache.K, cache.V, start, Qa, o

    with monkeypatch.context() as m:
        m.setattr(binding, "_native", Watched(binding._native))
        fast = everything()
        assert [rc for name, rc in taken if name in ("rotate", "paged_append", "decode_attn_paged")] == [0, 0, 0]
        with pytest.raises(z.ZipvlError, match="one GPU"):
            z.zipvl_rotate(Q, K, pos.cpu(), rope, Qo=torch.empty_like(Q), Ko=torch.empty_like(K))
        with pytest.raises(z.ZipvlError, match="pos has"):
            z.zipvl_rotate(Q, K, pos[:2], rope, Qo=torch.empty_like(Q), Ko=torch.empty_like(K))
        with pytest.raises(z.ZipvlError, match="contiguous"):
            z.zipvl_rotate(Q, K, pos.transpose(1, 2).contiguous().transpose(1, 2), rope, Qo=torch.empty_like(Q), Ko=torch.empty_like(K))
        assert [rc for name, rc in taken[-3:]] == [None] * 3
    with monkeypatch.context() as m:
        m.setattr(binding, "_native", binding._NoExtension())
        general = everything()
    assert all(torch.equal(a, b) for a, b in zip(fast, general))


@pytest.mark.gpu
@pytest.mark.parametrize("extension", [True, False])
def test_pools_that_were_replaced(extension, monkeypatch):
    """A pool that has grown by assignment, and has shrunk: pages are counted as they are at the call, by the extension module and without it."""
    from paper_2410_08584_amd import binding
    if not extension:
        monkeypatch.setattr(binding, "_native", binding._NoExtension())
    Hkv, n, d, page = 2, 16, 64, 16
    _, K, V = layer(1, 1, Hkv, n, d, "bf16", "head", 81)
    cache = pools(4, page, d, "bf16", 82)
    table = torch.tensor([[7], [3]], dtype=torch.int32, device=DEV)
    start = torch.zeros((Hkv,), dtype=torch.int32, device=DEV)
    q = K[0, :, 3].contiguous()
    o = torch.empty_like(q)
    ws = z.decode_paged_workspace(cache, table, B=1, Hq=Hkv, Hkv=Hkv)

    def attended(which):
        length, _ = z.zipvl_paged_append(K, V, cache, table, start, length=torch.empty_like(start))
        for u in range(Hkv):
            if which[u]:
                assert torch.equal(cache.K[int(table[u, 0])], K[0, u]) and torch.equal(cache.V[int(table[u, 0])], V[0, u])
        for kw in (dict(o=o, ws=ws), {}):
            got = z.zipvl_decode_attn_paged(q, cache, table, length, 0.125, B=1, Hq=Hkv, Hkv=Hkv, **kw)
            for u in range(Hkv):
                k, v = (x[0, u].cpu() if which[u] else x[0, u, :0].cpu() for x in (K, V))
                ref, bound = attention(q[u:u + 1].cpu(), k, v, 0.125)
                size = torch.softmax(q[u:u + 1].cpu().double() @ k.double().T * 0.125, dim=1) @ v.double().abs() if which[u] else torch.zeros_like(ref)
                assert_attention(got[u:u + 1], ref, bound, size)

    small = cache.K, cache.V
    attended([False, True])
    cache.K, cache.V = (torch.zeros((9, page, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    attended([True, True])
    cache.K, cache.V = small
    attended([False, True])
    cache.V = torch.zeros((9, page, d), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(z.ZipvlError, match="V has shape"):
        attended([False, True])


@pytest.mark.gpu
def test_rows_of_expanded_and_single_axes():
    """Inputs whose axes have stride 0, or one element and torch's own idea of its stride, are taken as they are."""
    d, page = 64, 16
    rope = z.Rope(frequencies(32))
    one = torch.randn((1, 1, 6, d), generator=torch.Generator().manual_seed(71)).to(DEV)
    wide = one.expand(3, 4, 6, d)
    pos = positions(1, 3, 6, 72)
    Qo, _ = z.zipvl_rotate(wide, None, pos, rope)
    assert torch.equal(Qo, z.zipvl_rotate(wide.contiguous(), None, pos, rope)[0])
    with pytest.raises(z.ZipvlError, match="overlap"):
        z.zipvl_rotate(wide, None, pos, rope, Qo=wide)
    odd = torch.randn((2, 7, d), generator=torch.Generator().manual_seed(73)).to(DEV)[:, 3:4].unsqueeze(1)       # [2,1,1,d]
    odd = odd.as_strided(odd.shape, (odd.stride(0), 5, 3, 1), odd.storage_offset())
    pos = positions(1, 2, 1, 74)
    assert torch.equal(z.zipvl_rotate(odd, None, pos, rope)[0], z.zipvl_rotate(odd.contiguous(), None, pos, rope)[0])
    cache, table = pools(4, page, d, "f32", 75), torch.arange(2, dtype=torch.int32, device=DEV).view(2, 1)
    length, _ = z.zipvl_paged_append(odd, odd, cache, table, torch.zeros((2,), dtype=torch.int32, device=DEV))
    assert length.tolist() == [1, 1] and torch.equal(cache.V[:2, 0], odd[:, 0, 0])


# ---------------------------------------------------------------- refusals, without a GPU
@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(z.library_path()):
        from paper_2410_08584_amd.build import build_library
        build_library(verbose=False)
    return z.load_library()


FAKE = C.c_void_p(0x1000)          # aligned, never dereferenced: every call below is rejected first
ODD = C.c_void_p(0x1002)


def dims(B=2, Hq=8, Hkv=2, n=10, d=64, dtype=1, q=None, k=None, v=None):
    dm = z.dims_of(None, None, None, B=B, Hq=Hq, Hkv=Hkv, n=n, d=d, dtype=dtype)
    for name, given, H in (("q_strides", q, Hq), ("k_strides", k, Hkv), ("v_strides", v, Hkv)):
        setattr(dm, name, (C.c_int64 * 3)(*(given or (H * n * d, n * d, d))))
    return dm


def rope_with(**fields):
    r = z.Rope(frequencies(32))
    for name, v in fields.items():
        if name in ("freq", "axis"):
            getattr(r, name)[3] = v
        else:
            setattr(r, name, v)
    return r


def test_rotate_refuses(lib):
    def call(dm=None, Q=FAKE, K=FAKE, pos=FAKE, rope=None, flags=0, Qo=FAKE, Ko=FAKE, out=None, no_rope=False):
        return lib.zipvl_rotate(Q, K, C.byref(dm or dims()), pos, None if no_rope else C.byref(rope or z.Rope(frequencies(32))), flags, Qo, Ko,
                                C.byref(out) if out is not None else None, None)
    assert call(dims(d=96)) == -2 and call(dims(dtype=2)) == -5 and call(dims(n=0)) == -1
    assert call(dims(B=3000, n=1 << 20, Hq=2, Hkv=1)) == -2 and "2^30" in z.zipvl_last_error()
    assert call(Q=None, K=None, Qo=None, Ko=None) == -1
    assert call(Q=None) == -1 and call(Ko=None) == -1
    assert call(pos=None) == -1 and call(pos=ODD) == -3 and call(Q=ODD) == -3 and call(Ko=ODD) == -3
    assert call(flags=2) == -5
    assert call(no_rope=True) == -1
    assert call(rope=rope_with(axes=0)) == -1 and call(rope=rope_with(axes=5)) == -1
    assert call(rope=rope_with(pairs=12)) == -2 and call(rope=rope_with(pairs=40)) == -2 and call(rope=rope_with(pairs=0)) == -2
    assert call(rope=rope_with(layout=2)) == -5 and call(rope=rope_with(reserved=1)) == -5
    assert call(rope=rope_with(freq=7.0)) == -1 and call(rope=rope_with(freq=math.nan)) == -1 and call(rope=rope_with(axis=1)) == -1
    assert call(dims(q=(8 * 10 * 64, 10 * 64, 66))) == -3
    assert call(out=dims(q=(8 * 10 * 64, 0, 64))) == -1 and "overlap" in z.zipvl_last_error()
    assert call(out=dims(k=(64, 64, 128))) == -1 and "overlap" in z.zipvl_last_error()
    assert call(Q=FAKE, Qo=FAKE, K=None, Ko=None, out=dims(q=(8 * 20 * 64, 20 * 64, 128))) == -1 and "in the place" in z.zipvl_last_error()


def test_paged_append_refuses(lib):
    def call(dm=None, K=FAKE, V=FAKE, idx=None, k=None, pos=FAKE, rope=True, pages=None, table=FAKE, width=4, start=FAKE, length=FAKE, Q=None, Qo=None, flags=0):
        r = z.Rope(frequencies(32)) if rope is True else rope
        return lib.zipvl_paged_append(K, V, C.byref(dm or dims()), idx, k, pos, None if r is None else C.byref(r), C.byref(pages or z.Pages(0x1000, 0x1000, 9, 16)),
                                      table, width, start, length, Q, Qo, flags, None)
    assert call(dims(d=32)) == -2 and call(dims(v=(0, 64, 8))) == -1
    assert call(K=None) == -1 and call(V=ODD) == -3
    assert call(pages=z.Pages(0, 0x1000, 9, 16)) == -1 and call(pages=z.Pages(0x1008, 0x1000, 9, 16)) == -3
    assert call(pages=z.Pages(0x1000, 0x1000, 0, 16)) == -1
    for page in (0, 8, 24, 48, 512, -16):
        assert call(pages=z.Pages(0x1000, 0x1000, 9, page)) == -2
    assert call(table=None) == -1 and call(table=ODD) == -3 and call(width=0) == -1 and call(width=(1 << 20) + 1) == -2
    assert call(start=None) == -1 and call(length=None) == -1 and call(start=ODD) == -3 and call(length=ODD) == -3
    assert call(pos=None) == -1 and call(rope=rope_with(pairs=4)) == -2
    assert call(idx=FAKE) == -1 and "without k" in z.zipvl_last_error()
    assert call(k=ODD) == -3
    assert call(Q=FAKE) == -1 and call(Qo=FAKE) == -1
    assert call(Q=FAKE, Qo=FAKE, idx=FAKE, k=FAKE) == -5
    assert call(Q=FAKE, Qo=FAKE, rope=None) == -1
    assert call(dims(q=(8 * 20 * 64, 20 * 64, 128)), Q=FAKE, Qo=FAKE) == -1 and "in the place" in z.zipvl_last_error()
    assert call(flags=1) == -5


def test_paged_append_refuses_lengths_in_the_place_of_other_inputs(lib):
    at = lambda i, off=0: C.c_void_p(0x100000 * i + off)                # arrays a mebibyte apart; B Hkv = 4 units of 10 tokens, tables of 4 pages

    def call(length, rope=True, flags=0):
        r = z.Rope(frequencies(32))
        return lib.zipvl_paged_append(at(1), at(2), C.byref(dims()), at(3), at(4), at(5), C.byref(r) if rope else None,
                                      C.byref(z.Pages(0x1000, 0x1000, 9, 16)), at(6), 4, at(7), length, None, None, flags, None)
    for length in (at(3), at(3, 156), at(4), at(4, 12), at(4, -12), at(5), at(5, 76), at(6, 60), at(7, 4), at(7, -12)):
        assert call(length) == -1 and "overlaps" in z.zipvl_last_error()


def test_decode_attn_paged_refuses(lib):
    def call(dm=None, q=FAKE, pages=None, table=FAKE, width=4, length=FAKE, ptable=FAKE, pwidth=4, plen=FAKE, begin=FAKE, groups=1, scale=0.1, o=FAKE,
             ws=FAKE, ws_bytes=1 << 40):
        return lib.zipvl_decode_attn_paged(q, C.byref(pages or z.Pages(0x1000, 0x1000, 9, 16)), table, width, length, ptable, pwidth, plen, begin, groups,
                                           C.byref(dm or dims()), C.c_float(scale), o, ws, ws_bytes, None)
    assert call(dims(d=96)) == -2 and call(dims(Hq=33, Hkv=1)) == -2 and "query heads" in z.zipvl_last_error()
    assert call(q=None) == -1 and call(o=ODD) == -3 and call(length=None) == -1 and call(length=ODD) == -3
    assert call(table=None) == -1 and call(width=0) == -1 and call(ptable=None) == -1 and call(pwidth=0) == -1
    assert call(plen=None) == -1 and call(begin=None) == -1 and call(begin=ODD) == -3
    assert call(groups=-1) == -1 and call(groups=3) == -1
    assert call(pages=z.Pages(0x1000, 0x1000, 9, 20)) == -2
    big = z.Pages(0x1000, 0x1000, 9, 256)
    assert call(pages=big, width=65537) == -2 and call(pages=big, pwidth=65537) == -2 and "2^24" in z.zipvl_last_error()
    assert call(dims(B=256, Hq=8, Hkv=8), pages=big, width=65536, groups=0) == -2 and "2^35" in z.zipvl_last_error()
    assert call(dims(B=256, Hq=64, Hkv=8), pages=big, pwidth=65536, groups=48) == -2 and "2^35" in z.zipvl_last_error()
    for scale in (0.0, -1.0, math.nan, math.inf):
        assert call(scale=scale) == -1
    assert call(ws=None) == -4 and call(ws_bytes=1) == -4 and "workspace" in z.zipvl_last_error()
    assert call(ws=C.c_void_p(0x1008)) == -3
    assert z.workspace_bytes(z.OP_DECODE_PAGED, dims(), -1) == 0 and z.workspace_bytes(z.OP_DECODE_PAGED, dims(), 4096) > 0


def test_binding_refuses_what_does_not_fit():
    x = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype)
    i = lambda *shape: torch.zeros(shape, dtype=torch.int32)
    rope = z.Rope(frequencies(32))

    def refused(call, text):
        with pytest.raises(z.ZipvlError, match=text):
            call()
    refused(lambda: z.Rope([]), "frequencies")
    refused(lambda: z.Rope([1.0] * 65), "frequencies")
    refused(lambda: z.Rope([1.0] * 8, [0] * 7), "axes")
    refused(lambda: z.Rope([1.0] * 8, [4] * 8), "axes")
    refused(lambda: z.zipvl_rotate(None, None, i(1, 2, 5), rope), "None")
    refused(lambda: z.zipvl_rotate(x(2, 4, 5, 64), None, i(1, 2, 6), rope), "pos")
    refused(lambda: z.zipvl_rotate(x(2, 4, 5, 64), None, i(1, 2, 5).long(), rope), "pos")
    refused(lambda: z.zipvl_rotate(x(2, 4, 5, 64), x(2, 2, 6, 64), i(1, 2, 5), rope), "K")
    refused(lambda: z.zipvl_rotate(x(2, 4, 5, 64), None, i(1, 2, 5), rope, Qo=x(2, 4, 5, 128)), "Qo")
    refused(lambda: z.zipvl_rotate(x(2, 4, 5, 64, dtype=torch.float16), None, i(1, 2, 5), rope), "dtype")
    refused(lambda: z.zipvl_rotate(x(2, 4, 64, 5).transpose(2, 3), None, i(1, 2, 5), rope), "contiguous")
    refused(lambda: z.zipvl_rotate(x(2, 4, 5, 64), None, i(1, 2, 5), rope), "one GPU")
    refused(lambda: z.PagedCache(x(3, 16, 64), x(3, 16, 128)), "shape")
    refused(lambda: z.PagedCache(x(3, 16, 64), x(3, 16, 64, dtype=torch.bfloat16)), "expected")
    refused(lambda: z.PagedCache(x(48, 64), x(48, 64)), "pages")
    cache = z.PagedCache(x(9, 16, 64), x(9, 16, 64))
    K = x(2, 2, 5, 64)
    refused(lambda: z.zipvl_paged_append(K, x(2, 2, 4, 64), cache, i(4, 2), i(4)), "V")
    refused(lambda: z.zipvl_paged_append(x(2, 2, 5, 128), x(2, 2, 5, 128), cache, i(4, 2), i(4)), "pages")
    refused(lambda: z.zipvl_paged_append(K, K, cache, i(3, 2), i(4)), "table")
    refused(lambda: z.zipvl_paged_append(K, K, cache, i(4, 2), i(3)), "start")
    refused(lambda: z.zipvl_paged_append(K, K, cache, i(4, 2), i(4), length=i(5)), "length")
    refused(lambda: z.zipvl_paged_append(K, K, cache, i(4, 2), i(4), k=i(2)), "k has")
    refused(lambda: z.zipvl_paged_append(K, K, cache, i(4, 2), i(4), k=i(4), flags=z.T_PER_BATCH), "k has")
    refused(lambda: z.zipvl_paged_append(K, K, cache, i(4, 2), i(4), k=i(4), idx=i(4, 4)), "idx")
    refused(lambda: z.zipvl_paged_append(K, K, cache, i(4, 2), i(4), rope=rope), "pos")
    refused(lambda: z.zipvl_paged_append(K, K, cache, i(4, 2), i(4), rope=rope, pos=i(1, 2, 4)), "pos")
    refused(lambda: z.zipvl_paged_append(K, K, cache, i(4, 2), i(4), rope=rope, pos=i(1, 2, 5), Q=x(2, 4, 6, 64)), "Q")
    refused(lambda: z.zipvl_paged_append(K, K, cache, i(4, 2), i(4), rope=rope, pos=i(1, 2, 5), Q=x(2, 4, 5, 64), Qo=x(2, 5, 4, 64).transpose(1, 2)), "contiguous")
    refused(lambda: z.zipvl_paged_append(K, K, cache, i(4, 2), i(4)), "one GPU")
    attend = lambda q=None, table=None, length=None, **kw: z.zipvl_decode_attn_paged(x(8, 64) if q is None else q, cache, i(4, 2) if table is None else table,
                                                                                    i(4) if length is None else length, 0.1, B=2, Hq=4, Hkv=2, **kw)
    refused(lambda: attend(q=x(7, 64)), "q has")
    refused(lambda: attend(q=x(8, 64, dtype=torch.bfloat16)), "q has")
    refused(lambda: attend(table=i(5, 2)), "table")
    refused(lambda: attend(length=i(2)), "length")
    refused(lambda: attend(prefix_table=i(2, 3)), "all be")
    refused(lambda: attend(prefix_table=i(2, 3), prefix_len=i(2), group_begin=i(3)), "prefix_table")
    refused(lambda: attend(prefix_table=i(4, 3), prefix_len=i(2), group_begin=i(3)), "prefix_len")
    refused(lambda: attend(), "one GPU")


def test_pages_are_counted_as_they_are():
    x = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype)
    cache = z.PagedCache(x(4, 16, 64), x(4, 16, 64))
    cache.K, cache.V = x(9, 32, 128), x(9, 32, 128)
    pages = cache.struct()
    assert (pages.K, pages.V, pages.num_pages, pages.page) == (cache.K.data_ptr(), cache.V.data_ptr(), 9, 32)
    assert (cache.num_pages, cache.page, cache.d) == (9, 32, 128)
    for V, text in ((x(4, 32, 128), "shape"), (x(9, 32, 128, dtype=torch.bfloat16), "expected"), (x(9, 32, 256)[..., ::2], "contiguous")):
        cache.V = V
        with pytest.raises(z.ZipvlError, match=text):
            cache.struct()
        i = torch.zeros((4, 1), dtype=torch.int32)
        with pytest.raises(z.ZipvlError, match=text):
            z.zipvl_decode_attn_paged(x(8, 128), cache, i, i[:, 0].contiguous(), 0.1, B=2, Hq=4, Hkv=2)
        with pytest.raises(z.ZipvlError, match=text):
            z.zipvl_paged_append(x(2, 2, 5, 128), x(2, 2, 5, 128), cache, i, i[:, 0].contiguous())


def test_a_workspace_with_gaps_is_refused():
    x = lambda *shape: torch.zeros(shape)
    cache, i = z.PagedCache(x(4, 16, 64), x(4, 16, 64)), torch.zeros((4, 1), dtype=torch.int32)
    for ws in (torch.zeros((1 << 27,), dtype=torch.uint8)[::2], torch.zeros((1,), dtype=torch.uint8).expand(1 << 27)):
        with pytest.raises(z.ZipvlError, match="contiguous"):
            z.zipvl_decode_attn_paged(x(8, 64), cache, i, i[:, 0].contiguous(), 0.1, B=2, Hq=4, Hkv=2, o=x(8, 64), ws=ws)


def test_workspaces_of_decode_over_pages_go_by_the_tables(lib):
    size = lambda rows, prefix, **kw: z.workspace_bytes(z.OP_DECODE_PAGED, dims(n=rows, **kw), prefix)
    for kw in (dict(B=1, Hq=1, Hkv=1, d=128, dtype=1), dict(B=1, Hq=1, Hkv=1, d=64, dtype=0)):
        assert 0 < size(16, 0, **kw) <= size(16, 16, **kw) < 1 << 20
    for kw in (dict(), dict(B=64, Hq=32, Hkv=8, d=128), dict(B=40, Hq=32, Hkv=1, d=64, dtype=0)):
        sizes = [size(rows, prefix, **kw) for rows in (16, 100, 3000, 1 << 24) for prefix in (0, 16, 5000, 1 << 24)]
        assert all(sizes[4 * r + p] <= sizes[4 * r + p + 1] for r in range(4) for p in range(3)) and all(a <= b for a, b in zip(sizes, sizes[4:]))
        assert sizes[-1] < 140 << 20
