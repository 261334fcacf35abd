"""Rotary positions, pages in 8 bits and the attention over them, against plain forms in 64 bits.

Bounds, derived before their first run.  u: unit roundoff of the 16-bit type (2^-8 for bfloat16, 2^-11 for half).
Rotation: the angle is exact to 2^-32 turns and rounded to 24 bits (2^-24 of half a turn at most), sine and cosine are
within 2^-22, products and their sum add 3 * 2^-24: together below 2^-20 s (|a| + |b|), then one rounding, u |x|, or
2^-25 among half's subnormals.  An 8-bit number is the nearest one: 2^-4 of the value, or 2^-10 of the block's power
among subnormals.  What is not rotated is a 16-bit number divided by a power of two: its 8-bit number is decided
exactly.  Attention: the bounds of the 16-bit attention tests hold for the numbers that the pages stand for, since these are
numbers of the 16-bit type; weights of half are held to 2^-11 down to 2^-29 of the largest in either kernel.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytestmark = [pytest.mark.gpu, pytest.mark.skip(reason="needs a CUDA GPU")]
else:
    pytestmark = pytest.mark.gpu

DEV = torch.device("cuda", 0)
BF, HF, E4 = torch.bfloat16, torch.float16, torch.float8_e4m3fn
RANGE = {BF: (-100, 120), HF: (-15, 8)}


@pytest.fixture(scope="module")
def P():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_19677_gb300 as P
    return P


@pytest.fixture(scope="module")
def ctx(P):
    c = P.Context(0)
    yield c
    c.close()


def ints(a):
    return torch.tensor([int(x) for x in a], dtype=torch.int32, device=DEV)


def cum(lens):
    return ints(np.concatenate([[0], np.cumsum(lens)]))


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def randn(g, *shape, dtype=BF, spread=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * spread).to(dtype)


def unit(dtype):
    return 2.0 ** -8 if dtype == BF else 2.0 ** -11


def fails(P, ctx, code, call):
    call()
    with pytest.raises(P.CacheRouteError) as e:
        ctx.sync()
    assert e.value.code == code


# ---- rotary positions ----------------------------------------------------------------------------------------------
def turned(x, pos, rot, back=False):
    """x [T, h, d] and positions (any integers) in 64 bits: the rotated tokens and the bound of a 32-bit rotation."""
    y, b, r = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64, device=DEV), rot.dims
    p = torch.as_tensor(pos, device=DEV).double()
    for i, f in enumerate(rot.frequencies):
        angle = torch.remainder(p * f, 2 * math.pi) * (-1 if back else 1)
        c, s = (torch.cos(angle) * rot.scale)[:, None], (torch.sin(angle) * rot.scale)[:, None]
        m, n = (i, i + r // 2) if rot.layout == "half" else (2 * i, 2 * i + 1)
        u, v = x[..., m].double(), x[..., n].double()
        y[..., m], y[..., n] = u * c - v * s, v * c + u * s
        # the reference's own angle: a product of 53 bits
        b[..., m] = b[..., n] = (u.abs() + v.abs()) * abs(rot.scale) * (2.0 ** -20 + (p.abs() * abs(f)).max().item() * 2.0 ** -51)
    return y, b


ROPE = [
    # dtype, heads, dim, rotated, layout, tokens, scaling
    (BF, 32, 128, 128, "half", 1, {}),
    (HF, 1, 64, 64, "interleaved", 3, {}),
    (BF, 5, 128, 64, "half", 37, dict(scaling="linear", factor=8.0)),
    (HF, 28, 128, 32, "interleaved", 16, dict(scaling="ramp", factor=16.0, original=4096)),
    (BF, 3, 80, 80, "half", 17, dict(scaling="ntk", factor=4.0)),
    (HF, 2, 72, 40, "half", 50, {}),
    (BF, 9, 8, 8, "interleaved", 33, {}),
    (HF, 4, 96, 8, "half", 65, dict(scale=-1.5)),
    (BF, 2, 64, 48, "half", 2000, dict(base=500000.0)),
]


@pytest.mark.parametrize("dtype,h,d,r,layout,T,how", ROPE)
def test_rope(P, ctx, dtype, h, d, r, layout, T, how):
    g = gen(T + d)
    rot = P.Rotary(r, layout=layout, **how)
    x = randn(g, T, h + 3, d, dtype=dtype)[:, 1:h + 1]
    pos = torch.randint(0, 1 << 20, (T,), generator=g, device=DEV, dtype=torch.int32)
    pos[0] = 0 if T > 1 else 77
    out = P.rope(ctx, x, rot, pos)
    ctx.sync()
    want, off = turned(x, pos, rot)
    assert ((out.double() - want).abs() <= unit(dtype) * want.abs() * 1.01 + off * 1.01 + 2.0 ** -25).all()
    assert torch.equal(out[..., r:], x[..., r:])
    if T > 1:
        assert rot.scale != 1.0 or torch.equal(out[0], x[0])
    # in place, by head, and the other way round
    by_head = x.transpose(0, 1).contiguous().transpose(0, 1)
    assert P.rope(ctx, by_head, rot, pos, out=by_head) is by_head
    ctx.sync()
    assert torch.equal(by_head, out)


def test_rope_far_and_negative_positions(P, ctx):
    """The angle is exact however far: where position times frequency has 31 bits before the point and the check as well."""
    rot = P.Rotary(16, frequencies=[1.0, 0.7, 3.0, 1e-3, 2.0 ** -8, 0.1, 6.5, 5e-8])
    pos = [0, 1, -1, 2 ** 31 - 1, -2 ** 31, 123456789, -5, 2 ** 24 + 1]
    x = randn(gen(1), len(pos), 2, 16)
    out = P.rope(ctx, x, rot, ints(pos))
    ctx.sync()
    import fractions
    want = x.double().clone()
    # pi to 70 digits, so that whole turns are dropped exactly
    two_pi = 2 * fractions.Fraction(31415926535897932384626433832795028841971693993751058209749445923078164, 10 ** 70)
    for t, p in enumerate(pos):
        for i, f in enumerate(rot.frequencies):
            a = fractions.Fraction(f) * p
            a = float(a - (a // two_pi) * two_pi)
            u, v = float(x[t, 0, i]), float(x[t, 0, i + 8])
            want[t, 0, i], want[t, 0, i + 8] = u * math.cos(a) - v * math.sin(a), v * math.cos(a) + u * math.sin(a)
    # the share of a turn is a double: 2^-53 of f p / 2 pi turns more
    far = torch.tensor([abs(p) * 2.0 ** -52 for p in pos], dtype=torch.float64, device=DEV)[:, None] * 6.5
    size = x[:, 0].double().abs()
    size = (size[:, :8] + size[:, 8:]).repeat(1, 2)
    assert ((out[:, 0].double() - want[:, 0]).abs() <= 2.0 ** -8 * want[:, 0].abs() * 1.01 + size * (2.0 ** -20 + far)).all()


def test_rope_of_nothing_and_what_is_no_number(P, ctx):
    rot = P.Rotary(32, layout="half")
    empty = torch.zeros((0, 4, 64), dtype=BF, device=DEV)
    assert P.rope(ctx, empty, rot, ints([])).shape == (0, 4, 64)
    x = randn(gen(2), 4, 2, 64)
    x[1, 0, 3], x[2, 1, 40] = math.nan, math.inf
    out = P.rope(ctx, x, rot, ints([5, 6, 7, 8]))
    ctx.sync()
    bad = ~torch.isfinite(out)
    want = torch.zeros_like(bad)
    want[1, 0, 3] = want[1, 0, 19] = want[2, 1, 40] = True
    assert torch.equal(bad, want)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_inverse_is_the_gradient(P, ctx, layout):
    """Against the formula's gradient, and against differences of the rotation (it is linear: whole steps will do)."""
    g = gen(3)
    rot = P.Rotary(64, layout=layout, scale=1.25)
    x, w, step = (randn(g, 40, 3, 96, dtype=HF) for _ in range(3))
    pos = ints(range(1000, 1040))
    x.requires_grad_(False)
    got = P.rope(ctx, w, rot.inverse(), pos)
    ctx.sync()
    want, off = turned(w, pos, rot, back=True)
    assert ((got.double() - want).abs() <= 2.0 ** -11 * want.abs() * 1.01 + off + 2.0 ** -25).all()
    a, b = P.rope(ctx, x, rot, pos), P.rope(ctx, (x + step).to(HF), rot, pos)
    ctx.sync()
    moved = ((x + step).to(HF).double() - x.double())
    ahead = ((b.double() - a.double()) * w.double()).sum()
    gradient = (got.double() * moved).sum()
    # every output is rounded once, by 2^-11 of itself, and off by 2^-20 of its pair
    slack = ((a.double().abs() + b.double().abs()) * 2.0 ** -10 * w.double().abs()).sum() + (got.double().abs() * 2.0 ** -10 * moved.abs()).sum()
    assert (ahead - gradient).abs() <= slack
    assert slack < 0.05 * (got.double().abs() * moved.abs()).sum()


def test_rope_refuses(P, ctx):
    rot = P.Rotary(64)
    x, pos = randn(gen(4), 4, 2, 64), ints(range(4))
    for call in (lambda: P.rope(ctx, x.float(), rot, pos), lambda: P.rope(ctx, x, rot, pos[:3]),
                 lambda: P.rope(ctx, x, rot, pos.long()), lambda: P.rope(ctx, x[0], rot, pos),
                 lambda: P.rope(ctx, x, rot, pos, out=x[:, :1]), lambda: P.rope(ctx, x.transpose(1, 2), rot, pos),
                 lambda: P.rope(ctx, x.clone().requires_grad_(), rot, pos)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: P.rope(ctx, x[..., :56], rot, pos),                       # fewer elements than are rotated
                 lambda: P.rope(ctx, randn(gen(4), 4, 2, 136)[..., :132], rot, pos),
                 lambda: P.rope(ctx, randn(gen(4), 4, 2, 68)[..., 4:], rot, pos),  # not aligned
                 lambda: P.rope(ctx, x, rot, pos, out=x.as_strided(x.shape, (64, 256, 1)))):  # in place, other strides
        with pytest.raises(P.CacheRouteError) as e:
            call()
        assert e.value.code == P.CR_EINVAL
    ctx.sync()


# ---- pages in 8 bits -----------------------------------------------------------------------------------------------
def two(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def power(top, dtype):
    """The smallest 2^e with 448 2^e >= top, in 64 bits."""
    lo, hi = RANGE[dtype]
    e = torch.log2(top / 448.0).clamp(lo, hi).floor()
    return two(torch.where(top > 448.0 * two(e), e + 1, e).clamp(lo, hi))


def nearest(y):
    """Nearest e4m3 numbers of |y| <= 448, ties to even."""
    step = (y.abs().clamp_min(2.0 ** -6).view(torch.int64) >> 52 << 52).view(torch.float64) / 8
    return torch.round(y / step) * step


def numbers(x, s, dtype):
    """8-bit numbers of x (64 bits) in units of s."""
    most = torch.where(s >= 2.0 ** RANGE[dtype][1], 240.0, 448.0)
    y = nearest(torch.minimum(torch.maximum(x / s, -most), most))
    return torch.where(torch.isfinite(x.to(dtype)), y, math.nan)


class Held:
    """Rows of a pool in 64 bits, written a call at a time: numbers [2, tokens, heads, dim], powers [2, blocks, heads]."""

    def __init__(self, block, heads, d, dtype):
        self.B, self.dtype = block, dtype
        self.num = torch.zeros((2, 0, heads, d), dtype=torch.float64, device=DEV)
        self.pow = torch.zeros((2, 0, heads), dtype=torch.float64, device=DEV)

    def write(self, x):
        """x [2, m, heads, d] in 64 bits."""
        B, n0, m = self.B, self.num.shape[1], x.shape[1]
        self.num = torch.cat([self.num, torch.zeros_like(x)], 1)
        blocks = -(-(n0 + m) // B)
        self.pow = torch.cat([self.pow, torch.zeros((2, blocks - self.pow.shape[1], x.shape[2]), dtype=torch.float64, device=DEV)], 1)
        at = n0
        while at < n0 + m:
            b, end = at // B, min(n0 + m, (at // B + 1) * B)
            mine = x[:, at - n0:end - n0]
            s = power(torch.where(torch.isfinite(mine.to(self.dtype)), mine, 0.0).abs().amax((1, 3)), self.dtype)
            if at % B:
                s = torch.maximum(s, self.pow[:, b])
                self.num[:, b * B:at] = nearest(self.num[:, b * B:at] * (self.pow[:, b] / s)[:, None, :, None])
            self.pow[:, b] = s
            self.num[:, at:end] = numbers(mine, s[:, None, :, None], self.dtype)
            at = end

    def fork(self, keep):
        h = Held(self.B, self.num.shape[2], self.num.shape[3], self.dtype)
        h.num, h.pow = self.num[:, :keep].clone(), self.pow[:, :-(-keep // self.B)].clone()
        return h

    def values(self):
        return self.num * self.pow.repeat_interleave(self.B, 1)[:, :self.num.shape[1], :, None]


def pool8(P, page, block, n_pages, n_seqs, width, layers, heads, d, dtype, order="token"):
    """An empty pool whose places hold not-a-number, numbers and scales alike."""
    shape = (layers, 2, n_pages, page, heads, d) if order == "token" else (layers, 2, n_pages, heads, page, d)
    cache = torch.full(shape, 0x7f, dtype=torch.uint8, device=DEV).view(E4)
    if order != "token":
        cache = cache.transpose(3, 4)
    z = P.KVPages.empty(n_pages, page, n_seqs, width, 1, 1, 16)
    scale = torch.full((layers, 2, n_pages, heads, page // block), math.nan, device=DEV)
    return P.KVPages(cache, z.ref, z.table, z.lens, scale=scale, dtype=dtype)


def row_of(pg, layer, row):
    """Numbers [2, tokens, heads, d] and powers [2, blocks, heads] of a row, in 64 bits."""
    n = int(pg.lens[row])
    used = pg.table[row, :-(-n // pg.page)].long().cpu()
    num = torch.stack([torch.cat([pg.cache[layer, c, int(p)].view(torch.uint8).contiguous().view(E4).double() for p in used])
                       for c in range(2)])[:, :n]
    pw = torch.stack([torch.cat([pg.scale[layer, c, int(p)].T.double() for p in used]) for c in range(2)])
    return num, pw[:, :-(-n // pg.block)]


def same(a, b):
    return a.shape == b.shape and bool(((a == b) | (a.isnan() & b.isnan())).all())


def assert_holds(pg, layer, row, held):
    num, pw = row_of(pg, layer, row)
    assert same(pw, held.pow), f"row {row}: powers"
    assert same(num, held.num), f"row {row}: numbers"


WRITE = [
    # dtype, page, block, heads, dim, order, calls of (row, tokens)
    (BF, 16, 16, 2, 128, "token", [[(0, 1)], [(0, 1), (1, 40)], [(0, 30), (1, 1)]]),
    (HF, 8, 8, 1, 16, "head", [[(2, 3), (0, 17)], [(0, 1)] , [(2, 5), (0, 6)]]),
    (BF, 64, 16, 3, 64, "head", [[(0, 100), (1, 1), (2, 64)], [(1, 7), (0, 3)], [(1, 8), (2, 65), (0, 1)]]),
    (HF, 64, 64, 8, 128, "token", [[(0, 63)], [(0, 1)], [(0, 1), (1, 200)]]),
    (BF, 256, 256, 1, 80, "token", [[(0, 300), (1, 5)], [(1, 250), (0, 1)], [(1, 1)]]),
    (HF, 32, 8, 5, 96, "token", [[(0, 9), (1, 8), (2, 7)], [(2, 1), (0, 7), (1, 24)]]),
    (BF, 128, 32, 12, 48, "head", [[(0, 31)], [(0, 1)], [(0, 1)], [(0, 100)]]),
]


@pytest.mark.parametrize("dtype,page,block,heads,d,order,calls", WRITE)
def test_write_holds_the_nearest_numbers(P, ctx, dtype, page, block, heads, d, order, calls):
    """Calls that begin and end inside blocks, magnitudes that grow and shrink from call to call: bit for bit."""
    g = gen(page + d)
    pg = pool8(P, page, block, 40, 3, 8, 2, heads, d, dtype, order)
    rows = [Held(block, heads, d, dtype) for _ in range(3)]
    for n, call in enumerate(calls):
        seqs, new = [r for r, _ in call], [m for _, m in call]
        T = sum(new)
        P.pages_extend(ctx, pg, ints(seqs), ints(new))
        kv = randn(g, T, 2 * heads + 1, d, dtype=dtype, spread=[1.0, 30.0, 0.02, 300.0][n])
        kv[:, :heads] *= 2.0 ** torch.arange(heads, device=DEV).to(dtype)[:, None]
        k, v = kv[:, :heads], kv[:, heads:2 * heads]
        P.kv_write(ctx, pg, 1, k, v, cum(new), seqs=ints(seqs))
        ctx.sync()
        at = 0
        for r, m in call:
            rows[r].write(torch.stack([k[at:at + m].double(), v[at:at + m].double()]))
            at += m
        for r in set(seqs):
            assert_holds(pg, 1, r, rows[r])
    assert bool((pg.cache[0].view(torch.uint8) == 0x7f).all()), "another layer"
    # what the rows stand for, back: exact
    lens = pg.lens.tolist()
    k, v = P.kv_read(ctx, pg, 1, cum(lens))
    ctx.sync()
    at = 0
    for r, n in enumerate(lens):
        assert same(k[at:at + n].double(), rows[r].values()[0]) and same(v[at:at + n].double(), rows[r].values()[1])
        at += n


@pytest.mark.parametrize("dtype", [BF, HF])
def test_write_at_the_edges_of_the_range(P, ctx, dtype):
    """Zeros, subnormal numbers, ties, the largest numbers, infinities and what is no number."""
    top = torch.finfo(dtype).max
    small = 2.0 ** -24 if dtype == HF else 2.0 ** -133
    x = torch.zeros((8, 6, 16), dtype=torch.float64)
    x[0, 1] = torch.linspace(-17, 17, 16).double() * small                    # e's lower end
    x[0, 2, :4] = torch.tensor([448.0, 17.0, 19.0, 232.0])                    # ties: 17 -> 16, 19 -> 20, 232 -> 224
    x[0, 3, :4] = torch.tensor([top, -top, top / 2, 1.0])
    x[1, 3, 5] = math.inf
    x[0, 4, :5] = torch.tensor([math.nan, math.inf, -math.inf, 1.0, -3.0])
    x[0, 5, :3] = torch.tensor([449.0 if dtype == HF else 450.0, 448.0, 2.0 ** -9])   # the next power
    x = x.to(dtype).to(DEV)
    pg = pool8(P, 8, 8, 4, 1, 2, 1, 6, 16, dtype)
    P.pages_extend(ctx, pg, ints([0]), ints([8]))
    P.kv_write(ctx, pg, 0, x, x, ints([0, 8]))
    held = Held(8, 6, 16, dtype)
    held.write(torch.stack([x.double(), x.double()]))
    ctx.sync()
    assert_holds(pg, 0, 0, held)
    k, _ = P.kv_read(ctx, pg, 0, ints([0, 8]))
    ctx.sync()
    fine = torch.isfinite(x)
    assert torch.equal(torch.isfinite(k), fine) and bool(k[~fine].isnan().all())
    s = held.pow[0].repeat_interleave(8, 0)[:, :, None]
    assert ((k.double() - x.double()).abs()[fine] <= torch.maximum(2.0 ** -4 * x.double().abs(), 2.0 ** -10 * s.expand(x.shape))[fine]).all()


def test_a_page_that_is_used_again_begins_anew(P, ctx):
    """Powers are those of the tokens that stand there now, not of an earlier row's."""
    g = gen(9)
    pg = pool8(P, 16, 8, 3, 2, 3, 1, 2, 32, BF)
    for spread in (1000.0, 0.001):
        P.pages_extend(ctx, pg, ints([0]), ints([40]))
        k, v = randn(g, 40, 2, 32, spread=spread), randn(g, 40, 2, 32, spread=spread)
        P.kv_write(ctx, pg, 0, k, v, ints([0, 40]))
        held = Held(8, 2, 32, BF)
        held.write(torch.stack([k.double(), v.double()]))
        ctx.sync()
        assert_holds(pg, 0, 0, held)
        P.pages_free(ctx, pg, ints([0]))


APPEND = [
    # dtype, bits, page, block, query heads, key heads, dim, rotated, layout, cached, new
    (BF, 8, 16, 16, 8, 2, 128, 128, "half", [0, 100, 15, 16], [1, 1, 1, 1]),
    (HF, 8, 64, 32, 28, 4, 128, 64, "interleaved", [0, 31, 500], [200, 2, 90]),
    (BF, 8, 8, 8, 7, 1, 64, 32, "half", [3, 0], [30, 1]),
    (HF, 8, 128, 128, 6, 3, 80, 80, "half", [0, 127, 5], [129, 1, 60]),
    (BF, 16, 16, 0, 8, 2, 128, 128, "half", [0, 100, 15], [1, 50, 17]),
    (HF, 16, 8, 0, 5, 5, 72, 40, "interleaved", [7, 0], [9, 1]),
    (BF, 16, 256, 0, 0, 3, 64, 64, "half", [0, 255], [70, 2]),
]


@pytest.mark.parametrize("dtype,bits,page,block,hq,hkv,d,r,layout,cached,new", APPEND)
def test_append_rotates_and_writes(P, ctx, dtype, bits, page, block, hq, hkv, d, r, layout, cached, new):
    g = gen(d + page)
    n, T = len(new), sum(new)
    rot = P.Rotary(r, layout=layout, scaling="ramp", factor=4.0, original=2048)
    rows = [3 * i + 1 for i in range(n)][::-1]
    if bits == 8:
        pg = pool8(P, page, block, 200, 3 * n, 80, 1, hkv, d, dtype)
    else:
        pg = P.KVPages.empty(200, page, 3 * n, 80, 1, hkv, d, dtype=dtype)
    old = [c for c in cached if c]
    P.pages_extend(ctx, pg, ints(r_ for r_, c in zip(rows, cached) if c), ints(old))
    kv = randn(g, sum(old), 2 * hkv, d, dtype=dtype, spread=0.3)
    P.kv_write(ctx, pg, 0, kv[:, :hkv], kv[:, hkv:], cum(old), seqs=ints(r_ for r_, c in zip(rows, cached) if c))
    ctx.sync()
    before = {r_: row_of(pg, 0, r_) for r_, c in zip(rows, cached) if c} if bits == 8 else None
    P.pages_extend(ctx, pg, ints(rows), ints(new))
    qkv = randn(g, T, hq + 2 * hkv, d, dtype=dtype)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    cu = np.concatenate([[0], np.cumsum(new)])
    out = P.kv_append(ctx, pg, 0, q if hq else None, k, v, rot, ints(cu), seqs=ints(rows))
    back = P.kv_read(ctx, pg, 0, ints(cu), seqs=ints(rows))
    ctx.sync()
    pos = np.concatenate([np.arange(c, c + m) for c, m in zip(cached, new)])
    u = unit(dtype)
    if hq:
        want, off = turned(q, pos, rot)
        assert ((out.double() - want).abs() <= u * want.abs() * 1.01 + off * 1.01 + 2.0 ** -25).all()
    else:
        assert out is None
    want, off = turned(k, pos, rot)
    if bits == 16:
        assert ((back[0].double() - want).abs() <= u * want.abs() * 1.01 + off * 1.01 + 2.0 ** -25).all()
        assert torch.equal(back[1], v)
        return
    for i, row in enumerate(rows):
        a, b, c = cu[i], cu[i + 1], cached[i]
        held = Held(block, hkv, d, dtype)
        if c:
            held.num, held.pow = (x.clone() for x in before[row])
        held.write(torch.stack([want[a:b], v[a:b].double()]))
        num, pw = row_of(pg, 0, row)
        assert same(pw[1], held.pow[1]) and same(num[1], held.num[1]), "values are not rotated: exact"
        # keys: the power may be the other one where the largest magnitude is within the rotation's error of 448 2^e
        first = c // block
        assert same(pw[0][:first], held.pow[0][:first])
        top = torch.stack([want[max(a, a + j * block - c):min(b, a + (j + 1) * block - c)].abs().amax((0, 2))
                           for j in range(first, -(-(c + b - a) // block))])
        slack = off[a:b].max() * 2
        lo, hi = power((top - slack).clamp_min(0), dtype), power(top + slack, dtype)
        if c % block:
            lo[0], hi[0] = torch.maximum(lo[0], before[row][1][0, first]), torch.maximum(hi[0], before[row][1][0, first])
        assert ((pw[0][first:] >= lo) & (pw[0][first:] <= hi)).all()
        s = pw[0].repeat_interleave(block, 0)[:num.shape[1]][:, :, None]
        got = num[0] * s
        assert ((got[c:] - want[a:b]).abs() <= torch.maximum(2.0 ** -4 * want[a:b].abs(), 2.0 ** -10 * s[c:]) + off[a:b] * 1.01).all()
        if c:  # tokens that were there, rounded again at most once
            was = (before[row][0] * before[row][1].repeat_interleave(block, 1)[:, :c, :, None])[0]
            assert ((got[:c] - was).abs() <= 2.0 ** -10 * s[:c]).all()


def test_append_in_place_and_a_token_at_a_time(P, ctx):
    """A row that grows token by token holds what 64 bits hold; queries may be rotated where they are."""
    g = gen(12)
    rot = P.Rotary(64)
    pg = pool8(P, 16, 16, 8, 1, 4, 1, 2, 64, HF)
    held = Held(16, 2, 64, HF)
    one = P.Rotary(64, frequencies=[0.0] * 32)     # turns nothing: exact
    for t in range(50):
        P.pages_extend(ctx, pg, ints([0]), ints([1]))
        k, v, q = (randn(g, 1, 2, 64, dtype=HF, spread=1.2 ** t * 0.01) for _ in range(3))
        was = q.clone()
        assert P.kv_append(ctx, pg, 0, q, k, v, one, ints([0, 1]), out=q) is q
        held.write(torch.stack([k.double(), v.double()]))
        ctx.sync()
        assert torch.equal(q, was)
        assert_holds(pg, 0, 0, held)
    q = randn(g, 1, 4, 64, dtype=HF)
    a = P.kv_append(ctx, pg, 0, q, k, v, rot, ints([0, 1]))
    b = P.rope(ctx, q, rot, ints([49]))
    ctx.sync()
    assert torch.equal(a, b)


def test_fork_and_compact_take_scales_along(P, ctx):
    g = gen(13)
    page, block = 32, 8
    pg = pool8(P, page, block, 40, 6, 6, 3, 2, 48, BF)
    P.pages_extend(ctx, pg, ints([4, 0]), ints([70, 90]))
    kv = randn(g, 3, 2, 160, 2, 48)
    kv[:, :, 30:60] *= 50
    rows = {0: [Held(block, 2, 48, BF) for _ in range(3)], 4: [Held(block, 2, 48, BF) for _ in range(3)]}
    for l in range(3):
        P.kv_write(ctx, pg, l, kv[l, 0], kv[l, 1], ints([0, 70, 160]), seqs=ints([4, 0]))
        rows[4][l].write(kv[l, :, :70].double())
        rows[0][l].write(kv[l, :, 70:].double())
    P.pages_fork(ctx, pg, ints([0, 0, 4]), ints([1, 2, 3]), ints([41, 64, 1]))
    for d, s, n in ((1, 0, 41), (2, 0, 64), (3, 4, 1)):
        rows[d] = [h.fork(n) for h in rows[s]]
    P.pages_free(ctx, pg, ints([4]))
    P.pages_extend(ctx, pg, ints([1, 2, 3]), ints([5, 1, 9]))
    more = randn(g, 3, 2, 15, 2, 48, spread=100.0)
    for l in range(3):
        P.kv_write(ctx, pg, l, more[l, 0], more[l, 1], ints([0, 5, 6, 15]), seqs=ints([1, 2, 3]))
        for d, a, b in ((1, 0, 5), (2, 5, 6), (3, 6, 15)):
            rows[d][l].write(more[l, :, a:b].double())
    ctx.sync()
    for r in (0, 1, 2, 3):
        for l in range(3):
            assert_holds(pg, l, r, rows[r][l])
    ref, table, _, live = P.pages_compact(ctx, pg)
    pg.replace(ref, table)
    ctx.sync()
    assert int(live) == int((pg.ref > 0).sum()) and bool((pg.ref[:int(live)] > 0).all())
    for r in (0, 1, 2, 3):
        for l in range(3):
            assert_holds(pg, l, r, rows[r][l])


@pytest.mark.parametrize("bits", [8, 16])
def test_read_any_part_of_rows(P, ctx, bits):
    g = gen(14)
    pg = P.KVPages.empty(30, 16, 4, 8, 2, 3, 64, dtype=HF, bits=bits, **({"block": 8} if bits == 8 else {}))
    lens = [50, 0, 17, 128]
    P.pages_extend(ctx, pg, ints(range(4)), ints(lens))
    k, v = randn(g, sum(lens), 3, 64, dtype=HF), randn(g, sum(lens), 3, 64, dtype=HF)
    P.kv_write(ctx, pg, 1, k, v, cum(lens))
    ka, va = P.kv_read(ctx, pg, 1, cum(lens))
    wide = torch.full((2, 40, 4, 72), 7.0, dtype=HF, device=DEV)
    got = P.kv_read(ctx, pg, 1, ints([0, 1, 1, 30, 40]), seqs=ints([3, 0, 0, 3]), start=ints([127, 5, 21, 0]),
                    out=(wide[0, :, :3, :64], wide[1, :, :3, :64]))
    ctx.sync()
    if bits == 16:
        assert torch.equal(ka, k) and torch.equal(va, v)
    at = np.concatenate([[0], np.cumsum(lens)])
    for x, y in ((got[0], ka), (got[1], va)):
        assert torch.equal(x[0], y[at[3] + 127]) and torch.equal(x[1:30], y[21:50]) and torch.equal(x[30:], y[at[3]:at[3] + 10])
    assert bool((wide[:, :, 3] == 7.0).all()) and bool((wide[..., 64:] == 7.0).all())
    # past a row's end, before its beginning, of a row that does not exist: zeros
    k2 = torch.full((6, 3, 64), 7.0, dtype=HF, device=DEV)
    v2 = k2.clone()
    fails(P, ctx, P.CR_EINVAL, lambda: P.kv_read(ctx, pg, 1, ints([0, 2, 4, 5, 6]), seqs=ints([2, 0, 9, -1]), start=ints([16, -1, 0, 0]),
                                                 out=(k2, v2)))
    assert torch.equal(k2[0], ka[66]) and torch.equal(k2[3], ka[0]) and torch.equal(v2[3], va[0])
    for i in (1, 2, 4, 5):
        assert bool((k2[i] == 0).all()) and bool((v2[i] == 0).all())


@pytest.mark.parametrize("n", [3, 1500])
@pytest.mark.parametrize("bits", [8, 16])
def test_a_row_named_twice_is_written_once(P, ctx, n, bits):
    """Short lists are looked through, long ones marked; the first entry of a row writes, queries turn in every one."""
    g, r = gen(15), np.random.default_rng(n)
    pg = P.KVPages.empty(n, 8, n, 1, 1, 1, 16, dtype=HF, bits=bits)
    P.pages_extend(ctx, pg, ints(range(n)), ints([1] * n))
    seqs = r.permutation(n)
    seqs[n // 2:] = seqs[r.integers(0, n // 2, n - n // 2)]
    k, v, q = (randn(g, n, 1, 16, dtype=HF) for _ in range(3))
    rot = P.Rotary(16, scale=2.0)
    out = []
    fails(P, ctx, P.CR_EINVAL, lambda: out.append(P.kv_append(ctx, pg, 0, q, k, v, rot, ints(range(n + 1)), seqs=ints(seqs))))
    first = {}
    for i, s in enumerate(seqs):
        first.setdefault(int(s), i)
    rows = ints(first)
    got, gv = P.kv_read(ctx, pg, 0, ints(range(len(first) + 1)), seqs=rows)
    ctx.sync()
    i = torch.tensor(list(first.values()), device=DEV)
    tol = 2.0 ** -4 if bits == 8 else 0.0
    assert ((gv - v[i]).abs().double() <= v[i].abs().double() * tol + (2.0 ** -9 if bits == 8 else 0)).all()
    assert ((got - 2 * k[i]).abs().double() <= k[i].abs().double() * 2 * tol + (2.0 ** -9 if bits == 8 else 0)).all()
    assert torch.equal(out[0], 2 * q)      # position 0


def test_writes_that_go_nowhere(P, ctx):
    """Rows that do not exist or are too short, and pages that others share: skipped, reported, nothing else touched."""
    g = gen(16)
    pg = pool8(P, 16, 16, 12, 4, 2, 1, 2, 64, BF)
    P.pages_extend(ctx, pg, ints([0]), ints([20]))
    k, v, q = (randn(g, 20, 2, 64) for _ in range(3))
    rot = P.Rotary(64)
    P.kv_write(ctx, pg, 0, k, v, ints([0, 20]), seqs=ints([0]))
    P.pages_fork(ctx, pg, ints([0]), ints([1]), ints([16]))
    ctx.sync()
    was, scale = pg.cache.view(torch.uint8).clone(), pg.scale.clone()
    out = []
    fails(P, ctx, P.CR_EINVAL, lambda: out.append(P.kv_append(ctx, pg, 0, q[:3], k[:3], v[:3], rot, ints([0, 1, 2, 3]), seqs=ints([7, -1, 1]))))
    assert torch.equal(pg.cache.view(torch.uint8), was) and torch.equal(pg.scale.nan_to_num(-1), scale.nan_to_num(-1))
    want = P.rope(ctx, q[2:3], rot, ints([15]))       # a page that is shared: its token's position is known
    ctx.sync()
    assert bool((out[0][:2] == 0).all()) and torch.equal(out[0][2:], want)
    # more tokens than the row has: those before it go nowhere, the others are written
    P.pages_extend(ctx, pg, ints([2]), ints([3]))
    out.clear()
    fails(P, ctx, P.CR_EINVAL, lambda: out.append(P.kv_append(ctx, pg, 0, q[:19], k[:19], v[:19], rot, ints([0, 19]), seqs=ints([2]))))
    want = P.rope(ctx, q[16:19], rot, ints([0, 1, 2]))
    _, gv = P.kv_read(ctx, pg, 0, ints([0, 3]), seqs=ints([2]))
    ctx.sync()
    assert bool((out[0][:16] == 0).all()) and torch.equal(out[0][16:], want)
    assert ((gv - v[16:19]).abs().double() <= 2.0 ** -4 * v[16:19].abs().double() + 2.0 ** -9).all()


def test_cache8_refuses(P, ctx):
    pg = pool8(P, 16, 16, 4, 2, 2, 1, 2, 64, BF)
    z = P.KVPages.empty(4, 16, 2, 2, 1, 2, 64)
    g = gen(17)
    k, cu, rot = randn(g, 2, 2, 64), ints([0, 2]), P.Rotary(64)
    for call in (lambda: P.KVPages(pg.cache, pg.ref, pg.table, pg.lens),
                 lambda: P.KVPages(z.cache, z.ref, z.table, z.lens, scale=pg.scale),
                 lambda: P.KVPages(z.cache, z.ref, z.table, z.lens, dtype=HF),
                 lambda: P.KVPages(pg.cache, pg.ref, pg.table, pg.lens, scale=pg.scale[:, :1]),
                 lambda: P.KVPages(pg.cache, pg.ref, pg.table, pg.lens, scale=pg.scale.double()),
                 lambda: P.KVPages(pg.cache, pg.ref, pg.table, pg.lens, scale=pg.scale, dtype=E4),
                 lambda: P.kv_write(ctx, pg, 0, k.half(), k.half(), cu), lambda: P.kv_write(ctx, pg, 0, k.to(E4), k.to(E4), cu),
                 lambda: P.kv_append(ctx, pg, 0, k, k, k, rot, cu, seqs=ints([0, 1])),
                 lambda: P.kv_append(ctx, pg, 0, k[:1], k, k, rot, cu), lambda: P.kv_append(ctx, pg, 0, None, k, k, rot, cu, out=k),
                 lambda: P.kv_append(ctx, pg, 0, k, k.clone().requires_grad_(), k, rot, cu),
                 lambda: P.kv_read(ctx, pg, 0, cu, out=(k.half(), k.half())), lambda: P.kv_read(ctx, pg, 0, cu, tokens=3, out=(k, k)),
                 lambda: P.kv_read(ctx, pg, 0, cu, start=ints([0, 0])),
                 lambda: P.attn_decode(ctx, k.half(), pg, 0), lambda: P.attn_paged(ctx, k.float(), pg, 0, cu)):
        with pytest.raises(ValueError):
            call()
    odd = torch.zeros((1, 2, 4, 16, 2, 24), dtype=torch.uint8, device=DEV).view(E4)   # 24 elements: not a multiple of 16
    bad = [P.KVPages(odd, pg.ref, pg.table, pg.lens, scale=pg.scale)]
    many = torch.ones((1, 2, 4, 2, 4), device=DEV)                                     # blocks of four tokens
    bad.append(P.KVPages(pg.cache, pg.ref, pg.table, pg.lens, scale=many))
    for b in bad:
        with pytest.raises(P.CacheRouteError) as e:
            P.pages_free(ctx, b, ints([0]))
        assert e.value.code == P.CR_EINVAL
    for call in (lambda: P.kv_append(ctx, pg, 1, k, k, k, rot, cu), lambda: P.kv_read(ctx, pg, 1, cu),
                 lambda: P.kv_append(ctx, pg, 0, k, k, k, P.Rotary(128), cu),
                 lambda: P.kv_append(ctx, pg, 0, randn(g, 2, 2, 68)[..., 4:], k, k, rot, cu)):
        with pytest.raises(P.CacheRouteError) as e:
            call()
        assert e.value.code == P.CR_EINVAL
    ctx.sync()
    # nothing to do
    none = torch.zeros((0, 2, 64), dtype=BF, device=DEV)
    P.kv_append(ctx, pg, 0, none, none, none, rot, ints([0, 0]))
    assert P.kv_read(ctx, pg, 0, ints([0, 0]))[0].shape == (0, 2, 64)
    ctx.sync()


# ---- attention over 8 bits -----------------------------------------------------------------------------------------
def reference(q, k, v, causal, scale):
    """One sequence: q [m, hq, d], k, v [n, hkv, d] in 64 bits -> (o, lse, bounds of both)."""
    m, hq, d = q.shape
    n, hkv, _ = k.shape
    u = unit(q.dtype)
    half = q.dtype != BF
    q, k, v = q.double(), k.repeat_interleave(hq // hkv, 1), v.repeat_interleave(hq // hkv, 1)
    if n == 0:
        z = torch.zeros((m, hq, d), dtype=torch.float64, device=DEV)
        return z, torch.full((m, hq), -math.inf, dtype=torch.float64, device=DEV), z + 1e-30, torch.zeros((m, hq), device=DEV)
    s = torch.einsum("ihd,jhd->hij", q, k) * scale
    e = torch.einsum("ihd,jhd->hij", q.abs(), k.abs()) * scale * 2.0 ** -18
    if causal:
        hidden = torch.arange(n, device=DEV)[None, :] > torch.arange(m, device=DEV)[:, None] + (n - m)
        s.masked_fill_(hidden, -math.inf)
        e.masked_fill_(hidden, 0.0)
    e = e.amax(-1)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[..., None])
    o = torch.einsum("hij,jhd->ihd", p, v)
    a = torch.einsum("hij,jhd->ihd", p, v.abs())
    e = e.T[:, :, None]
    bound = u * (o.abs() + a) * 1.01 + (4 * e + 2.0 ** -19) * a
    if half:
        bound = bound + n * 2.0 ** -25 * v.abs().amax()
    return o, lse.T, bound + 1e-30, (e[..., 0] * 2 + 2.0 ** -20 * lse.T.abs() + 2.0 ** -18).nan_to_num(0.0, posinf=0.0)


def check(out, lse, parts, cu):
    for b, (o, l, bo, bl) in enumerate(parts):
        got, gl = out[cu[b]:cu[b + 1]].double(), lse[cu[b]:cu[b + 1]].double()
        assert torch.isfinite(got).all(), f"sequence {b}"
        worst = ((got - o).abs() / bo).amax().item() if o.numel() else 0.0
        assert worst <= 1.0, f"sequence {b}: {worst} of the bound"
        none = l == -math.inf
        assert (gl[none] == -math.inf).all() and torch.isfinite(gl[~none]).all()
        assert ((gl - l).abs()[~none] <= bl[~none]).all(), f"sequence {b}: lse"


def fill8(P, ctx, g, page, block, lens, heads, d, dtype, layers=1, order="token", shared=None, group=None, spread=None,
          width=0):
    """Rows in a pool whose other places hold not-a-number; rows of a group share its first shared[group] tokens
    (whole pages).  Returns the pages and the (k, v) that each row stands for, in 64 bits."""
    r = np.random.default_rng(page + sum(lens))
    need = [-(-n // page) for n in lens]
    total = sum(need) + 5
    pg = pool8(P, page, block, total, len(lens), max(need + [1, width]) + 1, layers, heads, d, dtype, order)
    order_of = r.permutation(total)
    table, at, first = np.full(tuple(pg.table.shape), -1, np.int64), 0, {}
    begin = [0] * len(lens)
    for i, n in enumerate(lens):
        s = 0
        if group is not None and group[i] in first:
            s = shared[group[i]] // page
            table[i, :s] = table[first[group[i]], :s]
        elif group is not None:
            first[group[i]] = i
        begin[i] = s * page
        table[i, s:need[i]] = order_of[at:at + need[i] - s]
        at += need[i] - s
    pg.table.copy_(ints(table.reshape(-1)).view(pg.table.shape))
    pg.lens.copy_(ints(lens))
    own = [n - b for n, b in zip(lens, begin)]
    T = sum(own)
    k, v = randn(g, T, heads, d, dtype=dtype, spread=2.0), randn(g, T, heads, d, dtype=dtype)
    if spread is not None:
        k, v = spread(k, v)
    P.kv_write(ctx, pg, layers - 1, k, v, cum(own))     # pages count as nobody's: every row writes its own
    pg.ref.copy_(ints(np.bincount(table[table >= 0], minlength=total)))
    ctx.sync()
    out = []
    for i, n in enumerate(lens):
        if n == 0:
            out.append(tuple(torch.zeros((2, 0, heads, d), dtype=torch.float64, device=DEV)))
            continue
        num, pw = row_of(pg, layers - 1, i)
        x = num * pw.repeat_interleave(block, 1)[:, :n, :, None]
        out.append((x[0], x[1]))
    return pg, out


DECODE = [
    # page, block, key heads, query heads, dim, dtype, order, lengths
    (16, 16, 2, 8, 128, BF, "token", [1, 15, 16, 17, 63, 64, 65, 700]),
    (8, 8, 1, 7, 64, HF, "head", [2000, 3]),
    (64, 16, 4, 4, 128, HF, "token", [129, 0, 5]),
    (32, 8, 1, 16, 128, BF, "head", [333, 4000]),
    (256, 256, 2, 40, 64, BF, "token", [257, 1000]),
    (128, 64, 1, 128, 128, HF, "token", [500]),
    (16, 8, 3, 27, 80, BF, "token", [100, 31, 32]),
    (64, 64, 2, 12, 96, HF, "head", [64, 65, 1, 200]),
    (16, 16, 1, 3, 16, BF, "token", [50]),
    (32, 32, 8, 8, 48, HF, "token", list(range(0, 80, 2))),
]


@pytest.mark.parametrize("page,block,hkv,hq,d,dtype,order,lens", DECODE)
def test_decode8(P, ctx, page, block, hkv, hq, d, dtype, order, lens):
    g = gen(page * 7 + hq + d)
    pg, rows = fill8(P, ctx, g, page, block, lens, hkv, d, dtype, layers=2, order=order)
    q = randn(g, len(lens), hq + 1, d, dtype=dtype)[:, :hq]
    out, lse = P.attn_decode(ctx, q, pg, 1, lse=True)
    again = P.attn_decode(ctx, q, pg, 1)
    ctx.sync()
    n = len(lens)
    check(out, lse, [reference(q[i:i + 1], *rows[i], False, d ** -0.5) for i in range(n)], range(n + 1))
    assert torch.equal(out, again)


GROUPED = [
    # page, block, key heads, query heads, dim, dtype, shared tokens, members (own tokens)
    (16, 16, 2, 16, 128, BF, [160, 32], [[1, 5, 100], [17]]),
    (32, 8, 1, 7, 64, HF, [0, 640, 64], [[40, 3], [1, 2, 3, 4, 5, 6, 7, 8, 9, 10], [31, 64]]),
    (64, 32, 4, 32, 128, HF, [4096], [[20, 1, 70, 300]]),
    (8, 8, 1, 24, 80, BF, [200, 8, 16], [[5], [9, 9], [1, 1]]),
]


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("page,block,hkv,hq,d,dtype,shared,members", GROUPED)
def test_decode8_groups(P, ctx, page, block, hkv, hq, d, dtype, shared, members, wide):
    """Rows that can hold little read their prefixes themselves; of those that can hold more, a group's is read once."""
    g = gen(page + hq)
    group = [i for i, m in enumerate(members) for _ in m]
    lens = [shared[i] + n for i, m in enumerate(members) for n in m]
    pg, rows = fill8(P, ctx, g, page, block, lens, hkv, d, dtype, shared=shared, group=group,
                     width=8192 * 64 // (len(lens) * hkv * page) + 1 if wide else 0)
    q = randn(g, len(lens), hq, d, dtype=dtype)
    before = ctx.launches
    out, lse = P.attn_decode(ctx, q, pg, 0, group_off=cum([len(m) for m in members]), shared=ints(shared), lse=True)
    assert ctx.launches - before == (4 if wide else 2)
    alone, alse = P.attn_decode(ctx, q, pg, 0, lse=True)
    ctx.sync()
    n = len(lens)
    parts = [reference(q[i:i + 1], *rows[i], False, d ** -0.5) for i in range(n)]
    check(out, lse, parts, range(n + 1))
    check(alone, alse, parts, range(n + 1))


PAGED = [
    # page, block, key heads, query heads, dim, dtype, order, (cached, new) of each sequence
    (16, 16, 2, 8, 128, BF, "token", [(0, 1), (0, 128), (100, 28), (128, 64)]),
    (8, 8, 1, 7, 64, HF, "head", [(1000, 1), (3, 200)]),
    (32, 16, 4, 4, 128, HF, "token", [(300, 300), (31, 2), (0, 33)]),
    (64, 8, 2, 2, 96, BF, "head", [(129, 127)]),
    (128, 128, 1, 16, 128, BF, "token", [(700, 5), (128, 128), (0, 7)]),
    (256, 64, 2, 12, 64, HF, "head", [(600, 77), (255, 1)]),
    (64, 64, 1, 128, 80, BF, "token", [(70, 3), (0, 10)]),
    (16, 8, 4, 32, 128, BF, "token", [(5000, 64)]),
    (16, 16, 1, 1, 16, HF, "token", [(10, 300)]),
]


@pytest.mark.parametrize("page,block,hkv,hq,d,dtype,order,seqs", PAGED)
@pytest.mark.parametrize("causal", [True, False])
def test_paged8(P, ctx, page, block, hkv, hq, d, dtype, order, seqs, causal):
    g = gen(page + hq + d)
    lens, new = [a + b for a, b in seqs], [b for _, b in seqs]
    pg, rows = fill8(P, ctx, g, page, block, lens, hkv, d, dtype, order=order)
    q = randn(g, sum(new), hq, d, dtype=dtype)
    out, lse = P.attn_paged(ctx, q, pg, 0, cum(new), causal=causal, lse=True)
    again = P.attn_paged(ctx, q, pg, 0, cum(new), causal=causal)
    ctx.sync()
    cu = np.concatenate([[0], np.cumsum(new)])
    check(out, lse, [reference(q[a:b], *rows[i], causal, d ** -0.5) for i, (a, b) in enumerate(zip(cu, cu[1:]))], cu)
    assert torch.equal(out, again)


def test_attention8_rows_without_keys(P, ctx):
    """More queries than keys, rows that are empty or do not exist: zeros and minus infinity."""
    g = gen(21)
    pg, rows = fill8(P, ctx, g, 16, 16, [5, 0, 40], 2, 64, BF)
    q = randn(g, 300, 4, 64)
    out, lse = P.attn_paged(ctx, q, pg, 0, ints([0, 200, 250, 300]), lse=True)
    ctx.sync()
    check(out, lse, [reference(q[a:b], *r, True, 64 ** -0.5) for r, a, b in zip(rows, (0, 200, 250), (200, 250, 300))], [0, 200, 250, 300])
    assert bool((out[:195] == 0).all()) and bool((lse[:195] == -math.inf).all())
    out = []
    fails(P, ctx, P.CR_EINVAL, lambda: out.extend(P.attn_decode(ctx, q[:3], pg, 0, seqs=ints([2, 9, -1]), lse=True)))
    o, lse = out
    check(o[:1], lse[:1], [reference(q[:1], *rows[2], False, 64 ** -0.5)], [0, 1])
    assert bool((o[1:] == 0).all()) and bool((lse[1:] == -math.inf).all())


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("hq", [2, 16])
def test_attention8_over_blocks_of_very_different_size(P, ctx, dtype, hq):
    """Values' powers that differ by 2^18 from block to block, keys' that make some blocks' scores vanish and others
    decide; queries from 2^-20 to 2^20; a sink whose values are zero.  Each row's error is bounded by its own weights' sum."""
    g = gen(22)
    n, d = 500, 64

    def spread(k, v):
        i = torch.arange(n, device=DEV) // 16
        k = (k * 2.0 ** (i % 5 - 3)[:, None, None]).to(dtype)
        v = (v.double() * 2.0 ** ((i * 7 % 19) - 14).double()[:, None, None]).to(dtype)
        v[:16] = 0
        return k, v

    pg, rows = fill8(P, ctx, g, 16, 16, [n], 1, d, dtype, spread=spread)
    q = randn(g, 1, hq, d, dtype=dtype, spread=0.5)
    if dtype == BF:
        q = (q.double() * 2.0 ** torch.linspace(-20, 3, hq, device=DEV).double()[None, :, None]).to(dtype)
    q[0, -1] *= 4
    out, lse = P.attn_decode(ctx, q, pg, 0, scale=0.25, lse=True)
    many = P.attn_paged(ctx, q, pg, 0, ints([0, 1]), scale=0.25)
    ctx.sync()
    o, l, bound, bl = reference(q, *rows[0], False, 0.25)
    check(out, lse, [(o, l, bound, bl)], [0, 1])
    # weights of the 128-row kernel are halves without the blocks' powers: a key may lose 2^-25 of its value
    check(many, lse, [(o, l, bound, bl)], [0, 1])


def test_attention8_what_is_no_number_reaches_who_sees_it(P, ctx):
    g = gen(23)

    def spread(k, v):
        v[300, 0, 5] = math.inf
        return k, v

    pg, rows = fill8(P, ctx, g, 16, 8, [290, 330], 1, 64, BF, spread=lambda k, v: spread(k, v))
    q = randn(g, 2, 4, 64)
    out = P.attn_decode(ctx, q, pg, 0)
    many = P.attn_paged(ctx, q, pg, 0, ints([0, 1, 2]))
    ctx.sync()
    for o in (out, many):    # token 10 of the second row
        assert torch.isfinite(o[0]).all() and o[1, :, 5].isnan().all() and torch.isfinite(o[1, :, 6:]).all()


# ---- together ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("bits", [8, 16])
def test_a_run_of_calls(P, ctx, bits):
    """Prefixes are appended, forked, extended, appended to, attended over and decoded from, as a destination does."""
    g, r = gen(31), np.random.default_rng(31)
    page, hq, hkv, d, dtype = 16, 8, 2, 128, BF
    rot = P.Rotary(d, scaling="linear", factor=2.0)
    pg = P.KVPages.empty(120, page, 12, 20, 2, hkv, d, dtype=dtype, bits=bits)
    text = {}
    u = 2.0 ** -8

    def step(rows, new, groups=None):
        T = sum(new)
        P.pages_extend(ctx, pg, ints(rows), ints(new))
        cu = cum(new)
        for layer in range(2):
            qkv = randn(g, T, hq + 2 * hkv, d, dtype=dtype)
            q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
            qr = P.kv_append(ctx, pg, layer, q, k, v, rot, cu, seqs=ints(rows))
            if groups is None:
                out, lse = P.attn_paged(ctx, qr, pg, layer, cu, seqs=ints(rows), lse=True)
            else:
                out, lse = P.attn_decode(ctx, qr, pg, layer, seqs=ints(rows), group_off=groups[0], shared=groups[1], lse=True)
            ctx.sync()
            parts, at = [], 0
            for row, m in zip(rows, new):
                n = int(pg.lens[row])
                kk, vv = (x.double() for x in P.kv_read(ctx, pg, layer, ints([0, n]), seqs=ints([row])))
                pos = np.arange(n - m, n)
                want, off = turned(k[at:at + m], pos, rot)
                old = text.setdefault((row, layer), [torch.zeros((0, hkv, d), dtype=torch.float64, device=DEV)] * 2)
                tk, tv = torch.cat([old[0], want]), torch.cat([old[1], v[at:at + m].double()])
                text[row, layer] = [tk, tv]
                # 448 2^e is at most twice the block's largest magnitude; a token is rounded anew as its block's power grows
                near = u if bits == 16 else 2.0 ** -4 * 1.01
                slack = 0 if bits == 16 else 2.0 ** -7
                assert ((kk - tk).abs() <= near * tk.abs() * 1.02 + slack + 2.0 ** -10).all()
                assert ((vv - tv).abs() <= (0 if bits == 16 else near) * tv.abs() + slack).all()
                parts.append(reference(qr[at:at + m], kk, vv, True, d ** -0.5))
                at += m
            check(out, lse, parts, np.concatenate([[0], np.cumsum(new)]))

    step([0, 1], [75, 40])
    P.pages_fork(ctx, pg, ints([0, 0, 1, 0]), ints([5, 6, 7, 8]), ints([75, 60, 33, 48]))
    for dst, src, keep in ((5, 0, 75), (6, 0, 60), (7, 1, 33), (8, 0, 48)):
        for layer in range(2):
            text[dst, layer] = [x[:keep] for x in text[src, layer]]
    step([7, 5, 8, 6], [3, 20, 1, 70])
    for _ in range(4):
        step([5, 6, 8, 7], [1, 1, 1, 1], (ints([0, 3, 4]), ints([48, 32])))
    P.pages_free(ctx, pg, ints([0, 6]))
    ref, table, _, _ = P.pages_compact(ctx, pg)
    pg.replace(ref, table)
    step([5, 8, 7], [1, 1, 1], (ints([0, 2, 3]), ints([48, 32])))


def test_captured_and_replayed(P):
    """A layer's calls in a graph, replayed with other inputs, beside eager calls of the same context in between."""
    g = gen(41)
    s = torch.cuda.Stream()
    here, ctx = P.Context(0), P.Context(0, stream=s)
    rot = P.Rotary(64)
    pg, _ = fill8(P, here, g, 16, 16, [200, 33, 64], 2, 64, BF)
    here.close()
    pg.ref.copy_(ints((pg.ref > 0).int().tolist()))
    q, k, v = randn(g, 3, 8, 64), randn(g, 3, 2, 64), randn(g, 3, 2, 64)
    cu = ints(range(4))
    torch.cuda.synchronize()

    def layer():
        qr = P.kv_append(ctx, pg, 0, q, k, v, rot, cu)
        return qr, P.attn_decode(ctx, qr, pg, 0), P.attn_paged(ctx, qr, pg, 0, cu), *P.kv_read(ctx, pg, 0, cu, tokens=3)

    with torch.cuda.stream(s):
        layer()
        graph = torch.cuda.CUDAGraph()
        ctx.sync()
        with torch.cuda.graph(graph, stream=s):
            got = layer()
        for i in range(3):
            for x in (q, k, v):
                x.copy_(randn(g, *x.shape, spread=1.0 + i))
            start = [t.clone() for t in (pg.cache.view(torch.uint8), pg.scale)]
            graph.replay()
            first = [x.clone() for x in got]
            pg.cache.view(torch.uint8).copy_(start[0])
            pg.scale.copy_(start[1])
            again = layer()
            ctx.sync()
            s.synchronize()
            for a, b in zip(first, again):
                assert torch.equal(a, b)
    ctx.close()


def test_on_a_stream_that_is_not_the_current_one(P):
    g = gen(42)
    s = torch.cuda.Stream()
    here, there = P.Context(0), P.Context(0, stream=s)
    rot = P.Rotary(64)
    pg, _ = fill8(P, here, g, 16, 16, [200, 33], 2, 64, HF)
    x = randn(g, 2, 4, 64, dtype=HF)
    pos, cu = ints([3, 4]), ints([0, 1, 2])
    want = (P.rope(here, x, rot, pos), *P.kv_read(here, pg, 0, cu, tokens=2), P.attn_decode(here, x, pg, 0), P.attn_paged(here, x, pg, 0, cu))
    here.sync()
    torch.cuda.synchronize()
    got = (P.rope(there, x, rot, pos), *P.kv_read(there, pg, 0, cu, tokens=2), P.attn_decode(there, x, pg, 0), P.attn_paged(there, x, pg, 0, cu))
    there.sync()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    here.close()
    there.close()


def test_write8_refuses_what_is_not_aligned(P, ctx):
    """Through the C entry, which no check of tensors stands before."""
    pg = P.KVPages.empty(4, 16, 1, 4, 1, 2, 64, dtype=BF, device=DEV, bits=8)
    k, cu = torch.zeros(2, 3, 2, 64, dtype=BF, device=DEV), ints([0, 1])
    before = pg.cache.view(torch.uint8).clone()
    for bump, token, head in ((2, 128, 64), (8, 128, 64), (0, 130, 64), (0, 128, 65)):
        for bad_v in (False, True):
            good = (k[0].data_ptr(), 128, 64)
            bad = (k[0].data_ptr() + bump, token, head)
            first, second = (good, bad) if bad_v else (bad, good)
            st = P.lib().cr_kv_write(ctx._h, pg._addr, 0, *first, *second, cu.data_ptr(), None, 1, 1)
            with pytest.raises(Exception, match="aligned"):
                ctx.check(st, "cr_kv_write")
    torch.cuda.synchronize()
    assert torch.equal(pg.cache.view(torch.uint8), before)


def test_rotary_of_another_device_is_refused(P, ctx):
    x, pos = torch.zeros(1, 2, 64, dtype=BF, device=DEV), ints([0])
    rot = P.Rotary(64, device="cpu")
    with pytest.raises(ValueError, match="frequencies are on cpu"):
        P.rope(ctx, x, rot, pos)
    with pytest.raises(ValueError, match="frequencies are on cpu"):
        P.rope(ctx, x, rot.inverse(), pos)
    pg = P.KVPages.empty(4, 16, 1, 4, 1, 2, 64, dtype=BF, device=DEV, bits=8)
    with pytest.raises(ValueError, match="frequencies are on cpu"):
        P.kv_append(ctx, pg, 0, None, x, x, rot, ints([0, 1]))


def test_offsets_past_32_bits(P, ctx):
    """Pages whose numbers begin past 2^32 bytes of the cache."""
    g = gen(43)
    page, heads, d = 64, 8, 128
    n_pages = (1 << 32) // (page * heads * d) + 40
    cache = torch.zeros((1, 2, n_pages, page, heads, d), dtype=torch.uint8, device=DEV).view(E4)
    z = P.KVPages.empty(n_pages, page, 2, 8, 1, 1, 16)
    scale = torch.ones((1, 2, n_pages, heads, 4), device=DEV)
    pg = P.KVPages(cache, z.ref, z.table, z.lens, scale=scale, dtype=BF)
    pg.ref[:n_pages - 20] = 1
    n = 300
    P.pages_extend(ctx, pg, ints([1]), ints([n]))
    k, v, q = randn(g, n, heads, d), randn(g, n, heads, d), randn(g, n, heads, d)
    qr = P.kv_append(ctx, pg, 0, q, k, v, P.Rotary(d), ints([0, n]), seqs=ints([1]))
    out, lse = P.attn_paged(ctx, qr, pg, 0, ints([0, n]), seqs=ints([1]), lse=True)
    one, olse = P.attn_decode(ctx, qr[-1:], pg, 0, seqs=ints([1]), lse=True)
    ctx.sync()
    assert int(pg.table[1, 0]) == n_pages - 20
    num, pw = row_of(pg, 0, 1)
    x = num * pw.repeat_interleave(16, 1)[:, :n, :, None]
    assert ((x[1] - v.double()).abs() <= 2.0 ** -4 * v.double().abs() + 2.0 ** -9).all()
    check(out, lse, [reference(qr, x[0], x[1], True, d ** -0.5)], [0, n])
    check(one, olse, [reference(qr[-1:], x[0], x[1], False, d ** -0.5)], [0, 1])


# ---- the server ----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("rotary", [True, False])
def test_destination(P, ctx, bits, rotary):
    """A server's passes layer by layer: the attention of every pass against 64 bits over what its rows stand for."""
    from examples.serve_prefixes import TinyAttention
    from paper_2608_19677_gb300.destination import Destination
    rot = P.Rotary(64, layout="half", scaling="linear", factor=2.0) if rotary else None

    class Watched(TinyAttention):
        def qkv(self, layer, x):
            q, k, v = super().qkv(layer, x)
            self.q = q
            return q, k, v

        def mix(self, layer, x, out):
            ctx.sync()
            at = 0
            for row, m in self.rows():
                n = int(pages.lens[row])
                kk, vv = (t.double() for t in P.kv_read(ctx, pages, layer, ints([0, n]), seqs=ints([row])))
                q = self.q[at:at + m]
                if rot is not None:
                    q = turned(q, np.arange(n - m, n), rot)[0].to(BF)
                o, _, bound, _ = reference(q, kk, vv, True, 64 ** -0.5)
                # the 64-bit rotation may round a query to the neighbour of the 32-bit one: 2^-8 of what it multiplies
                s = torch.einsum("ihd,jhd->hij", q.double().abs(), kk.abs().repeat_interleave(4, 1)).amax((1, 2))
                slack = 2.0 ** -16 * s[None, :, None] * vv.abs().amax() if rot is not None else 0
                assert ((out[at:at + m].double() - o).abs() <= bound + slack).all(), (layer, row)
                at += m
            assert at == out.shape[0]
            return super().mix(layer, x, out)

    model = Watched(torch, DEV, rotary=rot)
    pages = P.KVPages.empty(200, 16, 12, 12, model.layers, model.kv_heads, model.dim, bits=bits)
    d = Destination(ctx, pages, model)
    g = gen(51)
    text = lambda n: torch.randint(0, 4096, (n,), generator=g, device=DEV)  # noqa: E731
    prefix = {1: text(100), 2: text(33)}
    asked = [(1, torch.cat([prefix[1], text(5)]), 100), (2, torch.cat([prefix[2][:30], text(40)]), 30),
             (1, torch.cat([prefix[1][:64], text(1)]), 64)]
    passes = iter([lambda: [(d.prefixes[1][0], 100), (d.prefixes[2][0], 30)], lambda: list(zip(d.order_of_call, [5, 40, 1]))])
    now = [next(passes)]
    model.rows = lambda: now[0]()
    forward = d._forward

    def watched(tokens, cu, rows, groups=None):
        d.order_of_call = rows.tolist()
        x = forward(tokens, cu, rows, groups)
        now[0] = next(passes, lambda: [(r, 1) for r in d.order()])
        return x

    d._forward = watched
    d.admit(asked)
    for _ in range(3):
        d.step(text(3))
    live = d.compact()
    d.step(text(3))
    ctx.sync()
    assert int(live) == int((pages.ref > 0).sum())
    # a prefix moves: the other destination holds the same numbers
    other = P.KVPages.empty(50, 16, 4, 12, model.layers, model.kv_heads, model.dim, bits=bits)
    e = Destination(ctx, other, TinyAttention(torch, DEV, rotary=rot))
    kv = d.export(1)
    e.install(1, kv)
    for (k, v), (k2, v2) in zip(kv, e.export(1)):
        assert torch.equal(k, k2) and torch.equal(v, v2)
    _, mine = e.admit([(1, torch.cat([prefix[1][:80], prefix[2][:9]]), 80)])
    now[0] = lambda: [(d.order_of_call[0], 9)]
    _, same_here = d.admit([(1, torch.cat([prefix[1][:80], prefix[2][:9]]), 80)])
    ctx.sync()
    assert torch.equal(mine, same_here)


@pytest.mark.parametrize("rotary,bits", [(True, 16), (True, 8), (False, 8)])
def test_example_runs(rotary, bits):
    """Against the model from scratch: 16 bits as without positions, 2^-9 sqrt(10) 2 (a rounding of the rotated queries and
    keys more: sqrt(12)); in 8 bits it runs and gives numbers."""
    import examples.serve_prefixes as m
    said = []
    worst = m.main(48, 3, log=said.append, rotary=rotary, bits=bits)
    assert len(said) == 2 and math.isfinite(worst)
    if bits == 16:
        assert worst < 2.0 ** -9 * math.sqrt(12) * 2
