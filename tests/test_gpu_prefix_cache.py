"""Pages of a destination's cache and the attention that reads them, against plain forms in 64 bits.

Bounds of the attention tests, derived before their first run.  With unit roundoff u of the 16-bit type (2^-8 for
bfloat16, 2^-11 for half), the weights are rounded once (u relative each, so at most u * sum p|v| in a row) and the
output once (u |o|).  Scores are 32-bit sums of exact 16-bit products: error at most e = 2^-18 sum |q||k| scale, which
changes a weight, and the sum it is divided by, by a factor within 1 +- 2e; the exponential adds 2^-21.  Half has no
weights below 2^-24: each key of a row may lose 2^-25 of its value beside the largest weight of 1.
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
BF, HF = torch.bfloat16, torch.float16


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
    return torch.tensor(list(a), dtype=torch.int32, device=DEV)


def cum(lens):
    return ints(np.concatenate([[0], np.cumsum(lens)]))


def randn(g, *shape, dtype=BF, spread=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * spread).to(dtype)


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def reference(q, k, v, causal, scale, first=0):
    """One sequence in 64 bits: q [m, hq, d], k, v [n, hkv, d] -> (o, lse, bound of |o' - o|, bound of |lse' - lse|)."""
    m, hq, d = q.shape
    n, hkv, _ = k.shape
    u = 2.0 ** -8 if q.dtype == BF else 2.0 ** -11
    q, k, v = q.double(), k.double().repeat_interleave(hq // hkv, 1), v.double().repeat_interleave(hq // hkv, 1)
    if n == 0:
        z = torch.zeros((m, hq, d), dtype=torch.float64, device=DEV)
        inf = torch.full((m, hq), -math.inf, dtype=torch.float64, device=DEV)
        return z, inf, z + 1e-30, torch.zeros_like(inf)
    s = torch.einsum("ihd,jhd->hij", q, k) * scale
    e = torch.einsum("ihd,jhd->hij", q.abs(), k.abs()) * scale * 2.0 ** -18
    if causal:
        i = torch.arange(m, device=DEV)[:, None] + (n - m)
        hidden = torch.arange(n, device=DEV)[None, :] > i
        s.masked_fill_(hidden, -math.inf)
        e.masked_fill_(hidden, 0.0)
    e = e.amax(-1)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[..., None])
    o = torch.einsum("hij,jhd->ihd", p, v)
    a = torch.einsum("hij,jhd->ihd", p, v.abs())
    e = e.T[:, :, None]
    bound = u * (o.abs() + a) * 1.01 + (4 * e + 2.0 ** -19) * a
    if q.dtype != BF:
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


# ---- packed --------------------------------------------------------------------------------------------------------
PACKED = [
    # dtype, query heads, key heads, dim, lengths
    (BF, 8, 8, 128, [1]),
    (BF, 8, 2, 128, [1, 2, 127, 128, 129]),
    (HF, 4, 1, 64, [300, 1, 0, 77]),
    (BF, 7, 1, 128, [255, 256, 257]),
    (HF, 6, 2, 128, [513, 64]),
    (BF, 16, 1, 64, [1000]),
    (HF, 5, 5, 96, [130, 40]),
    (BF, 3, 1, 8, [19, 200]),
    (BF, 128, 1, 128, [9, 33]),
    (HF, 2, 2, 72, [640]),
    (BF, 4, 4, 128, [1200, 3, 800]),
]


@pytest.mark.parametrize("dtype,hq,hkv,d,lens", PACKED)
@pytest.mark.parametrize("causal", [True, False])
def test_packed(P, ctx, dtype, hq, hkv, d, lens, causal):
    g = gen(len(lens) * 100 + hq + d)
    T = sum(lens)
    qkv = randn(g, T, hq + 2 * hkv, d, dtype=dtype)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    k.mul_(2.0)
    out, lse = P.attn_packed(ctx, q, k, v, cum(lens), causal=causal, lse=True)
    ctx.sync()
    cu = np.concatenate([[0], np.cumsum(lens)])
    check(out, lse, [reference(q[a:b], k[a:b], v[a:b], causal, d ** -0.5) for a, b in zip(cu[:-1], cu[1:])], cu)


@pytest.mark.parametrize("m,n", [(5, 300), (300, 5), (200, 0), (1, 1), (0, 9), (64, 1000), (257, 129)])
@pytest.mark.parametrize("causal", [True, False])
def test_packed_other_key_lengths(P, ctx, m, n, causal):
    """Queries before the first key see nothing: zeros, lse -inf."""
    g = gen(m * 1000 + n)
    q, k, v = randn(g, m + 3, 8, 64), randn(g, n + 2, 2, 64), randn(g, n + 2, 2, 64)
    scale = 0.3
    out, lse = P.attn_packed(ctx, q, k, v, ints([0, m, m + 3]), cu_k=ints([0, n, n + 2]), causal=causal, scale=scale,
                             lse=True)
    ctx.sync()
    check(out, lse, [reference(q[:m], k[:n], v[:n], causal, scale), reference(q[m:], k[n:], v[n:], causal, scale)],
          [0, m, m + 3])


def test_packed_without_any_keys(P, ctx):
    q, none = randn(gen(4), 6, 8, 64), torch.zeros((0, 2, 64), dtype=BF, device=DEV)
    out, lse = P.attn_packed(ctx, q, none, none, ints([0, 4, 6]), cu_k=ints([0, 0, 0]), lse=True)
    ctx.sync()
    assert (out == 0).all() and (lse == -math.inf).all()


def test_packed_neighbours_do_not_leak(P, ctx):
    """What stands behind a sequence's end is its neighbour's; not a number there stays there."""
    g = gen(5)
    lens = [100, 60, 130]
    cu = [0, 100, 160, 290]
    q, k, v = (randn(g, 290, 4, 128) for _ in range(3))
    want = [reference(q[a:b], k[a:b], v[a:b], True, 128 ** -0.5) for a, b in zip(cu[:-1], cu[1:])]
    k[100:160] = math.nan
    v[100:160] = math.inf
    out, lse = P.attn_packed(ctx, q, k, v, cum(lens), lse=True)
    ctx.sync()
    for b in (0, 2):
        check(out[cu[b]:cu[b + 1]], lse[cu[b]:cu[b + 1]], [want[b]], [0, lens[b]])
    assert torch.isnan(out[100:160]).any()


def test_packed_large_and_small_scores(P, ctx):
    """Maxima that grow late in a row, scores of hundreds, and rows of equal scores."""
    g = gen(6)
    n = 900
    q, k, v = randn(g, n, 2, 128), randn(g, n, 2, 128), randn(g, n, 2, 128)
    k *= torch.linspace(0.01, 12.0, n, device=DEV).to(BF)[:, None, None]
    q[:300] = 0
    out, lse = P.attn_packed(ctx, q, k, v, ints([0, n]), lse=True)
    ctx.sync()
    check(out, lse, [reference(q, k, v, True, 128 ** -0.5)], [0, n])


def test_packed_is_deterministic_and_strides_do_not_matter(P, ctx):
    g = gen(7)
    lens = [700, 20, 333]
    T = sum(lens)
    q, k, v = randn(g, T, 12, 128), randn(g, T, 4, 128), randn(g, T, 4, 128)
    a = P.attn_packed(ctx, q, k, v, cum(lens))
    b = P.attn_packed(ctx, q, k, v, cum(lens))
    by_head = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v)]
    wide = torch.full((T, 12, 136), 7.0, dtype=BF, device=DEV)
    c = P.attn_packed(ctx, *by_head, cum(lens), out=wide[..., :128])
    ctx.sync()
    assert torch.equal(a, b) and torch.equal(a, c)
    assert (wide[..., 128:] == 7.0).all()


# ---- pages: a model on the host ------------------------------------------------------------------------------------
class Model:
    def __init__(self, n_pages, page, n_seqs, max_pages):
        self.page, self.ref = page, np.zeros(n_pages, np.int64)
        self.table, self.lens = np.full((n_seqs, max_pages), -1, np.int64), np.zeros(n_seqs, np.int64)

    def pages(self, n):
        return -(-n // self.page)

    def extend(self, seqs, add):
        free, at = np.nonzero(self.ref == 0)[0], 0
        for s, a in zip(seqs, add):
            lo, hi = self.pages(self.lens[s]), self.pages(self.lens[s] + a)
            self.table[s, lo:hi] = free[at:at + hi - lo]
            self.ref[free[at:at + hi - lo]] = 1
            at += hi - lo
            self.lens[s] += a

    def fork(self, src, dst, keep, cache=None):
        free, at = np.nonzero(self.ref == 0)[0], 0
        for s, d, n in zip(src, dst, keep):
            full, tail = divmod(int(n), self.page)
            self.table[d, :full] = self.table[s, :full]
            np.add.at(self.ref, self.table[s, :full], 1)
            if tail:
                to, frm = free[at], self.table[s, full]
                at += 1
                self.table[d, full], self.ref[to] = to, 1
                if cache is not None:
                    cache[:, :, to, :tail] = cache[:, :, frm, :tail]
            self.lens[d] = n

    def free(self, seqs):
        for s in seqs:
            used = self.pages(self.lens[s])
            np.subtract.at(self.ref, self.table[s, :used], 1)
            self.table[s], self.lens[s] = -1, 0

    def compact(self):
        L = int((self.ref > 0).sum())
        frm = np.nonzero((self.ref > 0) & (np.arange(self.ref.size) >= L))[0]
        to = np.nonzero((self.ref == 0) & (np.arange(self.ref.size) < L))[0]
        m = np.where(self.ref > 0, np.arange(self.ref.size), -1)
        m[frm] = to
        ref = np.where(np.arange(self.ref.size) < L, self.ref, 0)
        ref[to] = self.ref[frm]
        table = np.where(self.table >= 0, m[self.table], -1)
        return ref, table, m, L, frm, to

    def same(self, pg):
        assert (pg.ref.cpu().numpy() == self.ref).all()
        assert (pg.table.cpu().numpy() == self.table).all()
        assert (pg.lens.cpu().numpy() == self.lens).all()


def by_head(pg_args, P, g):
    """A pool whose pages hold their tokens head by head."""
    n_pages, page, n_seqs, width, layers, heads, d = pg_args
    c = randn(g, layers, 2, n_pages, heads, page, d).transpose(3, 4)
    z = P.KVPages.empty(n_pages, page, n_seqs, width, 1, 1, 8)
    return P.KVPages(c, z.ref, z.table, z.lens)


@pytest.mark.parametrize("page,heads,d,layers,order", [(16, 2, 64, 2, "token"), (8, 1, 8, 1, "token"),
                                                       (64, 3, 128, 1, "head"), (256, 1, 24, 3, "token"),
                                                       (32, 2, 40, 40, "head")])
def test_pages_against_the_model(P, ctx, page, heads, d, layers, order):
    g, r = gen(page), np.random.default_rng(page)
    n_pages, n_seqs, width = 1500 if page < 64 else 300, 40, 24
    if order == "token":
        pg = P.KVPages.empty(n_pages, page, n_seqs, width, layers, heads, d)
        pg.cache.copy_(randn(g, *pg.cache.shape))
    else:
        pg = by_head((n_pages, page, n_seqs, width, layers, heads, d), P, g)
    m, cache = Model(n_pages, page, n_seqs, width), pg.cache.clone()
    for step in range(12):
        empty, used = np.nonzero(m.lens == 0)[0], np.nonzero(m.lens > 0)[0]
        grow = r.permutation(n_seqs)[:r.integers(1, 20)]
        room = np.minimum(width * page - m.lens[grow], (m.ref == 0).sum() // 25 * page)
        add = np.array([r.integers(0, max(1, min(x, 4 * page)) + 1) for x in room])
        m.extend(grow, add)
        P.pages_extend(ctx, pg, ints(grow), ints(add))
        empty, used = np.nonzero(m.lens == 0)[0], np.nonzero(m.lens > 0)[0]
        n = min(len(empty), int((m.ref == 0).sum()), r.integers(0, 12))
        if n and len(used):
            src, dst = r.choice(used, n), r.permutation(empty)[:n]
            keep = np.array([r.integers(1, m.lens[s] + 1) for s in src])
            m.fork(src, dst, keep, cache)
            P.pages_fork(ctx, pg, ints(src), ints(dst), ints(keep))
        gone = r.permutation(n_seqs)[:r.integers(0, 12)]
        m.free(gone)
        P.pages_free(ctx, pg, ints(gone))
        ctx.sync()
        m.same(pg)
        assert torch.equal(pg.cache.view(torch.int16) if pg.cache.is_contiguous() else pg.cache, cache.view(torch.int16)
                           if pg.cache.is_contiguous() else cache)
        if step % 4 == 3:
            ref, table, pmap, L, frm, to = m.compact()
            got = P.pages_compact(ctx, pg)
            ctx.sync()
            for a, b in zip(got, (ref, table, pmap, [L])):
                assert (a.cpu().numpy() == np.asarray(b)).all()
            cache[:, :, to] = cache[:, :, frm]
            assert torch.equal(pg.cache, cache)
            pg.replace(got[0], got[1])
            m.ref, m.table = ref, table


def test_large_pool(P, ctx):
    """More pages than chunk counters of a thousand pages each: ranks across wider chunks."""
    n_pages = 3_000_001
    pg = P.KVPages.empty(n_pages, 8, 64, 40000, 1, 1, 8)
    r = np.random.default_rng(3)
    ref = (r.random(n_pages) < 0.7).astype(np.int32)
    pg.ref.copy_(torch.from_numpy(ref))
    add = r.integers(0, 40000 * 8 // 10, 64)
    m = Model(n_pages, 8, 64, 40000)
    m.ref = ref.astype(np.int64)
    m.extend(range(64), add)
    P.pages_extend(ctx, pg, ints(range(64)), ints(add))
    ctx.sync()
    m.same(pg)
    want = m.compact()
    got = P.pages_compact(ctx, pg)
    ctx.sync()
    for a, b in zip(got, want[:4]):
        assert (a.cpu().numpy() == np.asarray(b)).all()


def test_too_few_pages_change_nothing(P, ctx):
    pg = P.KVPages.empty(10, 16, 4, 12, 1, 1, 64)
    P.pages_extend(ctx, pg, ints([0, 1]), ints([60, 33]))
    ctx.sync()
    before = [t.clone() for t in (pg.ref, pg.table, pg.lens, pg.cache)]
    P.pages_extend(ctx, pg, ints([1, 2]), ints([15, 48]))    # 0 + 3 of the 3 free pages
    ctx.sync()
    P.pages_free(ctx, pg, ints([2]))
    P.pages_extend(ctx, pg, ints([1]), ints([-0]))
    ctx.sync()
    for call in (lambda: P.pages_extend(ctx, pg, ints([0, 2]), ints([16, 48])),
                 lambda: (P.pages_extend(ctx, pg, ints([2]), ints([48])),
                          P.pages_fork(ctx, pg, ints([0]), ints([3]), ints([17])))):
        call()
        with pytest.raises(P.CacheRouteError) as e:
            ctx.sync()
        assert e.value.code == P.CR_EOVERFLOW
        P.pages_free(ctx, pg, ints([2]))
        ctx.sync()
        assert int(pg.lens[3]) == 0 and int(pg.lens[0]) == 60
    assert torch.equal(pg.ref, before[0])
    assert torch.equal(pg.cache, before[3])


def test_bad_entries_are_skipped(P, ctx):
    pg = P.KVPages.empty(20, 16, 5, 4, 1, 1, 64)
    P.pages_extend(ctx, pg, ints([0, 1, 2]), ints([20, 5, 64]))
    ctx.sync()
    m = Model(20, 16, 5, 4)
    m.extend([0, 1, 2], [20, 5, 64])

    def bad(call):
        call()
        with pytest.raises(P.CacheRouteError) as e:
            ctx.sync()
        assert e.value.code == P.CR_EINVAL
        m.same(pg)

    m.extend([0], [1])
    bad(lambda: P.pages_extend(ctx, pg, ints([-1, 5, 0, 2, 1]), ints([1, 1, 1, 1, -2])))   # row 2 is full
    bad(lambda: P.pages_fork(ctx, pg, ints([0, 0, 3, 0, 9]), ints([1, 3, 4, -4, 3]), ints([3, 22, 1, 1, 1])))
    m.fork([0], [3], [3])
    bad(lambda: P.pages_fork(ctx, pg, ints([0, 0]), ints([3, 4]), ints([3, 0])))
    bad(lambda: P.pages_free(ctx, pg, ints([7, -1])))
    m.free([0])
    P.pages_free(ctx, pg, ints([0, 0, 4]))     # twice, and an empty row
    ctx.sync()
    m.same(pg)


# ---- attention over pages ------------------------------------------------------------------------------------------
def fill(P, ctx, g, page, lens, heads, d, dtype, layers=1, order="token", shared=None, group=None, width=None):
    """A pool of sequences with random tables; unused places hold NaN.  group[i]: sequences of a group share its
    first shared[group] tokens (whole pages).  Returns pages and each sequence's (k, v)."""
    r = np.random.default_rng(page + sum(lens))
    need = [-(-n // page) for n in lens]
    width = width or max(need + [1]) + 1
    total = sum(need) + 5
    order_of = r.permutation(total)
    shape = (layers, 2, total, page, heads, d) if order == "token" else (layers, 2, total, heads, page, d)
    cache = torch.full(shape, math.nan, dtype=dtype, device=DEV)
    if order != "token":
        cache = cache.transpose(3, 4)
    table = np.full((len(lens), width), -1, np.int64)
    at, seqs, first = 0, [], {}
    for i, n in enumerate(lens):
        s = 0
        if group is not None and group[i] in first:
            s = shared[group[i]] // page
            table[i, :s] = table[first[group[i]], :s]
        elif group is not None:
            first[group[i]] = i
        table[i, s:need[i]] = order_of[at:at + need[i] - s]
        at += need[i] - s
        k, v = randn(g, n, heads, d, dtype=dtype, spread=2.0), randn(g, n, heads, d, dtype=dtype)
        if s:
            k[:s * page], v[:s * page] = (x[:s * page] for x in seqs[first[group[i]]])
        for j in range(need[i]):
            e = min(n, (j + 1) * page)
            cache[layers - 1, 0, table[i, j], :e - j * page] = k[j * page:e]
            cache[layers - 1, 1, table[i, j], :e - j * page] = v[j * page:e]
        seqs.append((k, v))
    ref = np.bincount(table[table >= 0], minlength=total)
    return P.KVPages(cache, ints(ref), ints(table.reshape(-1)).view(len(lens), width), ints(lens)), seqs


PAGED = [
    # page, key heads, query heads, dim, dtype, order, (cached, new) of each sequence
    (16, 2, 8, 128, BF, "token", [(0, 1), (0, 128), (100, 28), (128, 64)]),
    (8, 1, 7, 64, HF, "head", [(1000, 1), (3, 200)]),
    (32, 4, 4, 128, HF, "token", [(300, 300), (31, 2), (0, 33)]),
    (64, 2, 2, 96, BF, "head", [(129, 127)]),
    (128, 1, 16, 128, BF, "token", [(700, 5), (128, 128), (0, 7)]),
    (256, 2, 12, 64, BF, "head", [(600, 77), (255, 1)]),
]


@pytest.mark.parametrize("page,hkv,hq,d,dtype,order,seqs", PAGED)
@pytest.mark.parametrize("causal", [True, False])
def test_paged(P, ctx, page, hkv, hq, d, dtype, order, seqs, causal):
    g = gen(page + hq)
    lens, new = [a + b for a, b in seqs], [b for _, b in seqs]
    pg, kv = fill(P, ctx, g, page, lens, hkv, d, dtype, layers=2, order=order)
    q = randn(g, sum(new), hq, d, dtype=dtype)
    rows = list(range(len(lens)))[::-1]                      # the batch takes the rows backwards
    cu = np.concatenate([[0], np.cumsum([new[i] for i in rows])])
    out, lse = P.attn_paged(ctx, q, pg, 1, ints(cu), seqs=ints(rows), causal=causal, lse=True)
    ctx.sync()
    check(out, lse, [reference(q[a:b], *kv[i], causal, d ** -0.5) for i, a, b in zip(rows, cu[:-1], cu[1:])], cu)


@pytest.mark.parametrize("order", ["token", "head"])
def test_write_then_attend(P, ctx, order):
    """Keys and values written token by token give what they give when packed."""
    g = gen(11)
    lens, new, page = [70, 1, 200, 16], [70, 1, 5, 16], 16
    pg, kv = fill(P, ctx, g, page, lens, 2, 64, BF, layers=2, order=order)
    before = pg.cache.clone()
    cu = np.concatenate([[0], np.cumsum(new)])
    k, v = randn(g, int(cu[-1]), 2, 64), randn(g, int(cu[-1]), 4, 64)[:, 1:3]
    P.kv_write(ctx, pg, 1, k, v, ints(cu))
    ctx.sync()
    assert torch.equal(torch.nan_to_num(pg.cache[0]), torch.nan_to_num(before[0]))
    for i, (a, b) in enumerate(zip(cu[:-1], cu[1:])):
        kv[i][0][lens[i] - new[i]:], kv[i][1][lens[i] - new[i]:] = k[a:b], v[a:b]
        for j in range(-(-lens[i] // page)):
            e = min(lens[i], (j + 1) * page)
            for c in range(2):
                got = pg.cache[1, c, int(pg.table[i, j])]
                assert torch.equal(got[:e - j * page], kv[i][c][j * page:e])
                assert torch.isnan(got[e - j * page:]).all()
    q = randn(g, int(cu[-1]), 4, 64)
    out, lse = P.attn_paged(ctx, q, pg, 1, ints(cu), lse=True)
    ctx.sync()
    check(out, lse, [reference(q[a:b], *kv[i], True, 64 ** -0.5) for i, (a, b) in enumerate(zip(cu[:-1], cu[1:]))], cu)


DECODE = [
    # page, key heads, query heads, dim, dtype, order, shared tokens, (group, own tokens) of each sequence
    (16, 2, 8, 128, BF, "token", [0], [(0, 1)]),
    (16, 8, 64, 128, BF, "token", [640, 128], [(0, 1), (0, 200), (0, 64), (1, 7), (1, 300)]),
    (8, 1, 7, 64, HF, "head", [8], [(0, 0), (0, 1), (0, 129)]),
    (32, 4, 4, 96, HF, "token", [0, 96, 2048], [(0, 5), (0, 0), (1, 1), (2, 40), (2, 1), (2, 500)]),
    (64, 1, 16, 128, BF, "head", [64, 192], [(0, 63), (1, 65), (1, 1)]),
    (16, 1, 40, 128, BF, "token", [160], [(0, i) for i in range(1, 20)]),
    (256, 2, 2, 64, BF, "token", [512, 0], [(0, 3), (0, 256), (1, 5000)]),
    (16, 1, 12, 8, HF, "token", [48], [(0, 1), (0, 2)]),
]


@pytest.mark.parametrize("page,hkv,hq,d,dtype,order,shared,seqs", DECODE)
def test_decode(P, ctx, page, hkv, hq, d, dtype, order, shared, seqs):
    g = gen(page * 7 + hq)
    group = [a for a, _ in seqs]
    lens = [shared[a] + b for a, b in seqs]
    pg, kv = fill(P, ctx, g, page, lens, hkv, d, dtype, order=order, shared=shared, group=group)
    q = randn(g, len(lens), hq, d, dtype=dtype)
    want = [reference(q[i:i + 1], *kv[i], False, d ** -0.5) for i in range(len(lens))]
    off = np.searchsorted(group, np.arange(len(shared) + 1))
    cu = range(len(lens) + 1)
    out, lse = P.attn_decode(ctx, q, pg, 0, lse=True)
    ctx.sync()
    check(out, lse, want, cu)
    out, lse = P.attn_decode(ctx, q, pg, 0, group_off=ints(off), shared=ints(shared), lse=True)
    ctx.sync()
    check(out, lse, want, cu)
    rows = np.random.default_rng(1).permutation(len(lens))
    out, lse = P.attn_decode(ctx, q, pg, 0, seqs=ints(rows), lse=True)
    ctx.sync()
    check(out, lse, [reference(q[i:i + 1], *kv[rows[i]], False, d ** -0.5) for i in range(len(lens))], cu)


@pytest.mark.parametrize("n,longest,hq,hkv,d,dtype", [
    (1, 30000, 8, 2, 128, BF), (2, 1, 4, 4, 64, HF), (8, 9000, 16, 2, 128, BF), (31, 700, 4, 1, 64, BF),
    (32, 5000, 8, 8, 64, HF), (33, 5000, 8, 8, 64, HF), (32, 0, 4, 2, 128, BF), (32, 2500, 40, 1, 128, HF),
])
def test_decode_of_lists_that_the_attention_kernel_makes_and_longer_ones(P, ctx, n, longest, hq, hkv, d, dtype):
    """Up to 32 tokens are listed by the kernel that works on them; pieces of long sequences are joined either way."""
    g = gen(1000 + n + longest)
    rng = np.random.default_rng(n + longest)
    lens = [int(x) for x in rng.integers(0, longest // 4 + 1, n)]
    lens[n // 2] = longest
    pg, kv = fill(P, ctx, g, 16, lens, hkv, d, dtype)
    q = randn(g, n, hq, d, dtype=dtype)
    want = [reference(q[i:i + 1], *kv[i], False, d ** -0.5) for i in range(n)]
    out, lse = P.attn_decode(ctx, q, pg, 0, lse=True)
    ctx.sync()
    check(out, lse, want, range(n + 1))
    rows = rng.permutation(n)
    again, lse = P.attn_decode(ctx, q, pg, 0, seqs=ints(rows), lse=True)
    ctx.sync()
    check(again, lse, [reference(q[i:i + 1], *kv[r], False, d ** -0.5) for i, r in enumerate(rows)], range(n + 1))
    rows[n - 1] = n  # no such row: reported, zeros, the others as before
    out, lse = P.attn_decode(ctx, q, pg, 0, seqs=ints(rows), lse=True)
    with pytest.raises(P.CacheRouteError) as e:
        ctx.sync()
    assert e.value.code == P.CR_EINVAL
    assert (out[n - 1] == 0).all() and (lse[n - 1] == -math.inf).all()
    check(out[:n - 1], lse[:n - 1], [reference(q[i:i + 1], *kv[r], False, d ** -0.5) for i, r in enumerate(rows[:-1])],
          range(n))


def test_decode_with_groups_that_are_not_ascending_stays_in_bounds(P, ctx):
    """Outputs mean nothing then; the call is reported and the next one is right."""
    g = gen(15)
    pg, kv = fill(P, ctx, g, 16, [200, 300, 40, 500], 2, 64, BF)
    q = randn(g, 4, 8, 64)
    for off, shared in (([0, 3, 1, 4], [64, 64, 32]), ([3, 2, 1, 0], [16, 16, 16]), ([2, 9, -5, 4], [600, -7, 48]),
                        ([0, 4, 4, 4], [5000, 16, 16])):
        P.attn_decode(ctx, q, pg, 0, group_off=ints(off), shared=ints(shared))
        try:
            ctx.sync()
        except P.CacheRouteError as e:
            assert e.code == P.CR_EINVAL
    out, lse = P.attn_decode(ctx, q, pg, 0, lse=True)
    ctx.sync()
    check(out, lse, [reference(q[i:i + 1], *kv[i], False, 0.125) for i in range(4)], range(5))


def test_decode_long_and_shared_not_whole_pages(P, ctx):
    """A context that many CTAs share, and a shared length that ends inside a page."""
    g = gen(12)
    lens = [40000, 1003, 1100]
    pg, kv = fill(P, ctx, g, 16, lens, 2, 128, BF, shared=[0, 1000], group=[0, 1, 1])
    for i in (2,):  # sequence 2 begins as sequence 1 does in its first 992 tokens: share 987 of them
        assert torch.equal(kv[2][0][:992], kv[1][0][:992])
    q = randn(g, 3, 16, 128)
    want = [reference(q[i:i + 1], *kv[i], False, 128 ** -0.5) for i in range(3)]
    for groups in (None, ([0, 1, 3], [0, 987])):
        kw = {} if groups is None else dict(group_off=ints(groups[0]), shared=ints(groups[1]))
        out, lse = P.attn_decode(ctx, q, pg, 0, lse=True, **kw)
        ctx.sync()
        check(out, lse, want, range(4))


def test_calls_replay_as_a_graph_on_their_own_stream(P):
    """A step's calls on a stream of their own, captured once and replayed on new values."""
    g = gen(13)
    stream = torch.cuda.Stream()
    c = P.Context(0, stream=stream)
    lens = [200, 33, 90]
    pg, kv = fill(P, c, g, 16, lens, 2, 128, BF)
    q, k, v = randn(g, 3, 8, 128), randn(g, 3, 2, 128), randn(g, 3, 2, 128)
    cu = ints(range(4))
    out = torch.empty_like(q)
    torch.cuda.synchronize()

    def step():
        P.kv_write(c, pg, 0, k, v, cu)
        P.attn_decode(c, q, pg, 0, out=out)

    with torch.cuda.stream(stream):
        step()
        c.sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        q.copy_(randn(g, 3, 8, 128))
        k.copy_(randn(g, 3, 2, 128))
        graph.replay()
        c.sync()
    for i in range(3):
        kv[i][0][-1], kv[i][1][-1] = k[i], v[i]
        o, l, bo, _ = reference(q[i:i + 1], *kv[i], False, 128 ** -0.5)
        assert ((out[i:i + 1].double() - o).abs() <= bo).all()
    c.close()


# ---- refusals ------------------------------------------------------------------------------------------------------
def test_refusals(P, ctx):
    g = gen(14)
    q, k, v = randn(g, 10, 8, 64), randn(g, 10, 2, 64), randn(g, 10, 2, 64)
    cu = ints([0, 10])

    def invalid(call, kind):
        with pytest.raises(kind):
            call()

    invalid(lambda: P.attn_packed(ctx, q, k[:9], v[:9], cu), ValueError)
    invalid(lambda: P.attn_packed(ctx, q.float(), k.float(), v.float(), cu), ValueError)
    invalid(lambda: P.attn_packed(ctx, q, k.half(), v.half(), cu), ValueError)
    invalid(lambda: P.attn_packed(ctx, q, k, v, cu.long()), ValueError)
    invalid(lambda: P.attn_packed(ctx, q[:, :7], k, v, cu), P.CacheRouteError)          # 7 heads on 2
    invalid(lambda: P.attn_packed(ctx, q, k, v, cu, scale=0.0), P.CacheRouteError)
    invalid(lambda: P.attn_packed(ctx, q, k, v, cu, scale=math.inf), P.CacheRouteError)
    invalid(lambda: P.attn_packed(ctx, q[..., :60], k[..., :60], v[..., :60], cu), P.CacheRouteError)
    invalid(lambda: P.attn_packed(ctx, q[..., 4:44], k[..., :40], v[..., :40], cu), P.CacheRouteError)  # 8-byte aligned
    z = torch.zeros((10, 2, 136), dtype=BF, device=DEV)
    invalid(lambda: P.attn_packed(ctx, z, z, z, cu), P.CacheRouteError)
    invalid(lambda: P.KVPages.empty(4, 24, 1, 1, 1, 1, 64)._bind() or P.pages_free(
        ctx, P.KVPages.empty(4, 24, 1, 1, 1, 1, 64), ints([0])), P.CacheRouteError)
    pg = P.KVPages.empty(4, 16, 2, 4, 1, 2, 64)
    invalid(lambda: P.attn_paged(ctx, q, pg, 1, cu), P.CacheRouteError)                  # layer 1 of 1
    invalid(lambda: P.kv_write(ctx, pg, 0, k[:, :1], v, cu), ValueError)
    invalid(lambda: P.attn_decode(ctx, q, pg, 0, group_off=ints([0, 10])), ValueError)
    invalid(lambda: P.pages_extend(ctx, pg, ints([0]), ints([1, 2])), ValueError)
    ctx.sync()
    # rows that do not exist, and tokens outside their row: skipped, reported by the next blocking call
    for call in (lambda: P.attn_decode(ctx, q[:3], pg, 0, seqs=ints([0, 2, -1])),
                 lambda: P.kv_write(ctx, pg, 0, k, v, cu),
                 lambda: P.attn_paged(ctx, q, pg, 0, cu, seqs=ints([9]))):
        call()
        with pytest.raises(P.CacheRouteError) as e:
            ctx.sync()
        assert e.value.code == P.CR_EINVAL
    ctx.sync()


def test_empty_calls(P, ctx):
    pg = P.KVPages.empty(4, 16, 2, 4, 1, 2, 64)
    q = torch.zeros((0, 4, 64), dtype=BF, device=DEV)
    assert P.attn_decode(ctx, q, pg, 0, seqs=ints([])).shape == q.shape
    assert P.attn_packed(ctx, q, q[:, :2], q[:, :2], ints([0, 0])).shape == q.shape
    P.kv_write(ctx, pg, 0, q[:, :2], q[:, :2], ints([0]))
    for call in (P.pages_free,):
        call(ctx, pg, ints([]))
    P.pages_extend(ctx, pg, ints([]), ints([]))
    P.pages_fork(ctx, pg, ints([]), ints([]), ints([]))
    one = randn(gen(1), 2, 4, 64)
    out, lse = P.attn_decode(ctx, one, pg, 0, lse=True)      # rows without tokens
    ctx.sync()
    assert (out == 0).all() and (lse == -math.inf).all()


# ---- the calls together --------------------------------------------------------------------------------------------
def test_example_serves_routed_requests():
    """Router, pages, prompts and shared decoding together, against the model from scratch.  Two layers of about five
    roundings to bfloat16 each (unit roundoff 2^-8, root mean square below 2^-9) stay below 2^-9 * sqrt(10) * 2."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_prefixes.py")
    spec = importlib.util.spec_from_file_location("serve_prefixes", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    said = []
    assert m.main(48, 3, log=said.append) < 2.0 ** -9 * math.sqrt(10) * 2
    assert len(said) == 2


def test_destination_keeps_within_its_rows_and_pages(P, ctx):
    """Idle prefixes leave, least recent first; a batch that does not fit changes nothing."""
    from paper_2608_19677_gb300.destination import Destination

    class Flat:
        layers = 1

        def embed(self, t):
            return t[:, None].to(BF).expand(-1, 64)

        def qkv(self, layer, x):
            y = x[:, None, :].contiguous()
            return y, y, y

        def mix(self, layer, x, out):
            return out

    pg = P.KVPages.empty(12, 16, 5, 8, 1, 1, 64)
    d = Destination(ctx, pg, Flat())
    t = lambda n: torch.arange(n, device=DEV) % 7  # noqa: E731
    rows, _ = d.admit([(1, t(40), 32)])
    d.finish(rows)
    rows, _ = d.admit([(2, t(20), 16)])
    assert set(d.prefixes) == {1, 2}
    with pytest.raises(RuntimeError):
        d.admit([(3, t(300), 200)])
    assert set(d.prefixes) == {1, 2} and d.order() == rows
    more, out = d.admit([(3, t(70), 64), (2, t(18), 16)])     # prefix 1 leaves
    assert set(d.prefixes) == {2, 3} and out.shape[0] == 8
    d.step(t(3))
    ctx.sync()
    used = int((pg.ref > 0).sum())
    assert used == pg.n_pages - d.free_pages
    assert [int(pg.lens[r]) for r in d.order()] == [21, 19, 71]
