"""Attention over pages in 8 bits where factors, scores, powers and tables are at their ends, against the plain form in 64
bits (helpers and bounds: test_gpu_cache8).
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytestmark = [pytest.mark.gpu, pytest.mark.skip(reason="needs a CUDA GPU")]
else:
    pytestmark = pytest.mark.gpu

from test_gpu_cache8 import BF, DEV, HF, P, check, ctx, cum, fails, fill8, gen, ints, randn, reference, turned  # noqa: E402,F401


def sequences(out, lse, q, rows, cu, causal, scale, extra=0.0):
    parts = []
    for i, (a, b) in enumerate(zip(cu, cu[1:])):
        o, l, bo, bl = reference(q[a:b], *rows[i], causal, scale)
        parts.append((o, l, bo + extra, bl))
    check(out, lse, parts, cu)


# ---- zeros ---------------------------------------------------------------------------------------------------------
ZEROS = {
    "queries": dict(q=0.0),
    "keys": dict(k=0.0),
    "both": dict(q=0.0, k=0.0),
    "a tile of keys": dict(q=0.0, tile=0.0),
    "small queries, zero keys": dict(q=2.0 ** -40, k=0.0),
    "zero queries, small keys": dict(q=0.0, k=2.0 ** -30),
    "a row of queries": dict(row=0.0, k=0.0),
}


@pytest.mark.parametrize("what", list(ZEROS))
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("d", [64, 128])
def test_zeros(P, ctx, what, dtype, d):
    """Queries and keys of zeros, or nearly so, beside masked ones: the mean of the values that a query sees."""
    how, g, hq, hkv = ZEROS[what], gen(d), 4, 2
    lens, new = [127, 128, 129, 255, 256, 300, 1, 600], [127, 5, 129, 1, 200, 300, 1, 3]
    at = np.concatenate([[0], np.cumsum(lens)])

    def spread(k, v):
        k = (k.double() * how.get("k", 1.0)).to(dtype)
        for a, n in zip(at, lens):
            if "tile" in how and n > 128:
                k[a + 128:a + 256] = 0
        return k, v

    pg, rows = fill8(P, ctx, g, 16, 16, lens, hkv, d, dtype, spread=spread)
    q = (randn(g, sum(new), hq, d, dtype=dtype).double() * how.get("q", 1.0)).to(dtype)
    if "row" in how:
        q[::3] = 0
    cu = np.concatenate([[0], np.cumsum(new)])
    for causal in (True, False):
        out, lse = P.attn_paged(ctx, q, pg, 0, cum(new), causal=causal, lse=True)
        ctx.sync()
        sequences(out, lse, q, rows, cu, causal, d ** -0.5)
    last = cu[1:] - 1
    one, olse = P.attn_decode(ctx, q[last], pg, 0, lse=True)
    ctx.sync()
    sequences(one, olse, q[last], rows, range(len(lens) + 1), False, d ** -0.5)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_zeros_in_a_shared_prefix(P, ctx, dtype):
    g, shared, members, hkv, hq, page = gen(3), [160, 32, 304], [[1, 5, 100], [17, 2], [9, 300]], 2, 16, 16
    group = [i for i, m in enumerate(members) for _ in m]
    lens = [shared[i] + n for i, m in enumerate(members) for n in m]
    pg, rows = fill8(P, ctx, g, page, 16, lens, hkv, 64, dtype, shared=shared, group=group, spread=lambda k, v: (k * 0, v),
                     width=8192 * 64 // (len(lens) * hkv * page) + 1)
    q = randn(g, len(lens), hq, 64, dtype=dtype) * 0
    before = ctx.launches
    out, lse = P.attn_decode(ctx, q, pg, 0, group_off=cum([len(m) for m in members]), shared=ints(shared), lse=True)
    assert ctx.launches - before == 4
    ctx.sync()
    sequences(out, lse, q, rows, range(len(lens) + 1), False, 0.125)


# ---- scores of any size --------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("hq", [4, 16])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("call,bits", [("decode", 8), ("paged", 8), ("decode", 16), ("paged", 16), ("packed", 16)])
def test_scores_of_any_finite_size(P, ctx, call, bits, hq, sign, dtype):
    """Equal keys, so that every weight is the same however large the score: the mean of the values, and lse = score + log n.
    Scores from 2^21 to -+2^112 (half: 2^13 to 2^26): below -1e30 and above 1e30; off by 2^-18 of their size, and lse by a
    few 32-bit roundings."""
    g, d, lens = gen(7), 64, [700, 40]
    up, low, high = (50, -32, 59) if dtype == BF else (10, 0, 13)
    key = randn(g, 1, 1, d, dtype=dtype).abs().clamp_min(0.5)
    if bits == 8:
        pg, rows = fill8(P, ctx, g, 16, 16, lens, 1, d, dtype, spread=lambda k, v: ((key * 2.0 ** up).expand_as(k).contiguous(), v))
    else:
        pg = P.KVPages.empty(60, 16, 2, 50, 1, 1, d, dtype=dtype)
        k, v = (key * 2.0 ** up).expand(740, 1, d).contiguous(), randn(g, 740, 1, d, dtype=dtype)
        P.pages_extend(ctx, pg, ints([0, 1]), ints(lens))
        P.kv_write(ctx, pg, 0, k, v, cum(lens))
        rows = [(k[:700].double(), v[:700].double()), (k[700:].double(), v[700:].double())]
    q = (sign * key.expand(2, hq, d).double() * 2.0 ** torch.linspace(low, high, hq, device=DEV).double()[None, :, None]).to(dtype)
    if call == "decode":
        out, lse = P.attn_decode(ctx, q, pg, 0, scale=0.125, lse=True)
    elif call == "paged":
        out, lse = P.attn_paged(ctx, q, pg, 0, ints([0, 1, 2]), scale=0.125, lse=True)
    else:
        out, lse = P.attn_packed(ctx, q, k, v, ints([0, 1, 2]), cu_k=cum(lens), scale=0.125, lse=True)
    ctx.sync()
    for i, (k, v) in enumerate(rows):
        mean, size = v.mean(0), v.abs().mean(0)
        u = 2.0 ** -8 if dtype == BF else 2.0 ** -11
        assert ((out[i].double() - mean).abs() <= u * (mean.abs() + size) * 1.01 + 2.0 ** -19 * size).all()
        s = 0.125 * (q[i].double() * k[0]).sum(-1)
        assert s[-1] * sign > (1e30 if dtype == BF else 2.0 ** 24)
        assert ((lse[i].double() - (s + math.log(len(k)))).abs() <= s.abs() * 2.0 ** -17).all()


@pytest.mark.parametrize("size", [2.0 ** 18, 2.0 ** 21, 2.0 ** 30, 2.0 ** 90])
@pytest.mark.parametrize("bits,call", [(8, "decode"), (8, "paged"), (16, "decode"), (16, "paged")])
def test_scores_far_apart(P, ctx, bits, call, size):
    """Keys of ordinary scores behind ones that are far below: the softmax of the former.  Equal keys far above, behind those:
    the mean of their values."""
    g, d, lens = gen(8), 64, [600, 300]
    key = randn(g, 1, 1, d).abs().clamp_min(0.5)
    k, v = randn(g, 900, 1, d), randn(g, 900, 1, d)
    k[:256], k[856:] = -size * key, size * key
    if bits == 8:
        pg, rows = fill8(P, ctx, g, 16, 16, lens, 1, d, BF, spread=lambda *_: (k, v))
    else:
        pg = P.KVPages.empty(60, 16, 2, 40, 1, 1, d)
        P.pages_extend(ctx, pg, ints([0, 1]), ints(lens))
        P.kv_write(ctx, pg, 0, k, v, cum(lens))
        rows = [(k[:600].double(), v[:600].double()), (k[600:].double(), v[600:].double())]
    q = randn(g, 2, 8, d).abs().clamp_min(0.25)
    if call == "decode":
        out, lse = P.attn_decode(ctx, q, pg, 0, lse=True)
    else:
        out, lse = P.attn_paged(ctx, q, pg, 0, ints([0, 1, 2]), lse=True)
    ctx.sync()
    seen = [tuple(x[256:] for x in rows[0])]
    check(out[:1], lse[:1], [reference(q[:1], *seen[0], False, d ** -0.5)], [0, 1])
    mean, sizes = rows[1][1][256:].mean(0), rows[1][1][256:].abs().mean(0)
    assert ((out[1].double() - mean).abs() <= 2.0 ** -8 * (mean.abs() + sizes) * 1.01 + 2.0 ** -19 * sizes).all()
    s = d ** -0.5 * (q[1].double() * rows[1][0][-1]).sum(-1)
    assert ((lse[1].double() - (s + math.log(44))).abs() <= s * 2.0 ** -17).all()


# ---- tables of the caller's own ------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [8, 16, 64, 128])
def test_pages_outside_the_pool_are_zeros(P, ctx, dtype, d, page):
    """A table of the caller's own that names no page within a row's length: keys and values of zeros, as over 16 bits,
    whatever the memory held that they would have come to."""
    g, n = gen(page + d), 900
    full, _ = fill8(P, ctx, g, page, 8, [40000], 2, d, dtype)
    full.cache.view(torch.uint8).fill_(0x7f)              # not-a-number into every place of shared memory
    full.scale.fill_(1.0)
    pg, rows = fill8(P, ctx, g, page, 8, [n, n], 2, d, dtype)
    gone = [1, 3, n // page - 1, n // page]                # the last one holds the row's end
    for j, p in zip(gone, (-1, pg.n_pages, 2 ** 31 - 1, -2 ** 31)):
        pg.table[0, j] = p
        for x in rows[0]:
            x[j * page:(j + 1) * page] = 0
    q = randn(g, 2, 8, d, dtype=dtype)
    P.attn_decode(ctx, randn(g, 1, 8, d, dtype=dtype), full, 0)
    one, olse = P.attn_decode(ctx, q, pg, 0, lse=True)
    P.attn_paged(ctx, randn(g, 1, 8, d, dtype=dtype), full, 0, ints([0, 1]))
    many, mlse = P.attn_paged(ctx, q, pg, 0, ints([0, 1, 2]), lse=True)
    again = P.attn_decode(ctx, q, pg, 0)
    ctx.sync()
    sequences(one, olse, q, rows, range(3), False, d ** -0.5)
    sequences(many, mlse, q, rows, range(3), False, d ** -0.5)
    assert torch.equal(one, again)


# ---- pieces --------------------------------------------------------------------------------------------------------
def test_pieces_hold_values_as_large_as_16_bits_do(P, ctx):
    """2,048 keys of equal weight, values near 2^115, cut into pieces whose unnormalised sums stay finite."""
    g, n, d = gen(11), 2048, 128
    spread = lambda k, v: (k, (v.abs().double() * 2.0 ** 115).to(BF))  # noqa: E731
    pg, rows = fill8(P, ctx, g, 16, 16, [n], 2, d, BF, spread=spread)
    wide = P.KVPages.empty(n // 16, 16, 1, n // 16, 1, 2, d)
    P.pages_extend(ctx, wide, ints([0]), ints([n]))
    P.kv_write(ctx, wide, 0, *(x.to(BF) for x in rows[0]), ints([0, n]))
    q = torch.zeros((1, 4, d), dtype=BF, device=DEV)
    for pool in (wide, pg):
        many, mlse = P.attn_paged(ctx, q, pool, 0, ints([0, 1]), lse=True)
        one, olse = P.attn_decode(ctx, q, pool, 0, lse=True)
        ctx.sync()
        sequences(many, mlse, q, rows, [0, 1], False, d ** -0.5)
        sequences(one, olse, q, rows, [0, 1], False, d ** -0.5)


# ---- rows that stand in a list twice -------------------------------------------------------------------------------
@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("bits", [8, 16])
def test_entries_without_tokens_do_not_claim_a_row(P, ctx, bits, many):
    """As the padding of a batch names a row: only an entry that has tokens writes it."""
    g, rot = gen(13), P.Rotary(64)
    pg = P.KVPages.empty(40, 16, 4, 8, 1, 2, 64, bits=bits)
    P.pages_extend(ctx, pg, ints([1, 2]), ints([20, 5]))
    k, v, q = randn(g, 25, 2, 64), randn(g, 25, 2, 64), randn(g, 25, 4, 64)
    pad = 1500 if many else 3
    seqs, cu = [2] * pad + [1, 2, 1], [0] * pad + [0, 20, 25, 25]
    want = P.rope(ctx, q, rot, ints(list(range(20)) + list(range(5))))
    assert torch.equal(P.kv_append(ctx, pg, 0, q, k, v, rot, ints(cu), seqs=ints(seqs)), want)
    ctx.sync()
    _, got = P.kv_read(ctx, pg, 0, ints([0, 20, 25]), seqs=ints([1, 2]))
    P.kv_write(ctx, pg, 0, v, k, ints(cu), seqs=ints(seqs))
    ctx.sync()
    _, back = P.kv_read(ctx, pg, 0, ints([0, 20, 25]), seqs=ints([1, 2]))
    ctx.sync()
    tol = 2.0 ** -4 if bits == 8 else 0.0
    for x, y in ((got, v), (back, k)):
        assert ((x - y).abs().double() <= y.abs().double() * tol + (2.0 ** -9 if bits == 8 else 0)).all()


# ---- reading back --------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("bits", [8, 16])
def test_reading_for_no_rows(P, ctx, bits):
    """Tokens of no entry are zeros, and reported, as those behind the last entry are."""
    pg = P.KVPages.empty(4, 16, 2, 2, 1, 2, 64, bits=bits)
    for cu in (ints([0]), ints([])):
        k, v = (torch.full((5, 2, 64), math.nan, dtype=BF, device=DEV) for _ in range(2))
        fails(P, ctx, P.CR_EINVAL, lambda: P.kv_read(ctx, pg, 0, cu, out=(k, v)))
        assert bool((k == 0).all()) and bool((v == 0).all())
        assert P.kv_read(ctx, pg, 0, cu)[0].shape == (0, 2, 64)
    ctx.sync()


# ---- prefixes that move --------------------------------------------------------------------------------------------
@pytest.mark.parametrize("bits", [8, 16])
def test_install_refuses_before_idle_prefixes_leave(P, ctx, bits):
    from examples.serve_prefixes import TinyAttention
    from paper_2608_19677_gb300.destination import Destination
    model = TinyAttention(torch, DEV)
    pages = P.KVPages.empty(8, 16, 3, 8, model.layers, model.kv_heads, model.dim, bits=bits)
    d = Destination(ctx, pages, model)
    text = torch.arange(70, device=DEV)
    rows, _ = d.admit([(1, text, 64)])
    d.finish(rows)                                   # an idle prefix of four pages; five more do not fit beside it
    kv = [tuple(randn(gen(5), 80, model.kv_heads, model.dim) for _ in range(2)) for _ in range(model.layers)]
    k, v = kv[1]
    free = d.free_pages, sorted(d.free_rows)
    for wrong in ((k.half(), v), (k, v.float()), (k[:, :1], v[:, :1]), (k[..., :32], v[..., :32]), (k, v[..., None]), (k.cpu(), v.cpu()),
                  (k, v, v), (k, v.transpose(1, 2).contiguous().transpose(1, 2)), (k, v.clone().requires_grad_()),
                  (k, torch.cat([v, v], -1)[..., 4:4 + model.dim])):
        with pytest.raises(ValueError):
            d.install(2, [kv[0], wrong])
        assert list(d.prefixes) == [1] and (d.free_pages, sorted(d.free_rows)) == free
    with torch.no_grad():
        d.install(2, [kv[0], (k, v.clone().requires_grad_())])
    assert list(d.prefixes) == [2]
    ctx.sync()


# ---- powers far apart ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("hq", [2, 16])
def test_many_rows_over_blocks_of_very_different_size(P, ctx, dtype, hq):
    """Several causal tokens over lengths off a tile; values' powers 2^18 apart, keys' 2^4, whole blocks and tiles of zeros,
    queries from zero and 2^-40 (bfloat16) to 2^3: outputs and the kernel's own lse.

    The bound has a term more, derived before its first run: the kernel's weights are halves of 2^6 times the row's own, so
    each is off by 2^-31 of the row's largest at most (half of a half's last subnormal place, 2^-25, over 2^6), and numbers
    are off by 2^-31 of the largest power so far; a row's sum is at least its largest weight.  Together (n + 1) 2^-31 of the
    largest value."""
    g, d = gen(29), 64
    lens, new = [500, 129, 777], [130, 3, 64]
    n = sum(lens)

    def spread(k, v):
        i = torch.arange(n, device=DEV) // 16
        k = (k * 2.0 ** (i % 5 - 3)[:, None, None]).to(dtype)
        v = (v.double() * 2.0 ** ((i * 7 % 19) - 14).double()[:, None, None]).to(dtype)
        k[i % 11 == 4], v[i % 13 == 2] = 0, 0
        k[640:1100] = 0
        return k, v

    pg, rows = fill8(P, ctx, g, 16, 16, lens, 1, d, dtype, spread=spread)
    q = randn(g, sum(new), hq, d, dtype=dtype, spread=0.5)
    if dtype == BF:
        q = (q.double() * 2.0 ** torch.linspace(-40, 3, hq, device=DEV).double()[None, :, None]).to(dtype)
    q[::7] = 0
    cu = np.concatenate([[0], np.cumsum(new)])
    for causal in (True, False):
        out, lse = P.attn_paged(ctx, q, pg, 0, cum(new), causal=causal, scale=0.25, lse=True)
        ctx.sync()
        most = max(float(v.abs().max()) for _, v in rows)
        sequences(out, lse, q, rows, cu, causal, 0.25, extra=(max(lens) + 1) * 2.0 ** -31 * most)


# ---- a server ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("rotary", [True, False])
def test_destination_holds_the_models_keys_and_values(P, ctx, bits, rotary):
    """After every pass, a row's new tokens are the model's keys, rotated to their positions, and its values: rounded once, by
    2^-4 (8 bits) or 2^-8 (rotated keys) of themselves, or by 2^-10 of their block's power, which is below 2^-7 times the
    row's largest magnitude (448 2^e is less than twice its block's)."""
    from examples.serve_prefixes import TinyAttention
    from paper_2608_19677_gb300.destination import Destination
    rot = P.Rotary(64, scaling="ramp", factor=4.0, original=256) if rotary else None
    met = []

    class Watched(TinyAttention):
        def qkv(self, layer, x):
            self.kv = super().qkv(layer, x)[1:]
            return *super().qkv(layer, x)[:1], *self.kv

        def mix(self, layer, x, out):
            ctx.sync()
            at = 0
            for row, m in met[-1]:
                n = int(pages.lens[row])
                held = P.kv_read(ctx, pages, layer, ints([0, n]), seqs=ints([row]))
                ctx.sync()
                k, v = (t[at:at + m] for t in self.kv)
                k, off = turned(k, np.arange(n - m, n), rot) if rot is not None else (k.double(), 0.0)
                for got, want, slack, exact in ((held[0], k, off, rot is None), (held[1], v.double(), 0.0, True)):
                    near = 2.0 ** -4 if bits == 8 else 0.0 if exact else 2.0 ** -8
                    small = 2.0 ** -17 * 1.07 * float(got.abs().max()) if bits == 8 else 0.0
                    assert ((got[n - m:].double() - want).abs() <= near * want.abs() * 1.01 + slack * 1.07 + small).all(), (layer, row)
                at += m
            assert at == out.shape[0]
            return super().mix(layer, x, out)

    model = Watched(torch, DEV, rotary=rot)
    pages = P.KVPages.empty(200, 16, 12, 12, model.layers, model.kv_heads, model.dim, bits=bits)
    d = Destination(ctx, pages, model)
    forward = d._forward

    def watched(tokens, cu, rows, groups=None):
        met.append(list(zip(rows.tolist(), np.diff(cu.tolist()).tolist())))
        return forward(tokens, cu, rows, groups)

    d._forward = watched
    g = gen(61)
    text = lambda n: torch.randint(0, 4096, (n,), generator=g, device=DEV)  # noqa: E731
    a, b = text(100), text(33)
    d.admit([(1, torch.cat([a, text(5)]), 100), (2, torch.cat([b[:30], text(40)]), 30), (1, torch.cat([a[:64], text(1)]), 64)])
    for _ in range(3):
        d.step(text(3))
    d.compact()
    d.step(text(3))
    assert len(met) == 6


def test_example_in_8_bits():
    """Keys and values are off by 2^-4 / sqrt(3) of themselves in the mean square at most, independently; the model's scores
    have a spread of 1, so that this moves a layer's attention by sqrt(2) times as much of itself, through its values and
    through its weights.  Attention is at most as large as what it is added to.  The second layer is off by that again, and
    by what the first layer's error does to its queries, keys and values: sqrt(1 + 1 + 3) in all; twice that for the worst of
    the requests, and the bound of 16 bits beside it."""
    import examples.serve_prefixes as m
    bound = 2 * 2.0 ** -4 / math.sqrt(3) * math.sqrt(2) * math.sqrt(5) + 2.0 ** -9 * math.sqrt(12) * 2
    for rotary in (True, False):
        assert m.main(48, 3, log=lambda *_: None, rotary=rotary, bits=8) < bound
