"""Pages and attention at the limits of their use: rows that were not grown, long lists, streams, graphs.  Bounds of the
attention tests are those derived in test_gpu_prefix_cache.py."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytestmark = [pytest.mark.gpu, pytest.mark.skip(reason="needs a CUDA GPU")]
else:
    pytestmark = pytest.mark.gpu

from test_gpu_prefix_cache import BF, DEV, HF, Model, P, check, ctx, fill, gen, ints, randn, reference  # noqa: E402, F401


def raises_at_sync(P, ctx, code):
    with pytest.raises(P.CacheRouteError) as e:
        ctx.sync()
    assert e.value.code == code


@pytest.mark.parametrize("add,pages,code", [(70, 64, "CR_EINVAL"), (30, 4, "CR_EOVERFLOW")])
@pytest.mark.parametrize("keep", [32, 40])
def test_a_row_that_was_not_grown_does_not_write_into_shared_pages(P, ctx, add, pages, code, keep):
    """A fork of 32 tokens (or 40: two shared pages and one of its own) whose extension the row's width, or the pool,
    does not allow: its new tokens would fall on the prefix' last ones."""
    g = gen(keep + add)
    pg = P.KVPages.empty(pages, 16, 3, 6, 2, 2, 64)
    pg.cache.copy_(randn(g, *pg.cache.shape))
    P.pages_extend(ctx, pg, ints([0]), ints([48]))
    P.pages_fork(ctx, pg, ints([0]), ints([1]), ints([keep]))
    ctx.sync()
    P.pages_extend(ctx, pg, ints([1]), ints([add]))
    raises_at_sync(P, ctx, getattr(P, code))
    assert int(pg.lens[1]) == keep
    before = pg.cache.clone()
    k, v = randn(g, 20, 2, 64), randn(g, 20, 2, 64)
    P.kv_write(ctx, pg, 1, k, v, ints([0, 20]), seqs=ints([1]))
    raises_at_sync(P, ctx, P.CR_EINVAL)
    if keep == 40:      # the row's own page holds its last 8 tokens
        before[1, 0, int(pg.table[1, 2]), :8], before[1, 1, int(pg.table[1, 2]), :8] = k[12:], v[12:]
    assert torch.equal(pg.cache, before)


@pytest.mark.parametrize("call", ["packed", "paged", "decode", "compact"])
def test_outputs_leave_memory_alone_that_the_current_stream_still_reads(P, call):
    """A context with a stream of its own makes an output while the current stream has not yet read a tensor of that
    shape that the program has already let go."""
    g = gen(31)
    stream = torch.cuda.Stream()
    c = P.Context(0, stream=stream)
    pg, _ = fill(P, c, g, 16, [700] * 300, 2, 64, BF)
    q, k = randn(g, 300, 8, 64), randn(g, 300, 2, 64)
    cu = ints(range(301))
    run = {"packed": lambda: [P.attn_packed(c, q, k, k, cu, lse=True)[0]],
           "paged": lambda: [P.attn_paged(c, q, pg, 0, cu)],
           "decode": lambda: [P.attn_decode(c, q, pg, 0)],
           "compact": lambda: list(P.pages_compact(c, pg)[:3])}[call]
    torch.cuda.synchronize()
    like = [(t.shape, t.dtype) for t in run()]
    c.sync()
    for _ in range(4):
        x = [torch.full(s, 3, dtype=d, device=DEV) for s, d in like]
        torch.cuda._sleep(20_000_000)
        y = [t + 1 for t in x]
        x = None
        out = run()
        torch.cuda.synchronize()
        assert all((t == 4).all() for t in y)
        y = out = None
    c.close()


@pytest.mark.parametrize("adds", [[1 << 25] * 1024, [1 << 25] * 1023 + [(1 << 25) - 8], [1 << 25] * 512 + [8]])
def test_needs_that_pass_32_bits_change_nothing(P, ctx, adds):
    """1,024 rows that ask for 2^22 pages of 8 tokens each: 2^32 pages, of the 64 that there are."""
    n = len(adds)
    z = P.KVPages.empty(64, 8, 1, 1, 1, 1, 8)
    pg = P.KVPages(z.cache, z.ref, torch.full((n, 1 << 22), -1, dtype=torch.int32, device=DEV),
                   torch.zeros(n, dtype=torch.int32, device=DEV))
    assert sum(-(-a // 8) for a in adds) >= 1 << 31
    P.pages_extend(ctx, pg, ints(range(n)), ints(adds))
    raises_at_sync(P, ctx, P.CR_EOVERFLOW)
    assert not pg.lens.any() and not pg.ref.any() and int(pg.table.amax()) == -1
    P.pages_extend(ctx, pg, ints([5, 3]), ints([100, 408]))      # 13 and 51: all of them
    ctx.sync()
    assert pg.ref.all() and pg.table[5, :13].tolist() == list(range(13)) and pg.table[3, :51].tolist() == list(range(13, 64))


def test_of_entries_that_name_a_row_twice_the_first_is_carried_out(P, ctx):
    """Within a round of 1,024 entries and across rounds, each entry with a need of its own; the first of a row may be
    one that cannot be carried out."""
    r = np.random.default_rng(8)
    n_seqs, width, n = 600, 40, 3000
    for trial in range(12):
        seqs, add = r.integers(0, n_seqs, n), r.integers(0, 300, n)
        add[r.random(n) < 0.05] = width * 16 + 1
        add[r.random(n) < 0.05] = -1
        m = Model(20000, 16, n_seqs, width)
        first = {}
        for i, (s, a) in enumerate(zip(seqs, add)):
            if s not in first and 0 <= a <= width * 16:
                first[s] = i
        m.extend(seqs[list(first.values())], add[list(first.values())])
        pg = P.KVPages.empty(20000, 16, n_seqs, width, 1, 1, 8)
        P.pages_extend(ctx, pg, ints(seqs), ints(add))
        raises_at_sync(P, ctx, P.CR_EINVAL)
        m.same(pg)
        # forks into rows that stand twice: each from a parent, and of a length, of its own
        some = [s for s in first if m.lens[s]]
        empty = np.nonzero(m.lens == 0)[0]
        src, dst = r.choice(some, 2000), r.choice(empty, 2000)
        keep = np.array([r.integers(1, m.lens[s] + 1) for s in src])
        keep[::37] = 0
        taken = {}
        for i, d in enumerate(dst):
            if d not in taken and keep[i] > 0:
                taken[d] = i
        taken = list(taken.values())
        m.fork(src[taken], dst[taken], keep[taken])
        P.pages_fork(ctx, pg, ints(src), ints(dst), ints(keep))
        raises_at_sync(P, ctx, P.CR_EINVAL)
        m.same(pg)


def test_a_graph_stays_right_after_larger_calls(P):
    """Larger lists of work, pieces and page calls replace the scratch that the captured calls work in."""
    g = gen(41)
    stream = torch.cuda.Stream()
    c = P.Context(0, stream=stream)
    lens, group = [900, 33, 917, 500], [0, 1, 0, 2]
    order = [0, 2, 1, 3]
    pg, kv = fill(P, c, g, 16, [lens[i] for i in order], 2, 128, BF, shared=[896, 0, 0], group=[group[i] for i in order])
    big, _ = fill(P, c, g, 16, [3000] * 700, 2, 128, BF)
    q, out, prompt = randn(g, 4, 16, 128), torch.empty(4, 16, 128, dtype=BF, device=DEV), randn(g, 300, 4, 128)
    whole = torch.empty_like(prompt)
    off, shared, cu = ints([0, 2, 3, 4]), ints([896, 0, 0]), ints([0, 300])
    rows = P.KVPages.empty(100, 16, 8, 16, 1, 1, 64)
    row, tokens = ints([3]), ints([40])
    torch.cuda.synchronize()

    def step():
        P.attn_decode(c, q, pg, 0, group_off=off, shared=shared, out=out)
        P.attn_packed(c, prompt, prompt, prompt, cu, out=whole)
        P.pages_extend(c, rows, row, tokens)
        P.pages_free(c, rows, row)

    with torch.cuda.stream(stream):
        step()
        c.sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        many = randn(g, 700, 32, 128)
        for _ in range(2):
            P.attn_decode(c, many, big, 0, group_off=ints(range(0, 701, 350)), shared=ints([0, 0]))
            P.attn_decode(c, many, big, 0)
            P.attn_packed(c, many, many, many, ints([0, 1, 700]))
            z = P.KVPages.empty(4_000_000, 8, 4, 4, 1, 1, 8)
            P.pages_extend(c, z, ints([0]), ints([8]))
            c.sync()
            q.copy_(randn(g, 4, 16, 128))
            prompt.copy_(randn(g, 300, 4, 128))
            graph.replay()
            c.sync()
            for i in range(4):
                o, _, bo, _ = reference(q[i:i + 1], *kv[i], False, 128 ** -0.5)
                assert ((out[i:i + 1].double() - o).abs() <= bo).all()
            o, _, bo, _ = reference(prompt, prompt, prompt, True, 128 ** -0.5)
            assert ((whole.double() - o).abs() <= bo).all()
            assert not rows.ref.any()
    c.close()


@pytest.mark.parametrize("way", ["default to own", "own to own", "own to default"])
def test_calls_after_a_switch_of_streams_wait_for_those_before(P, way):
    """Both work in the context's scratch."""
    g = gen(51)
    own = [torch.cuda.Stream(), torch.cuda.Stream()]
    old = torch.cuda.current_stream() if way.startswith("default") else own[0]
    new = torch.cuda.current_stream() if way.endswith("default") else own[1]
    c = P.Context(0, stream=old)
    pg, kv = fill(P, c, g, 16, [3000, 40], 2, 128, BF)
    q = randn(g, 2, 8, 128)
    torch.cuda.synchronize()
    P.attn_decode(c, q, pg, 0)
    c.sync()
    ended = torch.cuda.Event()
    with torch.cuda.stream(old):
        torch.cuda._sleep(100_000_000)
        ended.record()
    c.set_stream(new)
    assert c.stream.cuda_stream == new.cuda_stream
    out, lse = P.attn_decode(c, q, pg, 0, lse=True)
    new.synchronize()
    waited = ended.query()
    c.sync()
    check(out, lse, [reference(q[i:i + 1], *kv[i], False, 128 ** -0.5) for i in range(2)], range(3))
    c.close()
    assert waited


def test_a_switch_to_a_stream_under_capture_leaves_the_capture_alone(P):
    g = gen(52)
    c = P.Context(0)
    pg, kv = fill(P, c, g, 16, [300, 40], 2, 128, BF)
    q = randn(g, 2, 8, 128)
    out = torch.empty_like(q)
    P.attn_decode(c, q, pg, 0, out=out)
    c.sync()
    out.zero_()
    stream, home = torch.cuda.Stream(), c.stream
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        c.set_stream(torch.cuda.current_stream())
        P.attn_decode(c, q, pg, 0, out=out)
        c.set_stream(home)
    torch.cuda.synchronize()
    assert not out.any()
    graph.replay()
    torch.cuda.synchronize()
    for i in range(2):
        o, _, bo, _ = reference(q[i:i + 1], *kv[i], False, 128 ** -0.5)
        assert ((out[i:i + 1].double() - o).abs() <= bo).all()
    c.close()


@pytest.mark.parametrize("hq,hkv,d,n", [(8, 2, 128, 40), (16, 1, 64, 150)])
def test_steps_queued_one_after_the_other_see_each_others_tables_and_pages(P, ctx, hq, hkv, d, n):
    """Rows are freed, forked, grown and written again and again without a wait between, each step's tables and values
    unlike the last one's, and every step's grouped decoding is right."""
    g, r = gen(n), np.random.default_rng(n)
    page, pre, keys = 16, 900, 3
    pg = P.KVPages.empty(keys * 57 + n * 10 + 40, page, keys + n, 70, 1, hkv, d)
    own = list(range(keys, keys + n))
    m = Model(pg.n_pages, page, keys + n, 70)
    heads = [ints(range(keys)), ints([pre] * keys), ints(np.arange(keys + 1) * pre)]
    k0, v0 = randn(g, keys * pre, hkv, d, spread=2.0), randn(g, keys * pre, hkv, d)
    group = np.sort(r.integers(0, keys, n))
    off, dst = np.searchsorted(group, np.arange(keys + 1)), ints(own)
    steps = []
    for step in range(6):
        keep, add = r.integers(1, pre + 1, n), r.integers(1, 100, n)
        keep[r.random(n) < 0.7] = pre
        least = [min([pre] + [int(x) for x in keep[off[i]:off[i + 1]]]) // page * page for i in range(keys)]
        T = int(add.sum())
        steps.append((keep, add, [ints(group), ints(keep), ints(add), ints(np.concatenate([[0], np.cumsum(add)])), ints(off),
                                  ints(least)], randn(g, T, hkv, d, spread=2.0), randn(g, T, hkv, d), randn(g, n, hq, d)))
    torch.cuda.synchronize()
    P.pages_extend(ctx, pg, heads[0], heads[1])
    P.kv_write(ctx, pg, 0, k0, v0, heads[2], seqs=heads[0])
    m.extend(range(keys), [pre] * keys)
    got = []
    for keep, add, (src, kp, ad, cu, go, sh), k, v, q in steps:
        P.pages_free(ctx, pg, dst)
        P.pages_fork(ctx, pg, src, dst, kp)
        P.pages_extend(ctx, pg, dst, ad)
        P.kv_write(ctx, pg, 0, k, v, cu, seqs=dst)
        got.append(P.attn_decode(ctx, q, pg, 0, seqs=dst, group_off=go, shared=sh, lse=True))
    ctx.sync()
    for (keep, add, _, k, v, q), (out, lse) in zip(steps, got):
        m.free(own)
        m.fork(group, own, keep)
        m.extend(own, add)
        at = np.concatenate([[0], np.cumsum(add)])
        want = []
        for i in range(n):
            a = int(group[i]) * pre
            kk = torch.cat([k0[a:a + keep[i]], k[at[i]:at[i + 1]]])
            vv = torch.cat([v0[a:a + keep[i]], v[at[i]:at[i + 1]]])
            want.append(reference(q[i:i + 1], kk, vv, False, d ** -0.5))
        check(out, lse, want, range(n + 1))
    m.same(pg)


def test_the_longest_row(P, ctx):
    """2^31 - 8 tokens, 64 GB of keys and values.  Keys are zeros but for the last 24, values too: the sums are known.
    Beside the bounds of the other tests, the sum of 2^31 weights in up to 304 pieces: 2^-15 of it."""
    n, page, d, hq = (1 << 31) - 8, 8, 8, 4
    if torch.cuda.mem_get_info()[0] < 90 << 30:
        pytest.skip("needs 90 GB")
    g = gen(61)
    pages = n // page
    cache = torch.zeros((1, 2, pages, page, 1, d), dtype=BF, device=DEV)
    k, v = randn(g, 24, 1, d), randn(g, 24, 1, d)
    k[:, :, 0] = torch.linspace(3, 4.5, 24, device=DEV).to(BF)[:, None]
    cache[0, 0].view(-1, 1, d)[n - 24:], cache[0, 1].view(-1, 1, d)[n - 24:] = k, v
    pg = P.KVPages(cache, torch.ones(pages, dtype=torch.int32, device=DEV),
                   torch.arange(pages, dtype=torch.int32, device=DEV)[None], ints([n]))
    q = randn(g, 20, hq, d)
    q[..., 0] = 6.0
    outs = [(P.attn_decode(ctx, q[19:], pg, 0, scale=1.0, lse=True), 19),
            (P.attn_paged(ctx, q, pg, 0, ints([0, 20]), scale=1.0, lse=True), 0)]
    ctx.sync()
    for (out, lse), first in outs:
        for i in range(first, 20):
            sees = n - 20 + 1 + i
            few = sees - (n - 24)                                    # of the last 24 keys
            s = torch.einsum("hd,jd->hj", q[i].double(), k[:few, 0].double())
            z = torch.logsumexp(torch.cat([s, torch.full((hq, 1), math.log(n - 24), device=DEV, dtype=torch.float64)], 1), 1)
            p = torch.exp(s - z[:, None])
            o, a = p @ v[:few, 0].double(), p @ v[:few, 0].double().abs()
            e = torch.einsum("hd,jd->hj", q[i].double().abs(), k[:few, 0].double().abs()).amax() * 2.0 ** -18
            bound = 2.0 ** -8 * (o.abs() + a) * 1.01 + (4 * e + 2.0 ** -19 + 2.0 ** -15) * a
            got, gl = out[i - first].double(), lse[i - first].double()
            assert ((got - o).abs() <= bound).all(), (first, i)
            assert ((gl - z).abs() <= 2 * e + 2.0 ** -20 * z.abs() + 2.0 ** -18 + 2.0 ** -15).all(), (first, i)


@pytest.mark.parametrize("cu_k", [[0, 0, 0], [0, 1, 2], [0, 0, 1 << 30], [1, 1, 1]])
@pytest.mark.parametrize("causal", [True, False])
def test_no_keys_at_all_whatever_the_offsets_say(P, ctx, cu_k, causal):
    q, none = randn(gen(71), 6, 8, 64), torch.zeros((0, 2, 64), dtype=BF, device=DEV)
    out, lse = P.attn_packed(ctx, q, none, none, ints([0, 4, 6]), cu_k=ints(cu_k), causal=causal, lse=True)
    ctx.sync()
    assert (out == 0).all() and (lse == -math.inf).all()


def test_tensors_that_want_a_gradient_are_refused_where_gradients_are_recorded(P, ctx):
    g = gen(81)
    pg, _ = fill(P, ctx, g, 16, [20, 30], 2, 64, BF)
    q, k, v = randn(g, 2, 8, 64), randn(g, 2, 2, 64), randn(g, 2, 2, 64)
    cu = ints([0, 1, 2])
    calls = [("q", lambda t: P.attn_packed(ctx, t, k, v, cu)), ("k", lambda t: P.attn_packed(ctx, q, t, v, cu)),
             ("v", lambda t: P.attn_packed(ctx, q, k, t, cu)), ("q", lambda t: P.attn_paged(ctx, t, pg, 0, cu)),
             ("q", lambda t: P.attn_decode(ctx, t, pg, 0)), ("k", lambda t: P.kv_write(ctx, pg, 0, t, v, cu)),
             ("v", lambda t: P.kv_write(ctx, pg, 0, k, t, cu))]
    for name, call in calls:
        t = {"q": q, "k": k, "v": v}[name]
        want = call(t)
        asks = t.clone().requires_grad_()
        before = ctx.launches
        with pytest.raises(ValueError, match="gradient"):
            call(asks)
        assert ctx.launches == before
        with torch.no_grad():
            got = call(asks)
        also = call(asks.detach())
        ctx.sync()
        assert want is None or (torch.equal(got, want) and torch.equal(also, want))


# ---- lists of work that are longer than the plan kernel's shared memory (512 entries, blocks or groups) ----------------
@pytest.mark.parametrize("hq,hkv,d,dtype,lens", [
    (128, 1, 64, BF, [1203, 5]),                 # two tokens a block: 605 blocks of two entries
    (16, 1, 128, HF, [9001]),                    # 563 blocks of one entry
    (8, 2, 64, BF, None),                        # 1,500 entries
    (28, 4, 128, HF, None),
])
@pytest.mark.parametrize("causal", [True, False])
def test_long_lists_of_prompts(P, ctx, hq, hkv, d, dtype, lens, causal):
    r = np.random.default_rng(hq)
    lens = lens or [int(x) for x in r.integers(0, 40, 1500)]
    g, cu = gen(hq + d), np.concatenate([[0], np.cumsum(lens)])
    q, k, v = (randn(g, int(cu[-1]), h, d, dtype=dtype) for h in (hq, hkv, hkv))
    out, lse = P.attn_packed(ctx, q, k, v, ints(cu), causal=causal, lse=True)
    again = P.attn_packed(ctx, q, k, v, ints(cu), causal=causal)
    ctx.sync()
    assert torch.equal(out, again)
    if len(lens) == 1:      # the first and the last rows, and some between
        rows = [0, 1, 2, 3000, 3001, 8998, 8999, 9000]
        for i in rows:
            sees = i + 1 if causal else lens[0]
            o, l, bo, bl = reference(q[i:i + 1], k[:sees], v[:sees], False, d ** -0.5)
            assert ((out[i:i + 1].double() - o).abs() <= bo).all() and ((lse[i:i + 1].double() - l).abs() <= bl).all(), i
        return
    check(out, lse, [reference(q[a:b], k[a:b], v[a:b], causal, d ** -0.5) for a, b in zip(cu[:-1], cu[1:])], cu)


def test_long_lists_of_suffixes(P, ctx):
    r, g = np.random.default_rng(2), gen(91)
    new = [int(x) for x in r.integers(0, 30, 900)]
    lens = [n + int(x) for n, x in zip(new, r.integers(0, 200, 900))]
    pg, kv = fill(P, ctx, g, 16, lens, 2, 64, BF)
    rows = r.permutation(900)
    cu = np.concatenate([[0], np.cumsum([new[i] for i in rows])])
    q = randn(g, int(cu[-1]), 8, 64)
    out, lse = P.attn_paged(ctx, q, pg, 0, ints(cu), seqs=ints(rows), lse=True)
    ctx.sync()
    check(out, lse, [reference(q[a:b], *kv[i], True, 0.125) for i, a, b in zip(rows, cu[:-1], cu[1:])], cu)


@pytest.mark.parametrize("n,groups", [(1200, 0), (1200, 40), (1200, 512), (1300, 700), (700, 699)])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (20, 1, 128)])
def test_long_lists_of_single_tokens(P, ctx, n, groups, hq, hkv, d):
    """Entries, and groups of none to many of them, on both sides of what the plan kernel keeps."""
    r, g = np.random.default_rng(n + groups), gen(n + groups + d)
    group = np.sort(r.integers(0, groups, n)) if groups else np.arange(n)
    shared = [16 * int(x) for x in r.integers(0, 20, max(groups, 1))] if groups else [0] * n
    lens = [shared[a] + int(x) for a, x in zip(group, r.integers(0, 150, n))]
    pg, kv = fill(P, ctx, g, 16, lens, hkv, d, BF, shared=shared, group=list(group))
    q = randn(g, n, hq, d)
    kw = dict(group_off=ints(np.searchsorted(group, np.arange(groups + 1))), shared=ints(shared)) if groups else {}
    out, lse = P.attn_decode(ctx, q, pg, 0, lse=True, **kw)
    again = P.attn_decode(ctx, q, pg, 0, **kw)
    ctx.sync()
    assert torch.equal(out, again)
    check(out, lse, [reference(q[i:i + 1], *kv[i], False, d ** -0.5) for i in range(n)], range(n + 1))
