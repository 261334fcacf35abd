"""What is measured of a destination's prefix cache and the attention that reads it.

The router sends a request to a destination that holds its prompt's prefix.  There the prefix lies in pages of a
key/value cache; requests of the same key fork it, write the keys and values of their own tokens and attend over both.
Kinds of cases:

  prompt    attention over whole prompts packed back to back, causal, grouped heads (attn_packed)
  suffix    a batch of requests whose prefix is cached: the suffix' keys and values are written into pages, then the
            suffix attends over prefix and suffix (kv_write, attn_paged)
  decode    one new token for every running sequence; sequences of one key share their prefix' pages (kv_write,
            attn_decode)
  turnover  slots of finished requests are freed, new requests fork their key's prefix into them and get pages for
            their own tokens (pages_free, pages_fork, pages_extend)
  compact   live pages move to the front of the pool, tables follow (pages_compact)

Lengths, tables and page orders are made from the case alone, values from the seed.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda"


# ---- cases ---------------------------------------------------------------------------------------------------------
def listed():
    return [
        # the smallest prompt of the tiny workload, alone: latency of one call
        {"name": "prompt_one", "kind": "prompt", "n": 1, "median": 0, "pmin": 512, "pmax": 512, "hq": 32, "hkv": 8,
         "d": 128, "dtype": "bf16", "mix": 1},
        # cold requests of an interval, one batch of whole prompts from one token to thousands, heads in sevens
        {"name": "prompt_packed", "kind": "prompt", "n": 12, "median": 1024, "pmin": 1, "pmax": 4096, "hq": 28,
         "hkv": 4, "d": 128, "dtype": "fp16", "mix": 2},
        # the longest prefix of the 70B-shaped workload, uncached
        {"name": "prompt_long", "kind": "prompt", "n": 1, "median": 0, "pmin": 16384, "pmax": 16384, "hq": 32, "hkv": 8,
         "d": 128, "dtype": "bf16", "mix": 3},
        # one routed request whose median prefix is cached: 64 suffix tokens
        {"name": "suffix_one", "kind": "suffix", "n": 1, "median": 0, "pmin": 2048, "pmax": 2048, "smin": 64, "smax": 64,
         "hq": 32, "hkv": 8, "d": 128, "dtype": "bf16", "page": 16, "mix": 4},
        # a batch of routed requests, prefixes as the 70B-shaped workload has them, small heads, larger pages
        {"name": "suffix_batch", "kind": "suffix", "n": 48, "median": 2048, "pmin": 16, "pmax": 16384, "smin": 1,
         "smax": 128, "hq": 32, "hkv": 8, "d": 64, "dtype": "bf16", "page": 64, "mix": 5},
        # one running sequence: latency of one token
        {"name": "decode_one", "kind": "decode", "n": 1, "groups": 1, "median": 0, "pmin": 2048, "pmax": 2048,
         "smin": 64, "smax": 64, "hq": 32, "hkv": 8, "d": 128, "dtype": "bf16", "page": 16, "mix": 6},
        # a destination that serves four hot keys: long prefixes shared by many
        {"name": "decode_shared", "kind": "decode", "n": 128, "groups": 4, "median": 0, "pmin": 4096, "pmax": 8192,
         "smin": 64, "smax": 512, "hq": 64, "hkv": 8, "d": 128, "dtype": "bf16", "page": 16, "mix": 7},
        # most keys have one running request: long contexts of their own beside a few shared ones
        {"name": "decode_mixed", "kind": "decode", "n": 64, "groups": 45, "median": 8192, "pmin": 16, "pmax": 32768,
         "smin": 1, "smax": 2000, "hq": 28, "hkv": 4, "d": 128, "dtype": "fp16", "page": 32, "mix": 8},
        # a scheduler's step at a small destination
        {"name": "turnover_small", "kind": "turnover", "n": 16, "groups": 12, "median": 0, "pmin": 100, "pmax": 512,
         "smin": 1, "smax": 64, "pages": 2048, "page": 16, "hkv": 2, "d": 64, "layers": 2, "dtype": "bf16", "mix": 9},
        # a burst: a thousand requests forked off hundreds of keys
        {"name": "turnover_large", "kind": "turnover", "n": 1000, "groups": 128, "median": 1024, "pmin": 16,
         "pmax": 4096, "smin": 1, "smax": 128, "pages": 32768, "page": 16, "hkv": 4, "d": 128, "layers": 2,
         "dtype": "bf16", "mix": 10},
        # a small pool after some keys have left
        {"name": "compact_small", "kind": "compact", "n": 24, "median": 0, "pmin": 100, "pmax": 512, "gone": 0.4,
         "pages": 1024, "page": 16, "hkv": 2, "d": 64, "layers": 2, "dtype": "bf16", "mix": 11},
        # a large pool, half of it gone
        {"name": "compact_large", "kind": "compact", "n": 400, "median": 1024, "pmin": 16, "pmax": 8192, "gone": 0.5,
         "pages": 49152, "page": 16, "hkv": 4, "d": 128, "layers": 2, "dtype": "bf16", "mix": 12},
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return v + 1 if v == 3072 else v


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "suffix", "suffix", "decode", "decode", "turnover", "compact"])
    hkv = rng.choice([1, 2, 4, 8])
    c = {"kind": kind, "dtype": rng.choice(["bf16", "fp16"]), "hkv": hkv, "d": rng.choice([64, 128, 128]),
         "mix": rng.randrange(1 << 20)}
    if kind in ("prompt", "suffix", "decode"):
        c["hq"] = hkv * rng.choice([1, 4, 7, 8] if hkv > 2 else [1, 4, 6, 8, 16])
    if kind != "prompt":
        c["page"] = rng.choice([16, 32, 64])
    if kind == "prompt":
        hi = _log(rng, 64, 8192)
        most = max(1, min(32, int(6e9 / (c["hq"] * hi * hi))))  # the padded scores of the plain form stay below 24 GB
        n = min(most, _log(rng, 1, 32))
        c.update(n=n, median=max(1, hi // 3) if n > 1 else 0, pmin=1 if n > 1 else hi, pmax=hi)
    elif kind == "suffix":
        hi = _log(rng, 64, 16384)
        smax = _log(rng, 1, 256)
        most = max(1, min(64, int(6e9 / (c["hq"] * smax * (hi + smax)))))
        c.update(n=min(most, _log(rng, 1, 64)), median=max(16, hi // 4), pmin=min(16, hi), pmax=hi, smin=1, smax=smax)
    elif kind == "decode":
        hi = _log(rng, 64, 32768)
        n = min(_log(rng, 1, 200), max(1, int(1.0e9 / (hkv * c["d"] * hi))))
        c.update(n=n, groups=_log(rng, 1, n), median=max(16, hi // 3), pmin=min(16, hi), pmax=hi, smin=1,
                 smax=_log(rng, 1, 1000))
    else:
        hi = _log(rng, 64, 4096)
        groups = _log(rng, 4, 200)
        c.update(n=_log(rng, 4, 1000), median=max(16, hi // 3), pmin=16, pmax=hi, layers=rng.choice([1, 2]))
        if kind == "turnover":
            c.update(groups=groups, smin=1, smax=_log(rng, 1, 128))
        else:
            c.update(n=groups, gone=round(rng.uniform(0.1, 0.8), 2))
        pre, suf = _lengths(c)
        need = int(_pages(pre, c["page"]).sum() + (0 if suf is None else _pages(suf, c["page"]).sum() + c["n"]))
        c["pages"] = int(need * rng.uniform(1.1, 1.6)) + 8
    return c


def _pages(tokens, page):
    return -(-np.asarray(tokens, np.int64) // page)


def _lengths(c):
    """Prefix lengths (one for each prompt, request or key) and each request's own tokens."""
    r = np.random.RandomState(c["mix"])
    n = c["groups"] if "groups" in c else c["n"]
    if c["median"]:
        pre = np.exp(math.log(c["median"]) + 0.8 * r.standard_normal(n)).astype(np.int64)
    else:
        pre = r.randint(c["pmin"], c["pmax"] + 1, n)
    pre = np.clip(pre, c["pmin"], c["pmax"])
    suf = r.randint(c["smin"], c["smax"] + 1, c["n"]) if "smin" in c else None
    return pre, suf


def _members(c):
    """Group of each decoding sequence, in order: the hottest key has the most, every key at least one."""
    n, g = c["n"], c["groups"]
    w = 1.0 / np.arange(1, g + 1)
    size = 1 + np.floor((n - g) * w / w.sum()).astype(np.int64)
    size[0] += n - size.sum()
    return np.repeat(np.arange(g), size), np.concatenate([[0], np.cumsum(size)])


def _dtype(c):
    return {"bf16": torch.bfloat16, "fp16": torch.float16}[c["dtype"]]


# ---- inputs --------------------------------------------------------------------------------------------------------
def _values(g, shape, dtype, spread=1.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * spread).to(dtype)


def _ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)


def _heads(g, shape, dtype):
    """Keys: every head has a scale of its own, so that some heads attend to a few tokens and some to all."""
    k = torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)
    return (k * torch.linspace(0.5, 3.0, shape[-2], device=DEV)[:, None]).to(dtype)


def _cache(g, c, layers, n_pages):
    """[layers, 2, n_pages, page, heads, d]: a pool whose pages have all been used before."""
    x = torch.empty((layers, 2, n_pages, c["page"], c["hkv"], c["d"]), device=DEV, dtype=_dtype(c))
    for l in range(layers):
        x[l, 0] = _heads(g, x.shape[2:], x.dtype)
        x[l, 1] = _values(g, x.shape[2:], x.dtype)
    return x


def _paged(c, pre, suf, group):
    """Tables of sequences that share the whole pages of their group's prefix (group[i] = i: nothing shared)."""
    page = c["page"]
    r = np.random.RandomState(c["mix"] + 1)
    lens = pre[group] + suf
    width = int(_pages(lens, page).max())
    shared = pre // page
    total = int(shared.sum() + (_pages(lens, page) - shared[group]).sum())
    order = r.permutation(total)  # a pool in use hands out its pages in no order
    table = np.full((len(lens), width), -1, np.int64)
    first = np.concatenate([[0], np.cumsum(shared)])
    at = int(first[-1])
    for i, n in enumerate(_pages(lens, page)):
        s = int(shared[group[i]])
        table[i, :s] = order[first[group[i]]:first[group[i]] + s]
        table[i, s:n] = order[at:at + n - s]
        at += int(n - s)
    return lens, table, shared * page, total


def _pool(c):
    """Host state of the pool that turnover and compact start from: (ref, table, lens, src, dst, keep, add)."""
    page, n_pages = c["page"], c["pages"]
    r = np.random.RandomState(c["mix"] + 2)
    pre, suf = _lengths(c)
    keys = len(pre)
    slots = keys + (c["n"] if suf is not None else 0)
    width = int(_pages(pre, page).max() + (_pages(suf, page).max() + 1 if suf is not None else 0))
    ref, lens = np.zeros(n_pages, np.int64), np.zeros(slots, np.int64)
    table = np.full((slots, width), -1, np.int64)
    order = r.permutation(n_pages)
    at = 0
    for i in range(keys):
        k = int(_pages(pre[i], page))
        table[i, :k] = order[at:at + k]
        ref[order[at:at + k]] = 1
        lens[i] = pre[i]
        at += k
    if suf is None:
        for i in np.nonzero(r.random_sample(keys) < c["gone"])[0]:
            k = int(_pages(lens[i], page))
            ref[table[i, :k]] = 0
            table[i], lens[i] = -1, 0
        return ref, table, lens, None, None, None, None
    w = 1.0 / np.arange(1, keys + 1)
    src = r.choice(keys, c["n"], p=w / w.sum())
    keep = np.maximum(1, (pre[src] * (1 - 0.3 * r.random_sample(c["n"]) ** 2)).astype(np.int64))
    dst = keys + np.arange(c["n"])
    base = ref.copy()
    free = np.nonzero(base == 0)[0]  # the slots hold the same requests' last turn
    at = 0
    for i, s in enumerate(src):
        full = int(keep[i] // page)
        table[dst[i], :full] = table[s, :full]
        np.add.at(ref, table[s, :full], 1)
        if keep[i] % page:
            table[dst[i], full] = free[at]
            ref[free[at]] = 1
            at += 1
    for i in range(c["n"]):
        a, b = int(_pages(keep[i], page)), int(_pages(keep[i] + suf[i], page))
        table[dst[i], a:b] = free[at:at + b - a]
        ref[free[at:at + b - a]] = 1
        at += b - a
        lens[dst[i]] = keep[i] + suf[i]
    return ref, table, lens, src, dst, keep, suf


def prepare(case, seed):
    c, g = case, torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = _dtype(c)
    s = {"case": c}
    if c["kind"] == "prompt":
        lens, _ = _lengths(c)
        T = int(lens.sum())
        # one projection's output holds queries, keys and values of a token side by side
        qkv = _values(g, (T, c["hq"] + 2 * c["hkv"], c["d"]), dt)
        qkv[:, c["hq"]:c["hq"] + c["hkv"]] = _heads(g, (T, c["hkv"], c["d"]), dt)
        s.update(q=qkv[:, :c["hq"]], k=qkv[:, c["hq"]:c["hq"] + c["hkv"]], v=qkv[:, c["hq"] + c["hkv"]:],
                 cu=_ints(np.concatenate([[0], np.cumsum(lens)])), longest=int(lens.max()))
        return s
    if c["kind"] in ("suffix", "decode"):
        pre, suf = _lengths(c)
        group, off = _members(c) if c["kind"] == "decode" else (np.arange(c["n"]), None)
        lens, table, shared, total = _paged(c, pre, suf, group)
        qlen = np.ones(c["n"], np.int64) if c["kind"] == "decode" else suf
        T = int(qlen.sum())
        s.update(cache=_cache(g, c, 1, total), table=_ints(table), lens=_ints(lens),
                 cu=_ints(np.concatenate([[0], np.cumsum(qlen)])), q=_values(g, (T, c["hq"], c["d"]), dt),
                 k=_heads(g, (T, c["hkv"], c["d"]), dt), v=_values(g, (T, c["hkv"], c["d"]), dt),
                 longest=int(qlen.max()), ref=_ints(np.bincount(table[table >= 0], minlength=total)))
        if off is not None:
            s.update(off=_ints(off), shared=_ints(shared))
        return s
    ref, table, lens, src, dst, keep, add = _pool(c)
    s.update(cache=_cache(g, c, c["layers"], c["pages"]), ref=_ints(ref), table=_ints(table), lens=_ints(lens))
    if c["kind"] == "turnover":
        s.update(src=_ints(src), dst=_ints(dst), keep=_ints(keep), add=_ints(add))
    return s


# ---- the plain form ------------------------------------------------------------------------------------------------
def _pad(x, cu, longest):
    """Packed [T, h, d] as [n, h, longest, d] in 32 bits, and which places are filled."""
    i = torch.arange(longest, device=x.device)
    at = cu[:-1, None].long() + i
    filled = at < cu[1:, None]
    y = x[at.clamp_max(x.shape[0] - 1)].float().masked_fill_(~filled[:, :, None, None], 0.0)
    return y.transpose(1, 2), filled


def _softmax_product(q, k, v, seen):
    """q [n, hkv, g, m, d], k and v [n, hkv, s, d], seen [n, m, s]: rows that see nothing give zeros."""
    n, hkv, gr, m, d = q.shape
    w = (q.reshape(n, hkv, gr * m, d) * (1.0 / math.sqrt(d))) @ k.transpose(-1, -2)
    w = w.view(n, hkv, gr, m, -1)
    w.masked_fill_(~seen[:, None, None], float("-inf"))
    top = w.amax(-1, keepdim=True)
    w.sub_(top.masked_fill_(top == float("-inf"), 0.0)).exp_()
    total = w.sum(-1, keepdim=True)
    o = (w.view(n, hkv, gr * m, -1) @ v).view(n, hkv, gr, m, d)
    return o / total.masked_fill_(total == 0.0, 1.0)


def _plain_attention(q, k, v, cu, longest, klen):
    """q packed [T, hq, d]; k, v [n, hkv, s, d] in 32 bits, of which klen[i] are sequence i's; the last query sees all."""
    T, hq, d = q.shape
    n, hkv, s, _ = k.shape
    qp, _ = _pad(q, cu, longest)
    qlen = cu[1:] - cu[:-1]
    i = torch.arange(longest, device=q.device)
    j = torch.arange(s, device=q.device)
    last = i[None, :] + (klen - qlen)[:, None]
    seen = (j[None, None, :] <= last[:, :, None]) & (j[None, None, :] < klen[:, None, None])
    o = _softmax_product(qp.reshape(n, hkv, hq // hkv, longest, d), k, v, seen)
    o = o.reshape(n, hq, longest, d).transpose(1, 2)
    t = torch.arange(T, device=q.device, dtype=cu.dtype)
    seq = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    return o[seq, t - cu[seq]].to(q.dtype)


def _plain_write(s):
    cache, cu = s["cache"], s["cu"]
    page = cache.shape[3]
    t = torch.arange(s["q"].shape[0], device=cache.device, dtype=cu.dtype)
    seq = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    pos = (s["lens"][seq] - (cu[seq + 1] - t)).long()
    at = s["table"][seq, pos // page].long()
    cache[0, 0, at, pos % page] = s["k"]
    cache[0, 1, at, pos % page] = s["v"]


def _plain_paged(s):
    cache, table = s["cache"], s["table"].long().clamp_min(0)
    n, width = table.shape
    page, hkv, d = cache.shape[3:]
    kv = cache[0][:, table].view(2, n, width * page, hkv, d).transpose(2, 3).float()
    # what stands in a page behind a sequence's end is no value of it
    kv.masked_fill_((torch.arange(width * page, device=table.device) >= s["lens"][:, None])[None, :, None, :, None], 0.0)
    return _plain_attention(s["q"], kv[0], kv[1], s["cu"], s["longest"], s["lens"])


def _ceil_pages(tokens, page):
    return (tokens + (page - 1)) // page


def _take(ref, need):
    """The lowest free pages for needs in list order: for each entry where its pages begin in the order of free pages."""
    free = torch.sort((ref != 0).to(torch.int8), stable=True).indices
    return free, need.cumsum(0) - need


def _plain_free(ref, table, lens, seqs, page):
    rows = table[seqs].long()
    used = torch.arange(table.shape[1], device=ref.device) < _ceil_pages(lens[seqs], page)[:, None]
    ref.index_add_(0, rows.clamp_min(0).reshape(-1), -used.reshape(-1).to(ref.dtype))
    table[seqs] = -1
    lens[seqs] = 0


def _plain_fork(cache, ref, table, lens, src, dst, keep, page):
    full, tail = keep // page, keep % page
    j = torch.arange(table.shape[1], device=ref.device)
    free, begin = _take(ref, (tail > 0).to(torch.int32))
    new = free[begin.long()].to(table.dtype)
    rows = torch.where(j < full[:, None], table[src], -1)
    ref.index_add_(0, rows.long().clamp_min(0).reshape(-1), (rows >= 0).reshape(-1).to(ref.dtype))
    ref.index_put_((new.long(),), (tail > 0).to(ref.dtype), accumulate=True)
    rows = torch.where((j == full[:, None]) & (tail > 0)[:, None], new[:, None], rows)
    table[dst] = rows
    lens[dst] = keep
    have = (tail > 0)[:, None]
    r = torch.arange(page, device=ref.device)
    old_page = table[src].gather(1, (full - (tail == 0).to(full.dtype)).long()[:, None]).long()
    new_page = torch.where(have, new[:, None].long(), old_page)
    row = torch.where(r < tail[:, None], r, 0)  # rows behind the tail stay: the first row is written again
    cache[:, :, new_page, row] = cache[:, :, old_page, row]


def _plain_extend(ref, table, lens, seqs, add, page):
    had = _ceil_pages(lens[seqs], page)
    need = _ceil_pages(lens[seqs] + add, page) - had
    free, begin = _take(ref, need)
    j = torch.arange(table.shape[1], device=ref.device)
    rank = begin[:, None] + (j - had[:, None])
    fresh = (j >= had[:, None]) & (j < (had + need)[:, None])
    pages = free[rank.clamp(0, ref.shape[0] - 1).long()]
    table[seqs] = torch.where(fresh, pages.to(table.dtype), table[seqs])
    ref.index_add_(0, torch.where(fresh, pages, 0).reshape(-1), fresh.reshape(-1).to(ref.dtype))
    lens[seqs] = lens[seqs] + add


def _plain_compact(cache, ref, table, lens):
    live = ref > 0
    n = live.sum()
    i = torch.arange(ref.shape[0], device=ref.device)
    frm = torch.nonzero(live & (i >= n)).reshape(-1)
    to = torch.nonzero(~live & (i < n)).reshape(-1)
    page_map = torch.where(live, i, -1)
    page_map[frm] = to
    ref_out = torch.where(i < n, ref, 0)
    ref_out[to] = ref[frm]
    table_out = torch.where(table >= 0, page_map[table.long().clamp_min(0)].to(table.dtype), -1)
    cache[:, :, to] = cache[:, :, frm]
    return ref_out, table_out, page_map.to(torch.int32), n.to(torch.int32).reshape(1)


# ---- one pass ------------------------------------------------------------------------------------------------------
_kept = []


def _framework():
    if not _kept:
        import paper_2608_19677_gb300 as P
        _kept.extend((P, P.Context(0)))
    return _kept


def run(s):
    kind = s["case"]["kind"]
    if own:
        P, ctx = _framework()
        if kind == "prompt":
            return P.attn_packed(ctx, s["q"], s["k"], s["v"], s["cu"])
        if "pages" not in s:  # the program's handle of its cache
            s["pages"] = P.KVPages(s["cache"], s["ref"], s["table"], s["lens"])
        pg = s["pages"]
        if kind == "suffix":
            P.kv_write(ctx, pg, 0, s["k"], s["v"], s["cu"])
            return {"out": P.attn_paged(ctx, s["q"], pg, 0, s["cu"]), "cache": s["cache"]}
        if kind == "decode":
            P.kv_write(ctx, pg, 0, s["k"], s["v"], s["cu"])
            return {"out": P.attn_decode(ctx, s["q"], pg, 0, group_off=s["off"], shared=s["shared"]),
                    "cache": s["cache"]}
        if kind == "turnover":
            P.pages_free(ctx, pg, s["dst"])
            P.pages_fork(ctx, pg, s["src"], s["dst"], s["keep"])
            P.pages_extend(ctx, pg, s["dst"], s["add"])
            return {"ref": s["ref"], "table": s["table"], "lens": s["lens"], "cache": s["cache"]}
        ref, table, page_map, n_live = P.pages_compact(ctx, pg)
        return {"ref": ref, "table": table, "map": page_map, "n": n_live, "cache": s["cache"]}
    if kind == "prompt":
        klen = s["cu"][1:] - s["cu"][:-1]
        k, _ = _pad(s["k"], s["cu"], s["longest"])
        v, _ = _pad(s["v"], s["cu"], s["longest"])
        return _plain_attention(s["q"], k, v, s["cu"], s["longest"], klen)
    if kind in ("suffix", "decode"):
        _plain_write(s)
        return {"out": _plain_paged(s), "cache": s["cache"]}
    page = s["case"]["page"]
    if kind == "turnover":
        src, dst = s["src"].long(), s["dst"].long()
        _plain_free(s["ref"], s["table"], s["lens"], dst, page)
        _plain_fork(s["cache"], s["ref"], s["table"], s["lens"], src, dst, s["keep"], page)
        _plain_extend(s["ref"], s["table"], s["lens"], dst, s["add"], page)
        return {"ref": s["ref"], "table": s["table"], "lens": s["lens"], "cache": s["cache"]}
    ref, table, page_map, n_live = _plain_compact(s["cache"], s["ref"], s["table"], s["lens"])
    return {"ref": ref, "table": table, "map": page_map, "n": n_live, "cache": s["cache"]}


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "prompt":
        lens, _ = _lengths(c)
        T = int(lens.sum())
        return {"bytes": 2.0 * T * c["d"] * 2 * (c["hq"] + c["hkv"]),
                "flops": 4.0 * c["d"] * c["hq"] * float((lens * (lens + 1) // 2).sum())}
    if c["kind"] in ("suffix", "decode"):
        pre, suf = _lengths(c)
        if c["kind"] == "suffix":
            qlen, lens = suf, pre + suf
            tokens = int(lens.sum())
        else:
            group, _ = _members(c)
            qlen, lens = np.ones(c["n"], np.int64), pre[group] + suf
            shared = pre // c["page"] * c["page"]
            tokens = int(shared.sum() + (lens - shared[group]).sum())
        pairs = float((qlen * lens - qlen * (qlen - 1) // 2).sum())
        T = int(qlen.sum())
        # the new tokens' keys and values are read where they came from and written; the rest is read from the pages
        return {"bytes": 2.0 * c["d"] * (2 * T * c["hq"] + 2 * c["hkv"] * (tokens + T)),
                "flops": 4.0 * c["d"] * c["hq"] * pairs}
    page, row = c["page"], 2.0 * c["hkv"] * c["d"] * 2 * c["layers"]  # bytes of a token in all planes
    ref, table, lens, src, dst, keep, add = _pool(c)
    if c["kind"] == "turnover":
        held = int(_pages(keep + add, page).sum())
        return {"bytes": 2 * row * float((keep % page).sum()) + 4.0 * (2 * len(ref) + 4 * held + 6 * c["n"]), "flops": 0}
    n = int((ref > 0).sum())
    moved = int((ref[n:] > 0).sum())
    return {"bytes": 2 * row * page * moved + 4.0 * (3 * len(ref) + 2 * table.size), "flops": 0}


# ---- the definition in 64 bits -------------------------------------------------------------------------------------
def exact(case, seed):
    c = case
    if c["kind"] not in ("prompt", "suffix", "decode") or work(c)["flops"] > 6e12:
        return None
    s = prepare(c, seed)
    cu = s["cu"].tolist()
    G, d = c["hq"] // c["hkv"], c["d"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    for b in range(len(cu) - 1):
        lo, hi = cu[b], cu[b + 1]
        if hi == lo:
            continue
        if c["kind"] == "prompt":
            k, v = s["k"][lo:hi].double(), s["v"][lo:hi].double()
        else:
            n = int(s["lens"][b])
            used = s["table"][b, :-(-n // c["page"])].long()
            k = s["cache"][0, 0, used].reshape(-1, c["hkv"], d)[:n].double()
            v = s["cache"][0, 1, used].reshape(-1, c["hkv"], d)[:n].double()
            k[n - (hi - lo):], v[n - (hi - lo):] = s["k"][lo:hi].double(), s["v"][lo:hi].double()
        n = k.shape[0]
        for a in range(lo, hi, 2048):
            e = min(hi, a + 2048)
            sees = n - (hi - e)  # keys that the last query of this block sees
            hidden = torch.arange(sees, device=DEV)[None, :] > torch.arange(n - (hi - a), n - (hi - e), device=DEV)[:, None]
            for h in range(c["hq"]):
                x = (s["q"][a:e, h].double() @ k[:sees, h // G].T) / math.sqrt(d)
                x[hidden] = float("-inf")
                out[a:e, h] = torch.softmax(x, -1) @ v[:sees, h // G]
    return out if c["kind"] == "prompt" else {"out": out, "cache": None}
