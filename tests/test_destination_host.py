"""The bookkeeping of a destination's server, on the host: the library's calls are replaced by a model of the pages that
keeps, for every row, which request's text stands at each of its tokens."""
from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")


class Pool:
    """Pages, tables and lengths as the calls leave them; ``text``: what was written at each place of each page."""

    def __init__(self, n_pages, page, n_seqs, max_pages):
        self.page, self.n_pages, self.layers = page, n_pages, 1
        self.table = torch.full((n_seqs, max_pages), -1, dtype=torch.int32)
        self.lens = torch.zeros(n_seqs, dtype=torch.int32)
        self.ref = torch.zeros(n_pages, dtype=torch.int32)
        self.text = torch.full((n_pages, page), -1, dtype=torch.int64)
        self.calls = []

    def _take(self):
        p = int((self.ref == 0).nonzero()[0])
        self.ref[p] = 1
        return p

    def extend(self, ctx, pages, seqs, add):
        self.calls.append(("extend", seqs.tolist(), add.tolist()))
        for s, a in zip(seqs.tolist(), add.tolist()):
            n = int(self.lens[s])
            assert n + a <= self.table.shape[1] * self.page, "the row cannot hold it"
            for j in range(-(-n // self.page), -(-(n + a) // self.page)):
                self.table[s, j] = self._take()
            self.lens[s] = n + a

    def fork(self, ctx, pages, src, dst, keep):
        self.calls.append(("fork", src.tolist(), dst.tolist(), keep.tolist()))
        for s, d, n in zip(src.tolist(), dst.tolist(), keep.tolist()):
            assert self.lens[d] == 0 and 1 <= n <= self.lens[s], "a fork the pages refuse"
            full, tail = divmod(n, self.page)
            self.table[d, :full] = self.table[s, :full]
            self.ref[self.table[s, :full].long()] += 1
            if tail:
                p = self._take()
                self.table[d, full] = p
                self.text[p, :tail] = self.text[self.table[s, full], :tail]
            self.lens[d] = n

    def free(self, ctx, pages, seqs):
        self.calls.append(("free", seqs.tolist()))
        for s in seqs.tolist():
            used = self.table[s, :-(-int(self.lens[s]) // self.page)].long()
            assert (self.ref[used] > 0).all()
            self.ref[used] -= 1
            self.table[s], self.lens[s] = -1, 0

    def at(self, row, pos):
        return int(self.table[row, pos // self.page]), pos % self.page

    def write(self, ctx, pages, layer, k, v, cu, seqs=None):
        cu = cu.tolist()
        assert cu[-1] == k.shape[0]
        for i, row in enumerate(seqs.tolist()):
            for t in range(cu[i], cu[i + 1]):
                p, r = self.at(row, int(self.lens[row]) - (cu[i + 1] - t))
                assert self.ref[p] == 1, "a page that other rows read"
                self.text[p, r] = int(k[t, 0, 0])

    def read(self, row, n):
        return [int(self.text[self.at(row, j)]) for j in range(n)]

    def paged(self, ctx, q, pages, layer, cu, seqs=None, **kw):
        return q

    def decode(self, ctx, q, pages, layer, seqs=None, group_off=None, shared=None, **kw):
        """What each query reads: its group's first row's shared tokens, then its own."""
        rows, off, shared = seqs.tolist(), group_off.tolist(), shared.tolist()
        self.seen = {}
        for g, n in enumerate(shared):
            for row in rows[off[g]:off[g + 1]]:
                mine = self.read(row, int(self.lens[row]))
                self.seen[row] = self.read(rows[off[g]], n) + mine[n:]
        return q


class Model:
    """Keys are the tokens themselves."""
    layers = 1

    def embed(self, tokens):
        return tokens

    def qkv(self, layer, x):
        y = x.to(torch.int64)[:, None, None]
        return y, y, y

    def mix(self, layer, x, out):
        return x


@pytest.fixture
def serve(monkeypatch):
    from paper_2608_19677_gb300 import destination as D

    def make(n_pages=64, page=16, n_seqs=8, max_pages=8):
        pool = Pool(n_pages, page, n_seqs, max_pages)
        for name in ("extend", "fork", "free"):
            monkeypatch.setattr(D, f"pages_{name}", getattr(pool, name))
        monkeypatch.setattr(D, "kv_write", pool.write)
        monkeypatch.setattr(D, "attn_paged", pool.paged)
        monkeypatch.setattr(D, "attn_decode", pool.decode)
        return D.Destination(SimpleNamespace(), pool, Model()), pool

    return make


def text(seed, n):
    return torch.arange(n, dtype=torch.int64) + 1000 * seed


def prompt(seed, prefix, plen, own):
    return torch.cat([prefix[:plen], text(seed, own)])


@pytest.mark.parametrize("kept", [(32, 16), (16, 32), (48, 33), (47, 15), (48, 48)])
def test_requests_that_keep_different_parts_of_a_prefix_read_their_own_tokens(serve, kept):
    d, pool = serve()
    prefix = text(1, 48)
    rows, _ = d.admit([(5, prompt(2, prefix, 48, 3), 48)])
    said = {rows[0]: prompt(2, prefix, 48, 3).tolist()}
    for i, n in enumerate(kept):
        (row,), _ = d.admit([(5, prompt(3 + i, prefix, n, 20 + i), n)])
        said[row] = prompt(3 + i, prefix, n, 20 + i).tolist()
    d.finish(rows)
    del said[rows[0]]
    for step in range(3):
        new = text(9 + step, len(said))
        for row, t in zip(d.order(), new.tolist()):
            said[row].append(t)
        d.step(new)
        assert pool.seen == said


def state(d, pool):
    return (list(d.free_rows), d.free_pages, dict(d.prefixes), {k: list(v) for k, v in d.running.items()}, dict(d.own),
            dict(d.kept), pool.table.tolist(), pool.lens.tolist(), pool.ref.tolist(), list(pool.calls))


@pytest.mark.parametrize("plen,whole", [(0, 40), (-3, 40), (41, 40), (33, 60), (48, 48)])
def test_prefix_lengths_that_cannot_be_are_refused_before_anything_changes(serve, plen, whole):
    """None, more than the prompt, and more than is held of the key."""
    d, pool = serve()
    d.admit([(5, text(1, 40), 32)])
    before = state(d, pool)
    with pytest.raises(ValueError):
        d.admit([(6, text(2, 20), 16), (5, text(1, whole), plen)])
    assert state(d, pool) == before


def test_a_new_prefix_is_read_as_far_as_the_longest_request_of_the_call_keeps_it(serve):
    d, pool = serve()
    prefix = text(1, 48)
    asked = [(5, prompt(2 + i, prefix, n, 4), n) for i, n in enumerate((16, 48, 20))]
    rows, _ = d.admit(asked)
    assert d.prefixes[5][1] == 48 and pool.read(d.prefixes[5][0], 48) == prefix.tolist()
    assert [pool.read(r, int(pool.lens[r])) for r in rows] == [t.tolist() for _, t, _ in asked]


def test_requests_and_steps_that_a_row_cannot_hold_are_refused_before_anything_changes(serve):
    """Rows of four pages of 16 tokens, whose pool has many more."""
    d, pool = serve(max_pages=4)
    rows, _ = d.admit([(5, text(1, 63), 32)])
    before = state(d, pool)
    for asked in ([(5, text(1, 65), 32)], [(6, text(2, 20), 16), (7, text(3, 130), 64)]):
        with pytest.raises(RuntimeError):
            d.admit(asked)
        assert state(d, pool) == before
    d.step(text(2, 1))
    assert int(pool.lens[rows[0]]) == 64
    before = state(d, pool)
    with pytest.raises(RuntimeError):
        d.step(text(3, 1))
    assert state(d, pool) == before


def test_only_running_requests_are_finished_each_once(serve):
    """Not a prefix' row, an empty one, or one twice."""
    d, pool = serve()
    rows, _ = d.admit([(5, text(1, 40), 32), (5, text(1, 36), 32)])
    before = state(d, pool)
    for asked in ([d.prefixes[5][0]], [rows[0], rows[0]], [rows[1], d.free_rows[0]], [rows[0], 99], [-1]):
        with pytest.raises(ValueError):
            d.finish(asked)
        assert state(d, pool) == before
    d.finish([])
    assert state(d, pool) == before
    d.finish(rows)
    assert not d.running and not d.kept and int(pool.ref.sum()) == 2


class Failing(Model):
    """Raises at its n-th pass."""

    def __init__(self):
        self.left = -1

    def mix(self, layer, x, out):
        self.left -= 1
        if self.left == 0:
            raise ArithmeticError
        return x


@pytest.mark.parametrize("at", [1, 2])
def test_a_call_that_fails_leaves_nothing_half_read(serve, at):
    """While a prefix is read, and while the requests' own tokens are: neither may be found there later."""
    d, pool = serve()
    d.model = Failing()
    d.admit([(4, text(1, 30), 20)])
    ref, lens, held = pool.ref.clone(), pool.lens.clone(), dict(d.prefixes)
    d.model.left = at
    with pytest.raises(ArithmeticError):
        d.admit([(5, text(2, 40), 32), (4, text(1, 25), 20)])
    assert torch.equal(pool.ref, ref) and torch.equal(pool.lens, lens) and d.prefixes == held
    assert d.free_pages == int((pool.ref == 0).sum()) and len(d.free_rows) == 6 and list(d.running) == [4]
    (row,), _ = d.admit([(5, text(2, 40), 32)])
    assert pool.read(row, 40) == text(2, 40).tolist()


def test_a_step_that_fails_gives_its_requests_up(serve):
    d, pool = serve()
    d.model = Failing()
    d.admit([(4, text(1, 30), 20), (5, text(2, 32), 32)])
    before = state(d, pool)
    with pytest.raises(ValueError):
        d.step(text(3, 3))
    assert state(d, pool) == before
    d.model.left = 1
    with pytest.raises(ArithmeticError):
        d.step(text(3, 2))
    assert not d.running and not d.kept and set(d.prefixes) == {4, 5} and len(d.free_rows) == 6
    assert d.free_pages == int((pool.ref == 0).sum()) == 64 - 4


def test_arguments_may_be_named(serve):
    d, _ = serve()
    rows, _ = d.admit(requests=[(5, text(1, 40), 32)])
    d.step(tokens=text(2, 1))
    d.finish(rows=rows)
    assert not d.running
