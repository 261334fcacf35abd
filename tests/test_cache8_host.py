"""Host side of rotary positions and of pages in 8 bits: structures, refusals, frequencies, and the writing kernel's
index arithmetic compiled for the host."""
import ctypes
import math
import os
import struct
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_19677_gb300", "csrc")

PROGRAM = r"""
#include <stddef.h>
#include <stdio.h>
#include "cacheroute.h"
#define F(s, f) printf("%s.%s %zu %zu\n", #s, #f, offsetof(s, f), sizeof(((s *)0)->f))
int main(void)
{
    printf("cr_kv_pages %zu\ncr_rotary %zu\ncr_append_args %zu\n", sizeof(cr_kv_pages), sizeof(cr_rotary), sizeof(cr_append_args));
    printf("cr_rope_args %zu\ncr_read_args %zu\n", sizeof(cr_rope_args), sizeof(cr_read_args));
    F(cr_rope_args, d_x); F(cr_rope_args, d_out); F(cr_rope_args, d_pos); F(cr_rope_args, x_token); F(cr_rope_args, x_head);
    F(cr_rope_args, o_token); F(cr_rope_args, o_head); F(cr_rope_args, n_tokens); F(cr_rope_args, heads);
    F(cr_rope_args, head_dim); F(cr_rope_args, dtype);
    F(cr_read_args, d_k); F(cr_read_args, d_v); F(cr_read_args, d_cu); F(cr_read_args, d_seqs); F(cr_read_args, d_start);
    F(cr_read_args, k_token); F(cr_read_args, k_head); F(cr_read_args, v_token); F(cr_read_args, v_head);
    F(cr_read_args, n); F(cr_read_args, n_tokens);
    F(cr_append_args, q_head); F(cr_append_args, o_head); F(cr_append_args, k_head); F(cr_append_args, v_token);
    F(cr_kv_pages, d_scale); F(cr_kv_pages, block); F(cr_kv_pages, reserved);
    F(cr_rotary, d_turn); F(cr_rotary, pairs); F(cr_rotary, layout); F(cr_rotary, inverse); F(cr_rotary, scale);
    F(cr_append_args, d_q); F(cr_append_args, d_q_out); F(cr_append_args, d_k); F(cr_append_args, d_v);
    F(cr_append_args, q_token); F(cr_append_args, o_token); F(cr_append_args, k_token); F(cr_append_args, v_head);
    F(cr_append_args, d_cu); F(cr_append_args, d_seqs); F(cr_append_args, n); F(cr_append_args, n_tokens);
    F(cr_append_args, q_heads); F(cr_append_args, reserved);
    return 0;
}
"""


@pytest.fixture(scope="module")
def header(tmp_path_factory):
    d = tmp_path_factory.mktemp("abi")
    src, exe = d / "abi.c", d / "abi"
    src.write_text(PROGRAM)
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout
    return {line.split()[0]: tuple(int(x) for x in line.split()[1:]) for line in out.splitlines()}


def test_structures_are_laid_out_as_the_header_declares_them(header):
    import paper_2608_19677_gb300 as P
    for name, kind in (("cr_kv_pages", P.KVPagesDesc), ("cr_rotary", P.RotaryDesc)):
        assert header[name] == (ctypes.sizeof(kind),)
        for key, place in header.items():
            if key.startswith(name + "."):
                field = getattr(kind, key.split(".")[1])
                assert place == (field.offset, field.size), key
    for name, pack, fields in (
            ("cr_append_args", P._pack_append, "d_q d_q_out d_k d_v q_token q_head o_token o_head k_token k_head v_token v_head "
                                               "d_cu d_seqs n n_tokens q_heads reserved"),
            ("cr_rope_args", P._pack_rope, "d_x d_out d_pos x_token x_head o_token o_head n_tokens heads head_dim dtype"),
            ("cr_read_args", P._pack_read, "d_k d_v d_cu d_seqs d_start k_token k_head v_token v_head n n_tokens")):
        fields = fields.split()
        packed = pack(*range(1, len(fields) + 1))
        assert header[name] == (len(packed),)
        for field in fields:
            at, size = header[f"{name}.{field}"]
            value = struct.unpack({4: "<I", 8: "<Q"}[size], packed[at:at + size])[0]
            assert value == fields.index(field) + 1, (name, field)


def test_calls_refuse_a_missing_context():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_19677_gb300 as P
    L = P.lib()
    assert L.cr_rope(None, None, None) == P.CR_EINVAL
    assert L.cr_kv_append(None, None, 0, None, None) == P.CR_EINVAL
    assert L.cr_kv_read(None, None, 0, None) == P.CR_EINVAL


# ---- frequencies ---------------------------------------------------------------------------------------------------
def turns(r):
    """Radians a token that the integers stand for."""
    return [(int(t) % 2 ** 64) / 2.0 ** 64 * 2 * math.pi for t in r.turn.tolist()]


@pytest.fixture(scope="module")
def P():
    pytest.importorskip("torch")
    import paper_2608_19677_gb300 as P
    return P


def test_frequencies(P):
    r = P.Rotary(64, base=500000.0, device="cpu")
    want = [500000.0 ** (-2.0 * i / 64) for i in range(32)]
    # a share of a turn is a double rounded to 2^-64: 2^-53 of it and 2^-65 turns
    for got, w in zip(turns(r), want):
        assert abs(got - w) <= w * 2.0 ** -50 + 2.0 ** -62
    assert r.scale == 1.0
    quarter = P.Rotary(64, base=500000.0, scaling="linear", factor=4.0, device="cpu")
    for got, w in zip(turns(quarter), want):
        assert abs(got - w / 4) <= w * 2.0 ** -50 + 2.0 ** -62
    ntk = P.Rotary(64, base=500000.0, scaling="ntk", factor=4.0, device="cpu")
    assert abs(turns(ntk)[0] - 1.0) < 1e-12                                  # the fastest pair stays
    assert abs(turns(ntk)[-1] * 4 / want[-1] - 1) < 1e-9                     # the slowest is stretched by the factor
    ramp = P.Rotary(64, base=500000.0, scaling="ramp", factor=8.0, original=4096, device="cpu")
    for got, w in zip(turns(ramp), want):
        t = 4096 * w / (2 * math.pi)
        k = min(1.0, max(0.0, (t - 1) / 31))
        assert abs(got - (w * k + w / 8 * (1 - k))) <= w * 2.0 ** -50 + 2.0 ** -62
    assert ramp.scale == 0.1 * math.log(8.0) + 1.0
    assert P.Rotary(64, scaling="ramp", factor=8.0, original=4096, scale=0.5, device="cpu").scale == 0.5


def test_frequencies_of_the_callers(P):
    f = [7.0, -0.25, 2 * math.pi, 1e-9]
    got = P.Rotary(8, frequencies=f, device="cpu").turn.tolist()
    for t, x in zip(got, f):   # any number of turns a token, either way
        d = (t - x / (2 * math.pi) * 2.0 ** 64) % 2.0 ** 64
        assert min(d, 2.0 ** 64 - d) <= 2.0 ** 13
    back = P.Rotary(8, frequencies=f, device="cpu").inverse()
    assert back._desc.inverse == 1 and back.inverse()._desc.inverse == 0


@pytest.mark.parametrize("wrong", [dict(dims=12), dict(dims=0), dict(dims=136), dict(layout="both"), dict(scaling="dynamic"),
                                   dict(factor=0.0), dict(base=-1.0), dict(base=math.inf), dict(scaling="ramp", factor=2.0),
                                   dict(scaling="ramp", factor=2.0, original=4096, slow=4.0, fast=4.0),
                                   dict(frequencies=[1.0] * 31), dict(frequencies=[math.nan] * 32),
                                   dict(frequencies=[1.0] * 32, scaling="ntk"), dict(scale=math.inf)])
def test_rotary_refuses(P, wrong):
    with pytest.raises(ValueError):
        P.Rotary(**{"dims": 64, "device": "cpu", **wrong})


def test_pages_refuse(P):
    for wrong in (dict(bits=4), dict(block=16), dict(bits=8, block=32), dict(bits=8, block=4), dict(bits=8, block=12),
                  dict(bits=8, dtype=__import__("torch").float32)):
        with pytest.raises(ValueError):
            P.KVPages.empty(4, 16, 2, 2, 1, 1, 64, device="cpu", **wrong)


# ---- slots ---------------------------------------------------------------------------------------------------------
def test_slots_cover_every_token_once(tmp_path):
    """Every token of every entry is in exactly one slot of the entry that the search finds, also where a row has fewer
    tokens than the entry writes, and no slot lies behind those that the call launches."""
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text('#include <stdint.h>\n#include <stdlib.h>\n#include <vector>\n#include "cr_attn_index.cuh"\n' + r"""
    int main()
    {
        srand(1);
        for (int trial = 0; trial < 4000; ++trial) {
            const unsigned log2 = 3 + rand() % 6, n = 1 + rand() % 6;
            std::vector<int> cu(n + 1), len(n);
            for (unsigned i = 0; i < n; ++i) {
                const int kind = rand() % 4, m = kind == 0 ? 0 : kind == 1 ? 1 : rand() % (kind == 2 ? 20 : 1500);
                cu[i + 1] = cu[i] + m;
                len[i] = rand() % 5 == 0 ? rand() % (m + 1) : m + rand() % 3000;
                if (rand() % 50 == 0) len[i] = 2147483640;
            }
            const long long total = ((long long)cu[n] >> log2) + 2ll * n;
            std::vector<int> seen(cu[n], 0);
            for (long long s = 0; s < total; ++s) {
                unsigned e = 0;
                for (unsigned i = 0; i < n; ++i)
                    if (cr_slot_of(cu[i], i, log2) <= (unsigned long long)s) e = i;
                const unsigned long long mine = cr_slot_of(cu[e], e, log2);
                if ((unsigned long long)s < mine) return 1;
                const int m = cu[e + 1] - cu[e];
                const cr_positions at = cr_slot_positions(len[e], m, s - mine, log2);
                if (at.begin >= at.end) continue;
                if (at.begin < 0 && at.end > 0) return 2;
                if ((at.begin >> log2) != ((at.end - 1) >> log2)) return 3;
                for (long long p = at.begin; p < at.end; ++p) {
                    const long long t = cu[e + 1] - (len[e] - p);
                    if (t < cu[e] || t >= cu[e + 1]) return 4;
                    ++seen[t];
                }
            }
            for (int x : seen)
                if (x != 1) return 5;
        }
        return 0;
    }
    """)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", CSRC, str(src), "-o",
                    str(exe)], check=True)
    subprocess.run([str(exe)], check=True)


def test_no_load_takes_the_path_for_data_that_nothing_writes():
    """As the attention kernels: kernels may still write what these read when they become resident."""
    for name in ("cr_kv.cu", "cr_pages.cuh"):
        text = open(os.path.join(CSRC, name)).read()
        assert not [w for w in ("__ldg(", "ld.global.nc", "__restrict__") if w in text], name


# ---- a destination that rotates, and prefixes that move ----------------------------------------------------------------
def test_a_model_with_rotary_positions_is_appended(monkeypatch):
    torch = pytest.importorskip("torch")
    from test_destination_host import Model, Pool, text
    from paper_2608_19677_gb300 import destination as D

    class Turning(Model):
        rotary = object()

    pool, said = Pool(64, 16, 8, 8), []

    def append(ctx, pages, layer, q, k, v, rotary, cu, seqs=None):
        said.append(rotary)
        pool.write(ctx, pages, layer, k, v, cu, seqs=seqs)
        return -q

    def paged(ctx, q, pages, layer, cu, seqs=None):
        assert (q <= 0).all(), "the rotated queries"
        return q

    for name in ("extend", "fork", "free"):
        monkeypatch.setattr(D, f"pages_{name}", getattr(pool, name))
    monkeypatch.setattr(D, "kv_append", append)
    monkeypatch.setattr(D, "kv_write", lambda *a, **k: pytest.fail("keys that are not rotated"))
    monkeypatch.setattr(D, "attn_paged", paged)
    d = D.Destination(None, pool, Turning())
    (row,), _ = d.admit([(5, text(1, 40), 32)])
    assert pool.read(row, 40) == text(1, 40).tolist()
    assert len(said) == 2 and all(r is Turning.rotary for r in said)


def test_prefixes_move_between_destinations(monkeypatch):
    torch = pytest.importorskip("torch")
    from test_destination_host import Model, Pool, text
    from paper_2608_19677_gb300 import destination as D
    pools = [Pool(12, 16, 4, 4) for _ in range(2)]
    for name in ("extend", "fork", "free"):
        monkeypatch.setattr(D, f"pages_{name}", lambda ctx, pages, *a, name=name: getattr(pages, name)(ctx, pages, *a))
    monkeypatch.setattr(D, "kv_write", lambda ctx, pages, *a, **k: pages.write(ctx, pages, *a, **k))
    monkeypatch.setattr(D, "attn_paged", lambda ctx, q, pages, *a, **k: q)

    def read(ctx, pages, layer, cu, seqs=None, tokens=None):
        assert cu.tolist() == [0, tokens]
        x = torch.tensor(pages.read(int(seqs[0]), tokens))[:, None, None]
        return x, x

    monkeypatch.setattr(D, "kv_read", read)
    a, b = (D.Destination(None, p, Model()) for p in pools)
    rows, _ = a.admit([(5, text(1, 40), 37)])
    a.finish(rows)
    kv = a.export(5)
    b.install(5, kv)
    row, n = b.prefixes[5]
    assert n == 37 and pools[1].read(row, 37) == text(1, 37).tolist() and b.free_pages == 12 - 3
    (mine,), _ = b.admit([(5, torch.cat([text(1, 37), text(2, 4)]), 37)])
    assert pools[1].read(mine, 41) == text(1, 37).tolist() + text(2, 4).tolist()
    before = dict(b.prefixes), b.free_pages, list(b.free_rows)
    for wrong in (lambda: b.install(5, kv), lambda: b.install(6, kv + kv), lambda: b.install(6, [(kv[0][0], kv[0][1][:3])]),
                  lambda: b.install(6, [(kv[0][0][:0], kv[0][1][:0])]), lambda: a.export(6)):
        with pytest.raises(ValueError):
            wrong()
    with pytest.raises(RuntimeError):
        b.install(6, [(text(3, 65)[:, None, None],) * 2])    # wider than a row
    monkeypatch.setattr(D, "kv_write", lambda *a, **k: (_ for _ in ()).throw(ValueError("another shape")))
    with pytest.raises(ValueError):
        b.install(6, kv)                                      # given up
    assert (dict(b.prefixes), b.free_pages, sorted(b.free_rows)) == (before[0], before[1], sorted(before[2]))
