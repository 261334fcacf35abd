"""CPU checks of the prefix-cache calls' binding: structures laid out as the header declares them."""
import ctypes
import os
import struct
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <stddef.h>
#include <stdio.h>
#include "cacheroute.h"
#define F(s, f) printf("%s.%s %zu %zu\n", #s, #f, offsetof(s, f), sizeof(((s *)0)->f))
int main(void)
{
    printf("cr_kv_pages %zu\ncr_attn_args %zu\n", sizeof(cr_kv_pages), sizeof(cr_attn_args));
    F(cr_kv_pages, d_cache); F(cr_kv_pages, d_lens); F(cr_kv_pages, dtype); F(cr_kv_pages, max_pages);
    F(cr_kv_pages, layer_stride); F(cr_kv_pages, head_stride);
    F(cr_attn_args, d_q); F(cr_attn_args, d_seqs); F(cr_attn_args, n); F(cr_attn_args, causal); F(cr_attn_args, scale);
    F(cr_attn_args, reserved); F(cr_attn_args, q_token); F(cr_attn_args, o_head);
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


def test_kv_pages_layout(header):
    import paper_2608_19677_gb300 as P
    assert header["cr_kv_pages"] == (ctypes.sizeof(P.KVPagesDesc),)
    for f in ("d_cache", "d_lens", "dtype", "max_pages", "layer_stride", "head_stride"):
        field = getattr(P.KVPagesDesc, f)
        assert header[f"cr_kv_pages.{f}"] == (field.offset, field.size), f


def test_attn_args_layout(header):
    import paper_2608_19677_gb300 as P
    values = (11, 12, 13, 14, 15, 1, 2, 3, 4, 0.5, 0, 21, 22, 23, 24)
    packed = P._pack_attn(*values)
    assert header["cr_attn_args"] == (len(packed),)
    names = ("d_q", "d_o", "d_lse", "d_cu_q", "d_seqs", "n", "n_tokens", "q_heads", "causal", "scale", "reserved",
             "q_token", "q_head", "o_token", "o_head")
    want = dict(zip(names, values))
    for f in ("d_q", "d_seqs", "n", "causal", "scale", "reserved", "q_token", "o_head"):
        at, size = header[f"cr_attn_args.{f}"]
        kind = "<f" if f == "scale" else {4: "<I", 8: "<Q"}[size]
        assert struct.unpack(kind, packed[at:at + size])[0] == want[f], f


def test_calls_refuse_a_missing_context():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_19677_gb300 as P
    L = P.lib()
    assert L.cr_pages_free(None, None, None, 0) == P.CR_EINVAL
    assert L.cr_kv_write(None, None, 0, None, 0, 0, None, 0, 0, None, None, 0, 0) == P.CR_EINVAL
    assert L.cr_attn_decode(None, None, 0, None, None, None, 0) == P.CR_EINVAL
