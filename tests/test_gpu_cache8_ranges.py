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

from test_gpu_cache8 import BF, DEV, HF, P, check, ctx, cum, fails, fill8, gen, ints, randn, reference  # noqa: E402,F401


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
