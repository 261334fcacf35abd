"""Requests of a synthetic trace routed by the library, and served by one of their destinations.

  python examples/serve_prefixes.py [--requests 96] [--steps 4] [--rotary] [--bits 8]

Keys are hashed from the prompts, an LPT plan is built from them, the requests are dispatched, and destination 0 serves
its share with a small two-layer attention model (random weights): it reads each key's prefix once, forks it for every
request of the key, and decodes a few tokens with the shared prefixes read once per step.  Every output is compared with
the same model computed from scratch in 64 bits; the script prints the largest relative error.  With --rotary the model
has rotary positions, with --bits 8 the destination holds keys and values in 8 bits (half the memory, errors of a few
per cent in this small model).
"""
from __future__ import annotations

import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


class TinyAttention:
    """Embedding, and per layer x + W_o attention(W_q x, W_k x, W_v x), with rotary positions or without."""

    def __init__(self, torch, dev, layers=2, heads=8, kv_heads=2, dim=64, width=256, vocab=4096, seed=0, rotary=None):
        g = torch.Generator(device=dev)
        g.manual_seed(seed)
        self.torch, self.layers, self.heads, self.kv_heads, self.dim = torch, layers, heads, kv_heads, dim
        self.rotary = rotary
        r = lambda *s: (torch.randn(s, generator=g, device=dev) / s[0] ** 0.5).to(torch.bfloat16)  # noqa: E731
        self.table = torch.randn((vocab, width), generator=g, device=dev).to(torch.bfloat16)
        self.wq = [r(width, heads * dim) for _ in range(layers)]
        self.wk = [r(width, kv_heads * dim) for _ in range(layers)]
        self.wv = [r(width, kv_heads * dim) for _ in range(layers)]
        self.wo = [r(heads * dim, width) for _ in range(layers)]

    def embed(self, tokens):
        return self.table[tokens]

    def qkv(self, layer, x):
        T = x.shape[0]
        return ((x @ self.wq[layer]).view(T, self.heads, self.dim), (x @ self.wk[layer]).view(T, self.kv_heads, self.dim),
                (x @ self.wv[layer]).view(T, self.kv_heads, self.dim))

    def mix(self, layer, x, out):
        return x + out.reshape(x.shape[0], self.heads * self.dim) @ self.wo[layer]

    def rotated(self, x):
        """Tokens 0 .. of a sequence at their positions, in 64 bits (pairs half a head apart)."""
        if self.rotary is None:
            return x
        torch, r = self.torch, self.rotary.dims
        f = torch.tensor(self.rotary.frequencies, dtype=torch.float64, device=x.device)
        angle = torch.arange(x.shape[0], dtype=torch.float64, device=x.device)[:, None, None] * f
        a, b, rest = x[..., :r // 2], x[..., r // 2:r], x[..., r:]
        cos, sin = torch.cos(angle) * self.rotary.scale, torch.sin(angle) * self.rotary.scale
        return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)

    def exact(self, tokens):
        """The whole sequence at once, in 64 bits."""
        torch = self.torch
        x = self.table[tokens].double()
        T = x.shape[0]
        for l in range(self.layers):
            q = self.rotated((x @ self.wq[l].double()).view(T, self.heads, self.dim))
            k, v = ((x @ w.double()).view(T, self.kv_heads, self.dim) for w in (self.wk[l], self.wv[l]))
            k, v = (y.repeat_interleave(self.heads // self.kv_heads, 1) for y in (self.rotated(k), v))
            s = torch.einsum("ihd,jhd->hij", q, k) * self.dim ** -0.5
            s.masked_fill_(torch.ones((T, T), dtype=torch.bool, device=x.device).triu(1), float("-inf"))
            x = x + torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), v).reshape(T, -1) @ self.wo[l].double()
        return x


def main(n_requests: int = 96, steps: int = 4, log=print, rotary: bool = False, bits: int = 16) -> float:
    import numpy as np
    import torch
    import paper_2608_19677_gb300 as P
    import tracegen as tg
    from paper_2608_19677_gb300.destination import Destination

    dev = torch.device("cuda", 0)
    ctx = P.Context(0)
    cfg = tg.CONFIGS["tiny"].scaled(n_requests, 1)
    tr = tg.Trace(cfg)
    iv = tr.interval(0)
    tok, off = tg.arena_host(tr, iv, 4)
    d_tok = torch.from_numpy(tok).to(dev)
    keys = P.hash_prefixes(ctx, d_tok, torch.from_numpy(off.view(np.int64)).to(dev),
                           torch.from_numpy(iv.plen.view(np.int32)).to(dev))
    plan = P.build_plan(ctx, keys, P.plan_params(cfg.R, cfg.W, 5 * n_requests, 4 * cfg.R))
    load = torch.zeros((1, cfg.R), dtype=torch.int64, device=dev)
    dest = P.route_batch(ctx, [plan], ["CR"], [0], cfg.R, keys, 0, 1024, load)
    ctx.sync()
    mine = np.nonzero(dest[0].cpu().numpy().view(np.uint16) == 0)[0]
    hkeys = keys.cpu().tolist()

    model = TinyAttention(torch, dev, rotary=P.Rotary(64, scaling="ramp", factor=4.0, original=256) if rotary else None)
    prompts = [d_tok[int(off[i]):int(off[i]) + int(iv.plen[i]) + int(iv.slen[i])].long() % 4096 for i in mine]
    pages = P.KVPages.empty(4096, 16, 2 * len(mine) + 1, 64, model.layers, model.kv_heads, model.dim, bits=bits)
    server = Destination(ctx, pages, model)
    rows, out = server.admit([(hkeys[i], t, int(iv.plen[i])) for i, t in zip(mine, prompts)])
    at, worst = 0, 0.0
    text = dict(zip(rows, prompts))

    def off_by(got, want):
        return float((got.double() - want).norm() / want.norm())

    for i, row in zip(mine, rows):
        n = int(iv.slen[i])
        worst = max(worst, off_by(out[at:at + n], model.exact(text[row])[-n:]))
        at += n
    for s in range(steps):
        order = server.order()
        new = torch.tensor([(7919 * row + 104729 * s + 1) % 4096 for row in order], device=dev)
        got = server.step(new)
        for j, row in enumerate(order):
            text[row] = torch.cat([text[row], new[j:j + 1]])
            worst = max(worst, off_by(got[j], model.exact(text[row])[-1]))
        if s == 0 and len(order) > 3:   # some requests end, and the pool is compacted under the others
            server.finish(order[1::3])
            live = server.compact()
            ctx.sync()
            log(f"{int(live)} live pages after {len(order[1::3])} of {len(order)} requests have ended")
    ctx.sync()
    log(f"destination 0 of {cfg.R}: {len(mine)} of {n_requests} requests, {len(server.prefixes)} prefixes, "
        f"{ctx.launches} kernel launches, largest relative error {worst:.4f}")
    ctx.close()
    return worst


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=96)
    ap.add_argument("--steps", type=int, default=4)
    ap.add_argument("--rotary", action="store_true")
    ap.add_argument("--bits", type=int, default=16, choices=(8, 16))
    a = ap.parse_args()
    main(a.requests, a.steps, rotary=a.rotary, bits=a.bits)
