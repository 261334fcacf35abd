"""A destination's server on the GPU: every output against the model from scratch in 64 bits, on contexts whose stream is
torch's current one and on contexts with a stream of their own."""
import math

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytestmark = [pytest.mark.gpu, pytest.mark.skip(reason="needs a CUDA GPU")]
else:
    pytestmark = pytest.mark.gpu

from test_gpu_prefix_cache import BF, DEV, P, gen  # noqa: E402, F401

# Two layers of about five roundings to bfloat16 each (unit roundoff 2^-8, root mean square below 2^-9).
BOUND = 2.0 ** -9 * math.sqrt(10) * 2
LONG = 20_000_000      # clock cycles: about a hundredth of a second


def model():
    from examples.serve_prefixes import TinyAttention
    return TinyAttention(torch, DEV)


def worst(got, model, texts):
    """Largest relative error of outputs [n, width] against the last positions of the texts (text, positions)."""
    at, w = 0, 0.0
    for t, n in texts:
        want = model.exact(t)[len(t) - n:]
        for a, b in zip(got[at:at + n].double(), want):
            w = max(w, float((a - b).norm() / b.norm()))
        at += n
    assert at == got.shape[0]
    return w


def serve(P, ctx, m, seed, busy=lambda: None):
    """Keys of which requests keep different parts, all texts different: largest error of every output."""
    from paper_2608_19677_gb300.destination import Destination
    g = gen(seed)
    text = lambda n: torch.randint(0, 4096, (n,), generator=g, device=DEV)  # noqa: E731
    prefix = {k: text(n) for k, n in ((1, 200), (2, 64), (3, 37))}
    pages = P.KVPages.empty(512, 16, 24, 24, m.layers, m.kv_heads, m.dim)
    d = Destination(ctx, pages, m)
    texts, w, done = {}, 0.0, []
    for batch in ([(1, 200, 5), (2, 64, 70), (3, 37, 1)], [(1, 96, 30), (1, 37, 3), (2, 16, 2)], [(3, 5, 90), (1, 160, 40)]):
        asked = [(k, torch.cat([prefix[k][:n], text(own)]), n) for k, n, own in batch]
        busy()
        rows, out = d.admit(asked)
        done.append((out, [(t, len(t) - n) for _, t, n in asked]))
        texts.update(zip(rows, (t for _, t, _ in asked)))
    for s in range(4):
        new = text(len(texts))
        order = d.order()
        busy()
        out = d.step(new)
        for row, t in zip(order, new):
            texts[row] = torch.cat([texts[row], t[None]])
        done.append((out, [(texts[row], 1) for row in order]))
        if s == 1:
            d.finish(order[::4])
            for row in order[::4]:
                del texts[row]
            d.compact()
    ctx.sync()
    for out, t in done:
        w = max(w, worst(out, m, t))
    assert int((pages.ref > 0).sum()) == pages.n_pages - d.free_pages
    assert all(int(pages.lens[row]) == len(t) for row, t in texts.items())
    return w


def test_requests_that_keep_different_parts_of_a_prefix(P):
    ctx = P.Context(0)
    assert serve(P, ctx, model(), 1) < BOUND
    ctx.close()


def test_a_context_with_a_stream_of_its_own(P):
    """Either stream far behind the other when the calls are made: lists that are dropped early, tokens that are not there
    yet and outputs that are not there yet would all show."""
    for late in ("own", "current", "both"):
        stream = torch.cuda.Stream()
        ctx = P.Context(0, stream=stream)
        assert ctx.stream.cuda_stream == stream.cuda_stream

        def busy():
            if late != "current":
                with torch.cuda.stream(stream):
                    torch.cuda._sleep(LONG)
            if late != "own":
                torch.cuda._sleep(LONG)

        assert serve(P, ctx, model(), 2, busy) < BOUND
        ctx.close()


@pytest.mark.parametrize("own_stream", [False, True])
def test_calls_return_while_the_gpu_is_still_busy(P, own_stream):
    from paper_2608_19677_gb300.destination import Destination
    stream = torch.cuda.Stream() if own_stream else torch.cuda.current_stream()
    ctx, m = P.Context(0, stream=stream), model()
    d = Destination(ctx, P.KVPages.empty(256, 16, 16, 16, m.layers, m.kv_heads, m.dim), m)
    t = torch.arange(100, device=DEV)

    def pass_():
        rows, _ = d.admit([(1, t[:40], 32), (2, t[3:60], 20), (1, t[:50], 32)])
        d.step(t[:3])
        d.finish(rows)
        d.compact()

    for _ in range(3):      # memory, libraries and kernels are there
        pass_()
    ctx.sync()
    end = torch.cuda.Event()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(50 * LONG)
        end.record()
    pass_()
    waited = end.query()
    ctx.sync()
    ctx.close()
    assert not waited


def test_a_model_whose_weights_want_gradients_is_served_without_them(P):
    ctx, m = P.Context(0), model()
    for w in (m.wq, m.wk, m.wv, m.wo):
        for i in range(len(w)):
            w[i] = torch.nn.Parameter(w[i])
    m.exact = torch.no_grad()(m.exact)
    assert serve(P, ctx, m, 3) < BOUND
    ctx.close()


@pytest.mark.parametrize("own_stream", [False, True])
def test_requests_without_tokens_of_their_own_and_steps_without_requests(P, own_stream):
    from paper_2608_19677_gb300.destination import Destination
    stream = torch.cuda.Stream() if own_stream else torch.cuda.current_stream()
    ctx, m, g = P.Context(0, stream=stream), model(), gen(7)
    d = Destination(ctx, P.KVPages.empty(64, 16, 8, 16, m.layers, m.kv_heads, m.dim), m)
    t = torch.randint(0, 4096, (40,), generator=g, device=DEV)
    rows, out = d.admit(requests=[(1, t, 40), (1, t[:33], 33)])
    assert out.shape[0] == 0
    new = torch.randint(0, 4096, (2,), generator=g, device=DEV)
    out = d.step(tokens=new)
    ctx.sync()
    assert worst(out, m, [(torch.cat([t, new[:1]]), 1), (torch.cat([t[:33], new[1:]]), 1)]) < BOUND
    d.finish(rows=rows)
    assert d.step(new[:0]).shape[0] == 0
    ctx.sync()
    assert int((d.pages.ref > 0).sum()) == 3 == 64 - d.free_pages
    ctx.close()
