"""What the binding of the calls on real-valued tensors refuses, and a run of the calls together as a transformer's block makes them."""
import threading
import time

import pytest
import torch

from gpu_util import api
from paper_2202_05239_b200 import synth
from scaled_util import check_codes, norm64, silu

pytestmark = pytest.mark.gpu

BF16, F32, S8 = torch.bfloat16, torch.float32, torch.int8


def test_products_refuse_tensors_that_do_not_fit():
    a = api()
    x, w, y = torch.zeros(4, 64, dtype=S8, device="cuda"), torch.zeros(8, 64, dtype=S8, device="cuda"), torch.zeros(4, 8, device="cuda")
    one, n4, n8 = torch.ones(1, device="cuda"), torch.ones(4, device="cuda"), torch.ones(8, device="cuda")
    good = dict(x=x, x_scale=n4, w=w, w_scale=n8, y=y, bias=n8)
    a.f8_linear_scaled(**good)
    a.f8_linear_scaled(**{**good, "x_scale": one, "w_scale": one, "bias": None})
    for name, bads in {"x": [x[0], x.float(), x.t(), x.cpu(), x[:, ::2], x[:, :63], x[:1].expand(4, 64)],
                       "w": [w.to(torch.uint8), w[:, :32], w[0], w.cpu()],
                       "y": [y[:3], y.t(), y.double(), y.to(torch.int32), y[:, ::2], y.cpu()],
                       "x_scale": [n8, n4.half(), None, torch.ones(8, device="cuda")[::2], n4.cpu()],
                       "w_scale": [n4, n8.double(), None],
                       "bias": [n4, n8.to(torch.int32), one]}.items():
        for bad in bads:
            with pytest.raises(ValueError):
                a.f8_linear_scaled(**{**good, name: bad})


def test_rows_refuse_tensors_that_do_not_fit():
    a = api()
    x, q, s, w = torch.zeros(4, 64, dtype=BF16, device="cuda"), torch.zeros(4, 64, dtype=S8, device="cuda"), torch.zeros(4, device="cuda"), torch.ones(64, device="cuda")
    a.f8_quantize_rows(x, q, s, y=x.clone(), u=x.clone())
    a.f8_norm_quantize(x, q, s, residual=x.clone(), gate=x[:1].clone(), pre_w=w)
    for kw in (dict(q=q[:3]), dict(q=q.to(torch.uint8)), dict(scale=s[:3]), dict(scale=s.half()), dict(y=x.float()), dict(u=x.half()), dict(u=x[:, :63]), dict(y=x.t())):
        with pytest.raises(ValueError):
            a.f8_quantize_rows(**{**dict(x=x, q=q, scale=s), **kw})
    for kw in (dict(residual=x.float()), dict(residual_out=x[:3].clone()), dict(gate=x[:2].clone()), dict(pre_w=w[:63]), dict(pre_w=w.half()), dict(pre_w=w, pre_b=w.to(BF16)),
               dict(y=x[:, ::2])):
        with pytest.raises((ValueError, a.F8Error)):
            a.f8_norm_quantize(**{**dict(x=x, q=q, scale=s), **kw})
    for f, kw in ((a.f8_quantize_rows, dict(x=x)), (a.f8_quantize_rows, dict(x=x, q=q)), (a.f8_quantize_rows, dict(x=x, scale=s, y=x.clone())), (a.f8_norm_quantize, dict(x=x)),
                  (a.f8_norm_quantize, dict(x=x, q=q, scale=s, pre_norm=a.F8_NORM_NONE, pre_w=w)), (a.f8_quantize_rows, dict(x=x, q=q, scale=s, act=a.F8_ACT_TANH))):
        with pytest.raises(a.F8Error):
            f(**kw)


def test_logprobs_refuse_tensors_that_do_not_fit():
    a = api()
    l, ids, lp, h = torch.zeros(4, 50, device="cuda"), torch.zeros(4, 2, dtype=torch.int64, device="cuda"), torch.zeros(4, 2, device="cuda"), torch.zeros(4, device="cuda")
    a.f8_token_logprobs(l, ids, lp, h, lp.clone(), ids.clone())
    for args in ((l[0], ids, lp), (l.double(), ids, lp), (l, ids.int(), lp), (l, ids[:3], lp), (l, ids, lp[:, :1]), (l, None, lp), (l, ids, lp, h[:3]),
                 (l, ids, lp, h, lp.clone(), ids[:, :1].clone()), (l, ids, lp, h, lp.half()), (l.t(), None, None, h), (l.cpu(), None, None, h)):
        with pytest.raises(ValueError):
            a.f8_token_logprobs(*args)
    with pytest.raises(a.F8Error):
        a.f8_token_logprobs(l, top_ids=torch.zeros(4, 33, dtype=torch.int64, device="cuda"))
    with pytest.raises(a.F8Error):
        a.f8_token_logprobs(l, ids)
    with pytest.raises(a.F8Error):
        a.f8_token_logprobs(l, entropy=h, inv_temperature=0.0)


def test_explicit_stream():
    a = api()
    side = torch.cuda.Stream()
    x = torch.randn(300, 4096, device="cuda").to(BF16)
    q, s = torch.zeros(300, 4096, dtype=S8, device="cuda"), torch.zeros(300, device="cuda")
    torch.cuda.synchronize()
    a.f8_quantize_rows(x, q, s, stream=side)
    side.synchronize()
    q2, s2 = torch.empty_like(q), torch.empty_like(s)
    a.f8_quantize_rows(x, q2, s2)
    assert torch.equal(q, q2) and torch.equal(s, s2)


@pytest.mark.parametrize("n,c,hidden,vocab", [(1, 256, 640, 1000), (7, 512, 1408, 5003), (64, 1024, 2048, 8192), (333, 768, 1024, 2000)])
def test_block_of_a_transformer(n, c, hidden, vocab):
    """Weights to codes, norm and residual to codes, widening product, gated activation to codes, narrowing product, the next norm with the residual sum,
    logits and their log probabilities: every step against its 64-bit form of what the step before gave."""
    a = api()
    g = torch.Generator(device="cuda").manual_seed(n)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")       # noqa: E731

    def weights(out, k):
        w = rand(out, k) / k ** 0.5
        q, s = torch.empty(out, k, dtype=S8, device="cuda"), torch.empty(out, device="cuda")
        a.f8_quantize_rows(w, q, s)
        return q, s
    wide, narrow, head = weights(2 * hidden, c), weights(c, hidden), weights(vocab, c)
    norm1, norm2 = rand(c) * 0.1 + 1, rand(c) * 0.1 + 1

    def codes(k):
        return torch.empty(n, k, dtype=S8, device="cuda"), torch.empty(n, device="cuda")

    def product(q, s, w, out, t=BF16):
        y = torch.empty(n, out, dtype=t, device="cuda")
        a.f8_linear_scaled(q, s, w[0], w[1], y)
        want = (q.double() @ w[0].double().t()) * s.double()[:, None] * w[1].double()
        assert bool(((y.double() - want).abs() <= want.abs() * (torch.finfo(t).eps / 2 + 2.0 ** -21) + 1e-30).all())
        return y

    x, r = rand(n, c).to(BF16), (rand(n, c) * 2).to(BF16)
    q, s = codes(c)
    stream = r.clone()
    a.f8_norm_quantize(x, q, s, residual=stream, residual_out=stream, pre_w=norm1)
    t = r.double() + x.double()
    v, e = norm64(t, t.abs() * 2.0 ** -23, 1, norm1, None, 0.0, 1e-5)
    check_codes(v, e, q, s)
    both = product(q, s, wide, 2 * hidden)
    q, s = codes(hidden)
    a.f8_quantize_rows(both[:, :hidden], q, s, u=both[:, hidden:], act=a.F8_ACT_SILU)
    gate = both[:, :hidden].double()
    v = silu(gate) * both[:, hidden:].double()
    check_codes(v, v.abs() * (10 + 2.4 * gate.abs()) * 2.0 ** -23, q, s)
    y = product(q, s, narrow, c)
    q, s = codes(c)
    before = stream.double()
    a.f8_norm_quantize(y, q, s, residual=stream, residual_out=stream, pre_w=norm2, branch_scale=0.5)
    t = before + 0.5 * y.double()
    v, e = norm64(t, t.abs() * 2.0 ** -23, 1, norm2, None, 0.0, 1e-5)
    check_codes(v, e, q, s)
    logits = product(q, s, head, vocab, F32)
    ids = torch.randint(0, vocab, (n, 1), generator=g, device="cuda")
    lp, h, tl, ti = torch.empty(n, 1, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, 5, device="cuda"), torch.empty(n, 5, dtype=torch.int64, device="cuda")
    a.f8_token_logprobs(logits, ids, lp, h, tl, ti)
    want = torch.log_softmax(logits.double(), dim=1)
    order = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :5]
    assert torch.equal(ti, order)
    assert bool(((lp.double() - want.gather(1, ids)).abs() <= 1e-5 * (1 + want.gather(1, ids).abs())).all())
    assert bool(((tl.double() - want.gather(1, order)).abs() <= 1e-5 * (1 + want.gather(1, order).abs())).all())
    assert bool(((h.double() + (want.exp() * want).sum(dim=1)).abs() <= 1e-5 * (1 + h.double())).all())
    torch.cuda.synchronize()
    a.f8_device_status()


def test_tensors_without_rows_do_not_count_as_left_out():
    """An optional matrix that has no rows fits a call of no rows alone."""
    a = api()
    x, q, s = torch.randn(4, 64, device="cuda").to(BF16), torch.zeros(4, 64, dtype=S8, device="cuda"), torch.zeros(4, device="cuda")
    none, no_codes = x[:0], q[:0]
    for kw in (dict(u=none), dict(y=none), dict(q=no_codes, scale=None, y=x.clone())):
        with pytest.raises(ValueError, match="shape"):
            a.f8_quantize_rows(**{**dict(x=x, q=q, scale=s), **kw})
    for kw in (dict(residual=none), dict(residual_out=none), dict(gate=none), dict(y=none), dict(q=no_codes, scale=None, y=x.clone())):
        with pytest.raises(ValueError, match="shape"):
            a.f8_norm_quantize(**{**dict(x=x, q=q, scale=s), **kw})
    a.f8_quantize_rows(none, no_codes, s[:0], y=none, u=none)
    a.f8_norm_quantize(none, no_codes, s[:0], y=none, residual=none, residual_out=none, gate=none)
    a.f8_norm_quantize(none, no_codes, s[:0], gate=x[:1])


def test_other_threads_run_while_a_launch_waits_for_the_queue():
    """A call that has to wait for room among the launches on their way does not stop the other Python threads."""
    a = api()
    x, q, s = torch.randn(1, 64, device="cuda"), torch.zeros(1, 64, dtype=S8, device="cuda"), torch.zeros(1, device="cuda")
    a.f8_quantize_rows(x, q, s)
    torch.cuda.synchronize()
    ticks, done = [], threading.Event()

    def tick():
        while not done.is_set():
            ticks.append(time.perf_counter())
            time.sleep(0.002)
    other = threading.Thread(target=tick)
    other.start()
    try:
        torch.cuda._sleep(1_500_000_000)        # three quarters of a second or more of the GPU
        start = time.perf_counter()
        for _ in range(5000):                   # far more launches than the queue holds
            a.f8_quantize_rows(x, q, s)
        took = time.perf_counter() - start
    finally:
        done.set()
        other.join()
        torch.cuda.synchronize()
    assert took > 0.4, "the queue was never full"
    gap = max(b - a for a, b in zip(ticks, ticks[1:]))
    assert gap < took / 2, f"another thread stood still for {gap:.2f} of {took:.2f} s"


def test_calls_on_several_streams_at_once():
    """Products by every kernel, rows, log probabilities and a network's forward passes on streams of their own give what they give alone."""
    a = api()
    g = torch.Generator(device="cuda").manual_seed(0)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")       # noqa: E731
    codes = lambda *s: torch.randint(-127, 128, s, generator=g, device="cuda", dtype=S8)       # noqa: E731
    one = torch.full((1,), 0.01, device="cuda")

    def product(n, k, out):
        x, w = codes(n, k), codes(out, k)

        def call():
            y = torch.empty(n, out, dtype=BF16, device="cuda")
            a.f8_linear_scaled(x, one, w, one, y)
            return [y]
        return call

    def rows(n, c):
        x, r, u, w = rand(n, c).to(BF16), rand(n, c).to(BF16), rand(n, c).to(BF16), rand(c)

        def call():
            q, s, t, p, z = torch.empty(n, c, dtype=S8, device="cuda"), torch.empty(n, device="cuda"), torch.empty_like(x), torch.empty(n, c, dtype=S8, device="cuda"), torch.empty(n, device="cuda")
            a.f8_norm_quantize(x, q, s, residual=r, residual_out=t, pre_w=w)
            a.f8_quantize_rows(t, p, z, u=u, act=a.F8_ACT_SILU)
            return [q, s, t, p, z]
        return call

    def logprobs(n, v):
        logits = rand(n, v)

        def call():
            h, ti = torch.empty(n, device="cuda"), torch.empty(n, 20, dtype=torch.int64, device="cuda")
            a.f8_token_logprobs(logits, entropy=h, top_ids=ti)
            return [h, ti]
        return call
    layers = synth.make_net("resnet50", 0, image=96)
    net, images = a.Net(layers, 16), a.to_device(synth.draw_image(16, 1, 96, 96))
    chains = [[product(1, 4096, 4096), product(23, 4096, 2048), product(100, 2048, 1000)], [product(2048, 1024, 2048), product(40, 1025, 999)],
              [rows(700, 2048), logprobs(16, 131072), logprobs(3000, 1000)], [lambda: [net.forward(images)]]]
    alone = [[call() for call in chain] for chain in chains]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in chains]
    results = []
    for _ in range(20):
        for i, (stream, chain) in enumerate(zip(streams, chains)):
            with torch.cuda.stream(stream):
                results.append((i, [call() for call in chain]))
    torch.cuda.synchronize()
    a.f8_device_status()
    for i, got in results:
        for x, y in zip(alone[i], got):
            assert all(torch.equal(p, q) for p, q in zip(x, y)), f"stream {i}"
    net.close()
