"""Log probabilities, entropy and largest alternatives of logits (f8_token_logprobs) against their 64-bit forms."""
import dataclasses

import numpy as np
import pytest
import torch

from gpu_util import api
from paper_2202_05239_b200 import synth
from scaled_util import U, strided

pytestmark = pytest.mark.gpu

BF16, F16, F32, S32 = torch.bfloat16, torch.float16, torch.float32, torch.int32
INF = float("inf")


def _reference(logits, c):
    z = logits.double() * c
    m = z.amax(dim=1, keepdim=True)
    d = m - z
    e = torch.exp(-d)
    total = e.sum(dim=1, keepdim=True)
    lse = torch.log(total)
    h = lse[:, 0] + (torch.where(e > 0, d, torch.zeros_like(d)) * e).sum(dim=1) / total[:, 0]
    return -d - lse, h, lse


def _bounds(lp, h, v):
    """32-bit sums of v positive terms of 2 + 2 steps each (their exponents, rounded, and their exponentials), in any of the kernels'
    orders: at most v / 128 terms one after the other and a tree; then a logarithm; a logit's distance rounds twice."""
    r = (v / 128 + 64 + 16) * 2 * U
    return r + lp.abs() * 4 * U, r * (1 + 3 * h) + h * 8 * U


def _run(logits, tokens=0, top=0, fl=0, inv_t=1.0, seed=0):
    a = api()
    n, v = logits.shape
    rng = np.random.default_rng(seed)
    ids = torch.from_numpy(rng.integers(0, v, size=(n, tokens))).cuda() if tokens else None
    lp = torch.full((n, tokens), 7.0, device="cuda") if tokens else None
    h = torch.full((n,), 7.0, device="cuda")
    tl, ti = (torch.full((n, top), 7.0, device="cuda"), torch.full((n, top), -7, dtype=torch.int64, device="cuda")) if top else (None, None)
    a.f8_token_logprobs(logits, ids, lp, entropy=h, top_logprobs=tl, top_ids=ti, fl=fl, inv_temperature=inv_t)
    torch.cuda.synchronize()
    c = inv_t * (2.0 ** -fl if logits.dtype == S32 else 1.0)
    want, wh, _ = _reference(logits, c)
    tol, tol_h = _bounds(want, wh, v)
    assert bool(((h.double() - wh).abs() <= tol_h).all()), f"entropy off by {(h.double() - wh).abs().max().item()}"
    if tokens:
        w, t = want.gather(1, ids), tol.gather(1, ids)
        assert bool((((lp.double() - w).abs() <= t) | (lp.double() == w)).all())
    if top:
        order = torch.sort(logits.float() if logits.dtype != S32 else logits, dim=1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(ti, order), "top ids"
        w, t = want.gather(1, order), tol.gather(1, order)
        assert bool((((tl.double() - w).abs() <= t) | (tl.double() == w)).all())
    return h


def _logits(rng, n, v, t, spread=3.0):
    z = torch.from_numpy(rng.normal(0, spread, size=(n, v)))
    return (z * 4096).round().to(S32).cuda() if t == S32 else z.to(t).cuda()


@pytest.mark.parametrize("t", [S32, F32, F16, BF16])
@pytest.mark.parametrize("n,v", [(1, 1), (3, 2), (2, 7), (5, 33), (1, 100), (4, 1000), (256, 1000), (3, 4097), (2, 32768), (1, 50001), (17, 20003), (1, 131072),
                                 (300, 3001), (2, 262144)])
def test_rows(n, v, t):
    rng = np.random.default_rng(v)
    _run(_logits(rng, n, v, t), tokens=3, top=min(v, 20), fl=12)
    _run(_logits(rng, n, v, t), tokens=1, fl=12)
    _run(_logits(rng, n, v, t), top=min(v, 1), fl=12, inv_t=1 / 0.7)


@pytest.mark.parametrize("top", [1, 2, 5, 8, 20, 31, 32])
@pytest.mark.parametrize("v", [32, 33, 300, 5000, 70000])
def test_alternatives_with_many_ties(top, v):
    """Few different values, so that most places are decided by the index."""
    rng = np.random.default_rng(top)
    for t in (BF16, S32):
        logits = torch.from_numpy(rng.integers(-2, 3, size=(6, v))).to(t).cuda()
        logits[1] = 1
        logits[2] = torch.arange(v, device="cuda").to(t)            # rising: every element is the largest so far
        logits[3] = -torch.arange(v, device="cuda").to(t)
        logits[4, v // 2:] = 5
        _run(logits, tokens=1, top=top, fl=1)


@pytest.mark.parametrize("v", [100, 9000])
def test_zeros_of_both_signs_are_equal(v):
    logits = torch.zeros(2, v, device="cuda")
    logits[:, ::2] = -0.0
    _run(logits, top=5)


@pytest.mark.parametrize("t", [F32, F16, BF16])
@pytest.mark.parametrize("v", [40, 3001, 70001])
def test_masked_logits(t, v):
    """Masks of -infinity and of the type's lowest value, down to one place left."""
    rng = np.random.default_rng(v)
    logits = _logits(rng, 6, v, t)
    logits[0, ::2] = -INF
    logits[1, 1:] = -INF
    logits[2, :-1] = -INF
    logits[3, 5:] = torch.finfo(t).min
    logits[4, v // 3: v // 2] = -INF
    _run(logits, tokens=4, top=min(v, 20))


@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("v", [64, 5000, 140000])
def test_empty_and_not_finite_rows(t, v):
    a = api()
    logits = torch.randn(6, v, device="cuda").to(t)
    logits[1] = -INF
    logits[2, 11] = float("nan")
    logits[3, 17] = INF
    logits[4, 3], logits[4, 60] = float("nan"), INF
    ids = torch.zeros(6, 2, dtype=torch.int64, device="cuda")
    lp, h = torch.empty(6, 2, device="cuda"), torch.empty(6, device="cuda")
    tl, ti = torch.empty(6, 3, device="cuda"), torch.empty(6, 3, dtype=torch.int64, device="cuda")
    a.f8_token_logprobs(logits, ids, lp, h, tl, ti)
    torch.cuda.synchronize()
    assert bool((lp[1] == -INF).all()) and float(h[1]) == 0 and bool((tl[1] == -INF).all()) and ti[1].tolist() == [0, 1, 2]
    for i in (2, 3, 4):
        assert torch.isnan(lp[i]).all() and torch.isnan(h[i]) and torch.isnan(tl[i]).all()
    assert int(ti[2, 0]) == 11 and int(ti[3, 0]) == 17 and ti[4, :2].tolist() == [3, 60]
    for i in (0, 5):
        assert bool(torch.isfinite(lp[i]).all()) and float(h[i]) > 0


def test_padded_and_wrong_tokens():
    a = api()
    logits = torch.randn(4, 50, device="cuda")
    ids = torch.tensor([[0, -1], [-100, 49], [50, 3], [2 ** 40, -2 ** 40]], device="cuda")
    lp = torch.empty(4, 2, device="cuda")
    a.f8_token_logprobs(logits, ids, lp)
    torch.cuda.synchronize()
    want = torch.log_softmax(logits.double(), dim=1)
    assert float(lp[0, 1]) == 0 and float(lp[1, 0]) == 0 and float(lp[3, 1]) == 0
    assert torch.isnan(lp[2, 0]) and torch.isnan(lp[3, 0])
    for i, j, k in ((0, 0, 0), (1, 1, 49), (2, 1, 3)):
        assert abs(float(lp[i, j]) - float(want[i, k])) < 1e-5


def test_certain_rows_keep_their_precision():
    """One logit with nearly all the probability: its log probability and the entropy keep their relative precision."""
    a = api()
    logits = torch.full((3, 1000), -20.0, device="cuda")
    logits[:, 321] = 0.0
    logits[1, 321] = 5.0
    logits[2, 400:] = -30.0
    ids = torch.full((3, 1), 321, dtype=torch.int64, device="cuda")
    lp, h = torch.empty(3, 1, device="cuda"), torch.empty(3, device="cuda")
    a.f8_token_logprobs(logits, ids, lp, h)
    z = logits.double()
    others = torch.exp(z - z[:, 321:322])
    others[:, 321] = 0
    r = others.sum(dim=1)
    want = -torch.log1p(r)
    wh = -want + (others * (z[:, 321:322] - z)).sum(dim=1) / (1 + r)
    assert bool(((lp[:, 0].double() - want).abs() <= 1e-5 * want.abs()).all())
    assert bool(((h.double() - wh).abs() <= 1e-5 * wh).all())


def test_large_codes_lose_nothing():
    """Codes beyond 2^24 whose differences are small, and the whole range of 32 bits."""
    base = torch.tensor([2 ** 31 - 1, -2 ** 31 + 5000, 2 ** 30 + 12345], device="cuda", dtype=torch.int64)
    rng = np.random.default_rng(1)
    off = torch.from_numpy(rng.integers(0, 5000, size=(3, 700))).cuda()
    _run((base[:, None] - off).to(S32), tokens=2, top=20, fl=9)
    wide = torch.from_numpy(rng.integers(-2 ** 31, 2 ** 31, size=(4, 700))).to(S32).cuda()
    _run(wide, tokens=2, top=5, fl=28)


@pytest.mark.parametrize("pad,offset", [(8, 8), (1, 0), (0, 1), (5, 3)])
@pytest.mark.parametrize("t", [BF16, F32, S32])
def test_strided_and_unaligned_rows(t, pad, offset):
    rng = np.random.default_rng(5)
    for n, v in ((4, 50), (3, 1003), (2, 40960)):
        x, flat = strided(n, v, t, pad, offset, fill=10000)         # a neighbour that was read would win
        x.copy_(_logits(rng, n, v, t))
        _run(x, tokens=2, top=min(20, v), fl=12)


@pytest.mark.parametrize("n,v,top", [(300, 262144, 20), (1, 400000, 32)])
def test_large_logits_that_one_thread_meets(n, v, top):
    """Large logits at one place of every stretch that the threads of a block share out, more of them than candidates are kept."""
    logits = torch.zeros(n, v, device="cuda")
    logits[0] = torch.randn(v, device="cuda") * 0.1
    for k in range(4):
        logits[0, 20 + k::1024] = 5 + torch.rand(logits[0, 20 + k::1024].shape[0], device="cuda")
    logits[n - 1, 20::1024] = 7
    logits[n - 1, 21::1024] = 7
    logits[n - 1, 22::1024] = 7
    logits[n - 1, 23::1024] = 7
    _run(logits, tokens=1, top=top)


def test_rows_beyond_four_gigabytes():
    """Rows whose distance from the first passes 32 bits, in bytes and in elements."""
    a = api()
    n, v = 2, 60001
    flat = torch.zeros(4_500_000_000 + v + 64, dtype=BF16, device="cuda")
    logits = torch.as_strided(flat, (n, v), (4_500_000_000, 1))
    logits[1] = torch.randn(v, device="cuda") * 3
    h, ti = torch.empty(n, device="cuda"), torch.empty(n, 4, dtype=torch.int64, device="cuda")
    a.f8_token_logprobs(logits, entropy=h, top_ids=ti)
    order = torch.sort(logits[1].float(), descending=True, stable=True).indices[:4]
    assert torch.equal(ti[1], order) and ti[0].tolist() == [0, 1, 2, 3]
    assert abs(float(h[0]) - float(torch.log(torch.tensor(v, dtype=torch.float64)))) < 1e-4


def test_single_outputs_and_no_rows():
    a = api()
    logits = torch.randn(7, 500, device="cuda").to(BF16)
    full = [torch.empty(7, 4, device="cuda"), torch.empty(7, device="cuda"), torch.empty(7, 3, device="cuda"), torch.empty(7, 3, dtype=torch.int64, device="cuda")]
    ids = torch.arange(28, device="cuda").view(7, 4)
    a.f8_token_logprobs(logits, ids, *full)
    for i in range(4):
        one = [torch.empty_like(t) if j == i else None for j, t in enumerate(full)]
        a.f8_token_logprobs(logits, ids if i == 0 else None, *one)
        assert torch.equal(one[i], full[i])
    a.f8_token_logprobs(logits[:0], None, None, torch.empty(0, device="cuda"))


def test_captured_and_replayed():
    a = api()
    for n, v in ((2, 131072), (64, 1000)):
        logits = torch.randn(n, v, device="cuda").to(BF16)
        h, ti = torch.empty(n, device="cuda"), torch.empty(n, 5, dtype=torch.int64, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            a.f8_token_logprobs(logits, entropy=h, top_ids=ti)
        logits.copy_(torch.randn(n, v, device="cuda"))
        g.replay()
        torch.cuda.synchronize()
        got = (h.clone(), ti.clone())
        a.f8_token_logprobs(logits, entropy=h, top_ids=ti)
        assert torch.equal(got[0], h) and torch.equal(got[1], ti)


def test_network_classifies(ref):
    """A network's own logits: classes and log probabilities of `Net.classify` against the oracle's codes."""
    a = api()
    layers = synth.make_net("resnet18", 0, image=64)
    images = synth.draw_image(3, 5, 64, 64)
    net = a.Net(layers, 3)
    ids, lp = net.classify(a.to_device(images), top=5)
    torch.cuda.synchronize()
    logits = torch.from_numpy(ref.net_forward(layers, images, keep_all=False)[-1].reshape(3, -1).astype(np.int64)).cuda()
    c = 2.0 ** -(layers[-1].fl_x + layers[-1].fl_w)
    want, h, _ = _reference(logits, c)
    order = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :5]
    assert torch.equal(ids, order)
    tol, _ = _bounds(want, h, logits.shape[1])
    assert bool(((lp.double() - want.gather(1, order)).abs() <= tol.gather(1, order)).all())
    net.close()


@pytest.mark.parametrize("t", [S32, F32, F16, BF16])
@pytest.mark.parametrize("v", [130, 250, 1000, 1031, 2045])
def test_short_rows_with_many_alternatives(v, t):
    """Rows that give fewer groups of threads an element than there are alternatives; equal logits; rows that start off a vector."""
    rng = np.random.default_rng(v)
    for top in (9, 17, 32):
        _run(_logits(rng, 3, v, t), tokens=2, top=top, fl=12)
        few = torch.from_numpy(rng.integers(-3, 3, size=(3, v))).to(t).cuda()
        _run(few, tokens=2, top=top, fl=2)
        view, _ = strided(3, v, t, 5, 3)
        view.copy_(_logits(rng, 3, v, t))
        _run(view, tokens=2, top=top, fl=12)


@pytest.mark.parametrize("t", [S32, F32, BF16])
@pytest.mark.parametrize("v", [10, 300, 600, 1000, 1216])
def test_thousands_of_short_rows_with_many_alternatives(v, t):
    """Every SM full of rows whose alternatives are bounded by single threads, or not at all, again and again: the same ones each time."""
    rng = np.random.default_rng(v)
    logits = _logits(rng, 6000, v, t)
    view, _ = strided(6000, v, t, 1, 1)             # the same off a vector: elements in front of the first and behind the last
    view.copy_(logits)
    a = api()
    order = torch.sort(logits.float() if t != S32 else logits, dim=1, descending=True, stable=True).indices
    for top in (5, 20, 32):
        if top > v:
            continue
        ti = torch.empty(6000, top, dtype=torch.int64, device="cuda")
        for rows in (logits, view) * 10:
            ti.fill_(-7)
            a.f8_token_logprobs(rows, top_ids=ti, fl=12)
            assert torch.equal(ti, order[:, :top])
        _run(logits, tokens=2, top=top, fl=12)


@pytest.mark.parametrize("classes,batch,top", [(10, 1, 5), (10, 300, 10), (100, 64, 32), (1000, 7, 1)])
def test_networks_of_few_classes(classes, batch, top):
    """`Net.classify` of a network whose last layer has few classes, its logits those of the forward pass."""
    a = api()
    layers = synth.make_net("mobilenetv1", 0, image=32)
    last = layers[-1]
    layers[-1] = dataclasses.replace(last, c_out=classes, weight=last.weight[:classes].copy(), bias=last.bias[:classes].copy())
    net = a.Net(layers, batch)
    x = a.to_device(synth.draw_image(batch, 5, 32, 32))
    ids, lp = net.classify(x, top=top)
    logits = net.forward(x).view(batch, classes)
    order = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :top]
    assert torch.equal(ids, order)
    want, h, _ = _reference(logits, 2.0 ** -(layers[-1].fl_x + layers[-1].fl_w))
    tol, _ = _bounds(want, h, classes)
    assert bool(((lp.double() - want.gather(1, order)).abs() <= tol.gather(1, order)).all())
    net.close()


@pytest.mark.parametrize("tokens,top", [(1, 1), (3, 5), (33, 31), (0, 7)])
def test_lanes_of_the_leading_block_have_different_work(tokens, top):
    """Rows shared by the blocks of a cluster, outputs that only some lanes of a warp write, rows ranked in one pass and by a pass for each
    alternative side by side."""
    logits = _logits(np.random.default_rng(top), 9, 80001, BF16)
    for fill in (0.0, 1.5):
        logits[::2] = fill              # equal logits: more candidates than there is room for
        _run(logits, tokens=tokens, top=top)


@pytest.mark.parametrize("t", [F32, F16, BF16])
@pytest.mark.parametrize("n,v", [(8, 1003), (8, 5001), (400, 20003), (8, 140001)])      # in registers, by a block, by many, by a cluster
def test_masks_of_low_numbers_in_front(n, v, t):
    """Threads that have met nothing but a mask of finite low numbers, then an open place: the mask adds nothing, and no NaN."""
    rng = np.random.default_rng(v)
    for low in (torch.finfo(t).min, -1e38, -6e4):
        low = max(low, torch.finfo(t).min)
        logits = _logits(rng, n, v, t)
        logits[0, :-5] = low
        logits[1, :-1] = low                                    # one open place, behind the last whole vector
        logits[2, : v // 2] = low
        logits[3, v // 3:] = low
        stretch = 1024 * 16 // logits.element_size()
        logits[4, torch.arange(v, device="cuda") // stretch % 2 == 0] = low
        logits[5] = low                                         # equal logits, low as they are
        logits[6] = low
        logits[6, v // 2] = -1e4
        logits[7:, ::3] = low
        _run(logits, tokens=3, top=20)
        assert bool((_run(logits, tokens=1, top=1) >= 0).all())


@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("n,v", [(3, 1003), (3, 5001), (400, 20003), (3, 140001)])
def test_large_logits_at_a_high_temperature(n, v, t):
    """Logits near the largest float, which the temperature takes back: only their product with its inverse counts."""
    rng = np.random.default_rng(v)
    logits = (_logits(rng, n, v, F32) * 2.0 ** 122).to(t)
    _run(logits, tokens=3, top=5, inv_t=2.0 ** -122)
    logits[:, : v // 2] = torch.finfo(t).min / 4
    _run(logits, tokens=3, top=5, inv_t=2.0 ** -122)
