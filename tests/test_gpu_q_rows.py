"""Rows of real values to codes (f8_quantize_rows) and the step between two blocks (f8_norm_quantize) against their 64-bit forms."""
import itertools

import numpy as np
import pytest
import torch

from gpu_util import Guarded, api
from scaled_util import U, check_codes, gelu, half_step, norm64, same_codes, silu, strided, tiny

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
INF = float("inf")
SHAPES = [(1, 1), (1, 2), (3, 7), (5, 16), (2, 63), (4, 64), (9, 100), (17, 256), (3, 513), (6, 1024), (2, 1537), (7, 2048), (3, 4100), (2, 8192), (1, 16384), (2, 16385),
          (1, 40001)]


def _values(rng, n, c, t, scale=1.0):
    return torch.from_numpy(rng.normal(0, scale, size=(n, c))).to(t).cuda()


@pytest.mark.parametrize("t", [BF16, F16, F32])
@pytest.mark.parametrize("n,c", SHAPES)
def test_plain_rows_have_the_defined_codes(n, c, t):
    a = api()
    x = _values(np.random.default_rng(c), n, c, t)
    q, s, y = Guarded((n, c), torch.int8), Guarded((n,), F32), Guarded((n, c), t)
    a.f8_quantize_rows(x, q.t, s.t, y=y.t)
    torch.cuda.synchronize()
    same_codes(x.float(), q.t, s.t, y.t)
    assert q.intact() and s.intact() and y.intact()
    q2, s2 = torch.empty_like(q.t), torch.empty_like(s.t)
    a.f8_quantize_rows(x, q2, s2)
    assert torch.equal(q2, q.t) and torch.equal(s2, s.t)


@pytest.mark.parametrize("n,c", [(5, 64), (300, 96), (1000, 2048), (513, 4096), (64, 5000)])
def test_many_rows(n, c):
    a = api()
    for t in (BF16, F32):
        x = _values(np.random.default_rng(n), n, c, t)
        q, s = torch.empty(n, c, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
        a.f8_quantize_rows(x, q, s)
        same_codes(x.float(), q, s)


def test_ties_round_up():
    """Values on the half step between two codes: the largest magnitude is 127, so a code is the value rounded half up."""
    a = api()
    v = torch.tensor([[127.0] + [k + 0.5 for k in range(-127, 127)] + [0.0, -0.0, 0.25, -0.25, np.nextafter(np.float32(0.5), np.float32(0)),
                                                                      np.nextafter(np.float32(-0.5), np.float32(-1))]], device="cuda", dtype=F32)
    q, s = torch.empty(v.shape, dtype=torch.int8, device="cuda"), torch.empty(1, device="cuda")
    a.f8_quantize_rows(v, q, s)
    want = [127] + [k + 1 for k in range(-127, 127)] + [0, 0, 0, 0, 0, -1]
    assert q[0].tolist() == want and float(s) == 1.0


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("t", [BF16, F16, F32])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("n,c", [(1, 1), (3, 7), (9, 100), (4, 1024), (33, 2049), (5, 8192), (2, 20000)])
def test_activations(n, c, gated, t, act):
    a = api()
    rng = np.random.default_rng(c)
    both = _values(rng, n, 2 * c, t, 3.0)          # gate and value as halves of one tensor, as the widening product leaves them
    x, u = both[:, :c], both[:, c:] if gated else None
    q, s, y = torch.empty(n, c, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, c, dtype=t, device="cuda")
    code = {"silu": a.F8_ACT_SILU, "gelu": a.F8_ACT_GELU}[act]
    a.f8_quantize_rows(x, q, s, y=y, u=u, act=code)
    v = (silu if act == "silu" else gelu)(x.double())
    if gated:
        v = v * u.double()
    # the exponential's documented error grows with its argument (2 + 1.2 |x| steps at most, a step 2^-23); the other steps are a handful
    err = v.abs() * (10 + 2.4 * x.double().abs()) * 2.0 ** -23
    check_codes(v, err, q, s, y, act)
    z = torch.empty(n, c, dtype=t, device="cuda")
    a.f8_quantize_rows(x, y=z, u=u, act=code)       # the values themselves
    off = (z.double() - v).abs()
    assert bool((off <= 1.01 * (err + half_step(t) * v.abs()) + tiny(t) + 1e-45).all())


def test_activations_far_out():
    a = api()
    x = torch.tensor([[-200.0, -100.0, -88.0, -20.0, -5.0, 0.0, 5.0, 88.0, 200.0, 3e38, -3e38]], device="cuda")
    for act, f in ((a.F8_ACT_SILU, silu), (a.F8_ACT_GELU, gelu)):
        y = torch.empty_like(x)
        a.f8_quantize_rows(x, y=y, act=act)
        want = f(x.double())
        want = torch.where(x < -1000, torch.zeros_like(want), want)
        assert bool(torch.isfinite(y).all())
        assert bool(((y.double() - want).abs() <= want.abs() * (10 + 2.4 * x.double().abs().clamp(max=200)) * 2.0 ** -23 + 1e-37).all()), (y, want)


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("c", [16, 20000])
def test_activations_far_out_in_16_bits(t, c):
    a = api()
    big = 6e4 if t == F16 else 3e38
    x = torch.zeros(1, c, device="cuda")
    x[0, :14] = torch.tensor([-big, -1000.0, -200.0, -100.0, -88.5, -87.5, -60.0, -20.0, 0.0, 20.0, 88.5, 200.0, 1000.0, big])
    x = x.to(t)
    for act, f in ((a.F8_ACT_SILU, silu), (a.F8_ACT_GELU, gelu)):
        y = torch.empty_like(x)
        a.f8_quantize_rows(x, y=y, act=act)
        v = x.double()
        want = torch.where(v < -1000, torch.zeros_like(v), f(v))
        assert bool(torch.isfinite(y).all())
        err = want.abs() * ((10 + 2.4 * v.abs().clamp(max=200)) * 2.0 ** -23 + half_step(t)) + tiny(t) + 1e-36
        assert bool(((y.double() - want).abs() <= 1.01 * err).all()), (y, want)


@pytest.mark.parametrize("c", [8, 100, 4096, 20000])
@pytest.mark.parametrize("t", [BF16, F32])
def test_zero_tiny_and_not_finite_rows(c, t):
    a = api()
    x = _values(np.random.default_rng(1), 8, c, t)
    x[1] = 0
    x[2] = 2.0 ** -101
    x[3, c // 2] = float("inf")
    x[4, c - 1] = float("nan")
    x[5, 0] = -float("inf")
    x[6] *= 1e30 if t == F32 else 1e20
    q, s, y = torch.full((8, c), 55, dtype=torch.int8, device="cuda"), torch.empty(8, device="cuda"), torch.empty(8, c, dtype=t, device="cuda")
    a.f8_quantize_rows(x, q, s, y=y)
    for i in (1, 2):
        assert float(s[i]) == 0 and not q[i].any() and not y[i].any()
    for i in (3, 5):
        assert torch.isinf(s[i]) and not q[i].any() and torch.isnan(y[i]).all()
    assert torch.isnan(s[4]) and not q[4].any() and torch.isnan(y[4]).all()
    same_codes(x[[0, 6, 7]].float(), q[[0, 6, 7]], s[[0, 6, 7]], y[[0, 6, 7]])


@pytest.mark.parametrize("pad,offset", [(8, 8), (1, 0), (0, 1), (3, 5), (16, 32)])
@pytest.mark.parametrize("t", [BF16, F32])
def test_strided_and_unaligned_rows(t, pad, offset):
    a = api()
    rng = np.random.default_rng(pad)
    for n, c in ((4, 96), (3, 1000), (5, 4096)):
        x, xf = strided(n, c, t, pad, offset, fill=1e4)
        x.copy_(_values(rng, n, c, t))
        q, qf = strided(n, c, torch.int8, pad, offset, fill=99)
        y, yf = strided(n, c, t, pad, offset, fill=99)
        s = torch.empty(n, device="cuda")
        a.f8_quantize_rows(x, q, s, y=y)
        same_codes(x.float(), q, s, y)
        for flat in (qf, yf):       # nothing between or around the rows is written
            rest = flat.clone()
            rest[offset:offset + n * (c + pad)].view(n, c + pad)[:, :c] = 99
            assert bool((rest == 99).all())


@pytest.mark.parametrize("c", [100, 2048, 20001])
def test_values_in_place(c):
    a = api()
    for t in (BF16, F32):
        x = _values(np.random.default_rng(4), 5, c, t)
        keep = x.clone()
        q, s = torch.empty(5, c, dtype=torch.int8, device="cuda"), torch.empty(5, device="cuda")
        a.f8_quantize_rows(x, q, s, y=x)
        same_codes(keep.float(), q, s, x)


# ------------------------------------------------------------------ the step between two blocks

KINDS = {"none": 0, "rms": 1, "layer": 2}


def _step(rng, n, c, t, *, post="none", pre="rms", gate="none", gate_act="none", residual=True, wt=F32, weights=True, bias=False, offset=0.0, beta=1.0,
          eps=1e-5, codes=True, values=True, total=True, shift=0.0, pad=0, off=0, inplace=False):
    a = api()

    def rows(scale, mean=0.0, fill=None):
        v, _ = strided(n, c, t, pad, off, fill=fill)
        v.copy_((torch.from_numpy(rng.normal(mean, scale, size=(n, c)))).to(t))
        return v
    x, r = rows(1.0), rows(2.0, shift) if residual else None
    g = None if gate == "none" else torch.from_numpy(rng.normal(0, 1, size=(n if gate == "token" else 1, c))).to(t).cuda()
    vec = lambda m, s: torch.from_numpy(rng.normal(m, s, size=c)).to(wt).cuda()      # noqa: E731
    post_w = vec(1 - offset, 0.1) if post != "none" and weights else None
    pre_w = vec(1 - offset, 0.1) if pre != "none" and weights else None
    post_b = vec(0, 0.1) if post != "none" and bias else None
    pre_b = vec(0, 0.1) if pre != "none" and bias else None
    act = {"none": a.F8_ACT_NONE, "sigmoid": a.F8_ACT_SIGMOID, "tanh": a.F8_ACT_TANH}[gate_act]
    x64, r64 = x.double(), r.double() if residual else torch.zeros(n, c, dtype=torch.float64, device="cuda")
    z, ze = norm64(x64, torch.zeros_like(x64), KINDS[post], post_w, post_b, offset, eps)
    if g is not None:
        g64 = g.double()
        g64 = torch.sigmoid(g64) if gate_act == "sigmoid" else torch.tanh(g64) if gate_act == "tanh" else g64
        ze = ze * g64.abs() + (z * g64).abs() * ((10 + 2.4 * g.double().abs()) * 2 * U if gate_act != "none" else 0) + U * (z * g64).abs()
        z = z * g64
    t64 = r64 + beta * z
    te = abs(beta) * ze + U * t64.abs() + abs(beta) * 2.0 ** -24 * z.abs()
    v, ve = norm64(t64, te, KINDS[pre], pre_w, pre_b, offset, eps)

    q, s = (strided(n, c, torch.int8, pad, off, fill=0)[0], torch.empty(n, device="cuda")) if codes else (None, None)
    y = strided(n, c, t, pad, off)[0] if values else None
    so = (r if inplace and residual else strided(n, c, t, pad, off)[0]) if total else None
    a.f8_norm_quantize(x, q, s, y, residual=r, residual_out=so, gate=g, gate_act=act, post_norm=KINDS[post], post_w=post_w, post_b=post_b,
                       pre_norm=KINDS[pre], pre_w=pre_w, pre_b=pre_b, eps=eps, weight_offset=offset, branch_scale=beta)
    torch.cuda.synchronize()
    if total:
        over = (so.double() - t64).abs() - 1.01 * (te + half_step(t) * t64.abs()) - tiny(t)
        assert bool((over <= 0).all()), f"residual sum off by {over.max().item()} more than the bound"
    if codes:
        check_codes(v, ve, q, s, y, "step")
    elif values:
        over = (y.double() - v).abs() - 1.01 * (ve + half_step(t) * v.abs()) - tiny(t)
        assert bool((over <= 0).all()), f"values off by {over.max().item()} more than the bound"


@pytest.mark.parametrize("post,pre", list(itertools.product(["none", "rms", "layer"], repeat=2)))
@pytest.mark.parametrize("gate", ["none", "channel", "token"])
@pytest.mark.parametrize("t", [BF16, F16, F32])
def test_step(post, pre, gate, t):
    rng = np.random.default_rng(11)
    for n, c in ((1, 1), (3, 65), (5, 1537), (2, 4096)):
        _step(rng, n, c, t, post=post, pre=pre, gate=gate, beta=0.25, bias=pre == "layer")


@pytest.mark.parametrize("n,c", SHAPES + [(300, 128), (777, 1537), (260, 3000), (150, 8192)])
def test_step_shapes(n, c):
    rng = np.random.default_rng(n + c)
    _step(rng, n, c, BF16, post="rms", pre="rms", gate="channel", beta=0.5)
    _step(rng, n, c, F16, pre="layer", bias=True, gate="token")


@pytest.mark.parametrize("n,c", [(1184, 8192), (1185, 8000), (2369, 4096), (4737, 2048), (9473, 1000), (9999, 1024), (1300, 16384)])
@pytest.mark.parametrize("t", [BF16, F16, F32])
def test_step_with_many_rows(n, c, t):
    """Several rounds of rows for every block, which then takes two rows at once between blocks with the usual options; odd numbers of rows."""
    rng = np.random.default_rng(n)
    _step(rng, n, c, t, post="rms", gate="channel", beta=0.5)
    _step(rng, n, c, t, values=False, inplace=True)
    _step(rng, n, c, t, post="rms", gate="token", gate_act="sigmoid", pre="layer", bias=True)


@pytest.mark.parametrize("c", [2048, 8192])
def test_rows_of_a_pair_do_not_mix(c):
    """Rows that are not finite, zero or tiny next to ordinary ones, where two rows share their sums."""
    a = api()
    n = 8 * 148 * (1024 // (c // 8)) + 3
    x, r = torch.randn(n, c, device="cuda").to(BF16), torch.randn(n, c, device="cuda").to(BF16)
    kinds = torch.arange(n, device="cuda") % 5
    x[kinds == 1], r[kinds == 1] = 0, 0
    r[kinds == 2, 7] = float("nan")
    x[kinds == 3, c - 1] = float("inf")
    q, s, so = torch.full((n, c), 9, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda"), torch.empty_like(r)
    w = torch.ones(c, device="cuda")
    a.f8_norm_quantize(x, q, s, residual=r, residual_out=so, post_norm=a.F8_NORM_RMS, post_w=w, pre_w=w)
    one = [i for i in range(n) if i % 5 in (0, 4)]
    q1, s1, so1 = torch.empty(1, c, dtype=torch.int8, device="cuda"), torch.empty(1, device="cuda"), torch.empty(1, c, dtype=BF16, device="cuda")
    assert not bool(s[kinds == 1].any()) and not bool(q[kinds == 1].any())
    assert bool(torch.isnan(s[(kinds == 2) | (kinds == 3)]).all()) and not bool(q[(kinds == 2) | (kinds == 3)].any())
    for i in one[:4] + one[-4:]:
        a.f8_norm_quantize(x[i:i + 1], q1, s1, residual=r[i:i + 1], residual_out=so1, post_norm=a.F8_NORM_RMS, post_w=w, pre_w=w)
        assert bool(((q1[0].int() - q[i].int()).abs() <= 1).all()) and abs(float(s1) - float(s[i])) <= 1e-5 * float(s1)
        assert bool(((so1[0].float() - so[i].float()).abs() <= 2.0 ** -7 * so[i].float().abs() + 1e-6).all())


@pytest.mark.parametrize("codes,values,total", [(True, False, True), (True, False, False), (False, True, True), (False, True, False), (False, False, True),
                                                (True, True, False)])
@pytest.mark.parametrize("c", [64, 1000, 4096, 20000])
def test_step_outputs(codes, values, total, c):
    _step(np.random.default_rng(c), 4, c, BF16, codes=codes, values=values, total=total, post="layer", bias=True)


@pytest.mark.parametrize("act", ["sigmoid", "tanh"])
@pytest.mark.parametrize("gate", ["channel", "token"])
def test_step_gates(act, gate):
    for t in (BF16, F32):
        _step(np.random.default_rng(1), 6, 640, t, gate=gate, gate_act=act, beta=1.5)


@pytest.mark.parametrize("kw", [dict(residual=False), dict(weights=False), dict(offset=1.0), dict(wt=BF16), dict(wt=BF16, bias=True, pre="layer"), dict(inplace=True),
                                dict(shift=300.0, pre="layer", bias=True), dict(eps=0.0), dict(pre="none"), dict(pad=8, off=8), dict(pad=1, off=3),
                                dict(beta=0.0), dict(post="rms", wt=BF16, offset=1.0)])
def test_step_options(kw):
    for n, c in ((3, 320), (2, 1001), (4, 4096), (1, 17000)):
        _step(np.random.default_rng(2), n, c, BF16, **kw)


def test_step_rows_without_spread_and_not_finite():
    a = api()
    c = 512
    x = torch.zeros(6, c, dtype=BF16, device="cuda")
    r = torch.zeros(6, c, dtype=BF16, device="cuda")
    r[1] = 3.0                       # a layer norm of equal values is zero
    r[2, 5] = float("nan")
    r[3, 7] = float("inf")
    r[4] = torch.randn(c, device="cuda").to(BF16)
    q, s, y = torch.full((6, c), 9, dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda"), torch.empty(6, c, dtype=BF16, device="cuda")
    a.f8_norm_quantize(x, q, s, y, residual=r, pre_norm=a.F8_NORM_LAYER)
    for i in (0, 1, 5):
        assert float(s[i]) == 0 and not q[i].any() and not y[i].any()
    for i in (2, 3):
        assert torch.isnan(s[i]) and not q[i].any() and torch.isnan(y[i]).all()
    assert float(s[4]) > 0 and int(q[4].abs().max()) == 127


def test_rows_captured_and_replayed():
    a = api()
    n, c = 65, 2048
    x, r = torch.randn(n, c, device="cuda").to(BF16), torch.randn(n, c, device="cuda").to(BF16)
    w = torch.ones(c, device="cuda")
    q, s, so = torch.empty(n, c, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda"), torch.empty_like(r)
    q2, s2 = torch.empty_like(q), torch.empty_like(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a.f8_norm_quantize(x, q, s, residual=r, residual_out=so, pre_w=w)
        a.f8_quantize_rows(so, q2, s2)
    x.copy_(torch.randn(n, c, device="cuda"))
    g.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in (q, s, so, q2, s2)]
    a.f8_norm_quantize(x, q, s, residual=r, residual_out=so, pre_w=w)
    a.f8_quantize_rows(so, q2, s2)
    assert all(torch.equal(u, v) for u, v in zip(got, (q, s, so, q2, s2)))
    same_codes(so.float(), q2, s2)


@pytest.mark.parametrize("ld,c", [(2_300_000_000, 4096), (2_300_000_001, 515), (1_200_000_000, 20001)])
def test_rows_beyond_four_gigabytes(ld, c):
    """Rows whose distance passes 32 bits, in bytes and in elements: the last row of each tensor is the one looked at."""
    a = api()
    flat = torch.zeros(2 * ld + c + 64, dtype=BF16, device="cuda")
    x = torch.as_strided(flat, (3, c), (ld, 1))
    x[2] = torch.randn(c, device="cuda")
    q, s, y = torch.empty(3, c, dtype=torch.int8, device="cuda"), torch.empty(3, device="cuda"), torch.empty(3, c, dtype=BF16, device="cuda")
    a.f8_quantize_rows(x, q, s, y=y)
    same_codes(x.float(), q, s, y)
    keep = x.float()
    a.f8_norm_quantize(x, None, None, y, residual=x, residual_out=x, pre_norm=a.F8_NORM_NONE)
    assert torch.equal(x.float(), 2 * keep) and torch.equal(y.float(), 2 * keep)


def test_many_rows_beyond_four_gigabytes():
    a = api()
    n, c = 600_000, 4096
    x = torch.zeros(n, c, dtype=BF16, device="cuda")
    x[-3:] = torch.randn(3, c, device="cuda")
    q, s = torch.full((n, c), 5, dtype=torch.int8, device="cuda"), torch.full((n,), 7.0, device="cuda")
    a.f8_quantize_rows(x, q, s)
    same_codes(x[-3:].float(), q[-3:], s[-3:])
    assert not bool(s[:-3].any()) and not bool(q[:-3].any())
    out = torch.empty_like(x)
    a.f8_norm_quantize(x, q, s, residual=x, residual_out=out, pre_norm=a.F8_NORM_NONE)
    assert torch.equal(out[-3:].float(), 2 * x[-3:].float()) and not bool(out[:-3].any())


def test_no_rows():
    a = api()
    x = torch.zeros(0, 64, device="cuda")
    a.f8_quantize_rows(x, torch.zeros(0, 64, dtype=torch.int8, device="cuda"), torch.zeros(0, device="cuda"))
    a.f8_norm_quantize(x, torch.zeros(0, 64, dtype=torch.int8, device="cuda"), torch.zeros(0, device="cuda"))


def _every_number(t):
    return torch.arange(-2 ** 15, 2 ** 15, dtype=torch.int32).to(torch.int16).view(t).cuda()


@pytest.mark.parametrize("t", [BF16, F16])
def test_silu_of_every_number_is_a_32_bit_result(t):
    """The scale of a row is a 32-bit number: of rows of one element each it shows the activation's own error."""
    a = api()
    x = _every_number(t)
    x = x[torch.isfinite(x) & (x > -88.7)].view(-1, 1).contiguous()         # (below, exp(-x) is infinite in 32 bits)
    # a gate that brings the far ends back into range: a power of two, exact
    u = torch.where(x < -40, 2.0 ** 60 if t == BF16 else 2.0 ** 15, torch.where((x.abs() < 2.0 ** -60), 2.0 ** 60, 1.0)).to(t)
    q, s = torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(x.shape[0], device="cuda")
    a.f8_quantize_rows(x, q, s, u=u, act=a.F8_ACT_SILU)
    want = (silu(x.double()) * u.double())[:, 0].abs()
    some = want >= 2.0 ** -100 * (1 + 2.0 ** -16)
    # exponential and reciprocal within 2^-22 and 2^-23, four roundings between them, the gate and the division of the scale: 4 + 2 + 6 half steps
    assert bool(((s.double() - want / 127).abs() <= 1.01 * 12 * U * want / 127)[some].all())
    assert int(some.sum()) > (30000 if t == BF16 else 40000) and bool((s[want < 2.0 ** -100 * (1 - 2.0 ** -16)] == 0).all())


@pytest.mark.parametrize("t", [BF16, F16, F32])
def test_silu_far_out_and_not_finite(t):
    a = api()
    far = torch.finfo(t).max
    x = torch.tensor([[far, -far, INF, -INF, float("nan"), 200.0, -200.0, 126.0, -126.0, 0.0, -0.0, -87.5, -88.5]], device="cuda").to(t)
    for c in (1, 20000):                            # in registers, and a row of any length
        rows = x.t().expand(-1, c).contiguous()
        y = torch.empty_like(rows)
        a.f8_quantize_rows(rows, y=y, act=a.F8_ACT_SILU)
        y = y.double()
        assert bool((y == y[:, :1]).logical_or(y.isnan()).all())
        got = y[:, 0].tolist()
        assert got[0] == far and got[1] == 0 and got[2] == INF and got[3] != got[3] and got[4] != got[4]
        assert got[5] == 200 and got[6] == 0 and got[7] == 126 and abs(got[8]) < 1e-36 and got[9] == 0 and got[10] == 0
        for i in (11, 12):
            z = silu(x[0, i].double()).item()
            assert abs(got[i] - z) <= (half_step(t) + 12 * U) * abs(z) + tiny(t) + 1e-45


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("c", [100, 3000, 20000])
def test_scales_of_negative_activations(t, c):
    """Rows whose values are all far below zero, where the exponential of a rounded product would be off by the size of the product."""
    a = api()
    rng = np.random.default_rng(c)
    x = torch.from_numpy(rng.uniform(-35, -15, size=(20, c)) if t == BF16 else rng.uniform(-16, -8, size=(20, c))).to(t).cuda()
    q, s = torch.empty(20, c, dtype=torch.int8, device="cuda"), torch.empty(20, device="cuda")
    a.f8_quantize_rows(x, q, s, act=a.F8_ACT_SILU)
    v = silu(x.double())
    check_codes(v, v.abs() * 11 * U, q, s)


@pytest.mark.parametrize("t", [BF16, F32])
@pytest.mark.parametrize("c", [480, 1000, 1500, 2040, 2500, 3000, 4000, 5000, 6100, 8000, 10000, 12200, 16000])
def test_every_number_of_threads(c, t):
    """Rows that take every number of threads a block may have, some elements short of all of them, in each of the layouts; with rows in every block's
    second round."""
    a = api()
    rng = np.random.default_rng(c)
    n = 1200
    for width, pad, offset in ((c, 0, 0), (c - 1, 0, 1), (c - 3, 2, 0)):
        x, _ = strided(n, width, t, pad, offset)
        x.copy_(_values(rng, n, width, t))
        x[::7] *= 100
        x[5, width - 1] = 1000          # the largest of its row is the last element, of another the first
        x[6, 0] = -1000
        q, s, y = torch.empty(n, width, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, width, dtype=t, device="cuda")
        a.f8_quantize_rows(x, q, s, y=y)
        same_codes(x.float(), q, s, y)
        u = _values(rng, n, width, t)
        a.f8_quantize_rows(x, q, s, u=u)
        same_codes(x.float() * u.float(), q, s)
