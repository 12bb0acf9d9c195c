"""8-bit products with a real scale per token and channel (f8_linear_scaled) against the product in 64 bits."""
import numpy as np
import pytest
import torch

from gpu_util import Guarded, api
from scaled_util import U, half_step, strided, tiny

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def _codes(rng, rows, cols, dtype):
    lo, hi = (0, 256) if dtype == torch.uint8 else (-128, 128)
    return torch.from_numpy(rng.integers(lo, hi, size=(rows, cols))).to(dtype)


def _check(y, x, xs, w, ws, bias):
    p = (x.double() @ w.double().t()) * xs.double().reshape(-1, 1) * ws.double().reshape(1, -1)
    want = p if bias is None else p + bias.double()
    t = y.dtype
    # acc to float, times sx, fused with sw and the bias: three roundings in 32 bits, then the type's own
    tol = 1.01 * (2 * U * p.abs() + (U + half_step(t)) * want.abs()) + tiny(t)
    off = (y.double() - want).abs()
    assert bool((off <= tol).all()), f"{int((off > tol).sum())} of {off.numel()} are off, worst {(off / tol).max().item():.3g} times the bound"


def _run(rng, n, k, out, *, xt=torch.int8, yt=BF16, bt=None, per_x=True, per_w=True, padx=0, padw=0, pady=0, offx=0, offw=0, offy=0, stream=None):
    a = api()
    x, _ = strided(n, k, xt, padx, offx, fill=99)
    w, _ = strided(out, k, torch.int8, padw, offw, fill=99)
    x.copy_(_codes(rng, n, k, xt))
    w.copy_(_codes(rng, out, k, torch.int8))
    xs = torch.from_numpy(rng.uniform(0.001, 0.05, n if per_x else 1)).float().cuda()
    ws = torch.from_numpy(rng.uniform(0.0005, 0.002, out if per_w else 1)).float().cuda()
    bias = None if bt is None else torch.from_numpy(rng.normal(0, 3, out)).to(bt).cuda()
    y, flat = strided(n, out, yt, pady, offy, fill=7.0)
    a.f8_linear_scaled(x, xs, w, ws, y, bias=bias, stream=stream)
    torch.cuda.synchronize()
    a.f8_device_status()
    _check(y, x, xs, w, ws, bias)
    assert not bool(x._base[offx + n * (k + padx):].ne(99).any())
    untouched = flat.clone()
    untouched[offy:offy + n * (out + pady)].view(n, out + pady)[:, :out] = 7.0
    assert bool((untouched == 7.0).all()), "something beside the output was written"
    return x, xs, w, ws, bias, y


@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 16, 17, 33, 64, 65, 127, 128, 129, 200, 257, 300])
@pytest.mark.parametrize("k,out", [(64, 16), (128, 128), (416, 136), (1024, 264), (4096, 72)])
def test_rows_and_widths(n, k, out):
    _run(np.random.default_rng(n * 7 + k), n, k, out)


@pytest.mark.parametrize("yt", [BF16, F16, F32])
@pytest.mark.parametrize("bt", [None, F32, F16, BF16])
@pytest.mark.parametrize("xt", [torch.int8, torch.uint8])
@pytest.mark.parametrize("n", [3, 150])
def test_types(xt, yt, bt, n):
    _run(np.random.default_rng(5), n, 320, 200, xt=xt, yt=yt, bt=bt)


@pytest.mark.parametrize("per_x,per_w", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("n", [1, 40, 260])
def test_one_scale_for_all(per_x, per_w, n):
    _run(np.random.default_rng(6), n, 256, 100, per_x=per_x, per_w=per_w, bt=F32)


@pytest.mark.parametrize("k", [1, 3, 15, 16, 17, 31, 33, 63, 65, 100, 127, 129, 1000, 1001, 2047])
@pytest.mark.parametrize("n,out", [(1, 1), (5, 33), (70, 65), (140, 300)])
def test_odd_k(n, k, out):
    _run(np.random.default_rng(k), n, k, out, bt=BF16)


@pytest.mark.parametrize("n", [1, 20, 131, 300])
@pytest.mark.parametrize("padx,padw,pady,offx,offw,offy", [
    (16, 32, 8, 16, 32, 8),      # rows farther apart, still at multiples of 16 bytes
    (1, 0, 0, 0, 0, 0), (0, 3, 1, 0, 0, 0), (0, 0, 0, 1, 0, 0), (0, 0, 0, 0, 5, 1), (4, 8, 3, 4, 8, 5), (0, 0, 1, 0, 0, 0)])
def test_strides_and_offsets(n, padx, padw, pady, offx, offw, offy):
    _run(np.random.default_rng(n), n, 192, 144, padx=padx, padw=padw, pady=pady, offx=offx, offw=offw, offy=offy)


@pytest.mark.parametrize("n,out", [(1, 1), (1, 7), (4, 1000), (23, 8191), (200, 1001), (256, 1000), (513, 2050)])
@pytest.mark.parametrize("yt", [BF16, F32])
def test_odd_outputs(n, out, yt):
    _run(np.random.default_rng(out), n, 512, out, yt=yt)


@pytest.mark.parametrize("n,k,out", [(1, 16384, 4096), (16, 8192, 1024), (48, 11008, 512), (700, 4096, 1536), (2049, 1024, 2304), (4500, 640, 520)])
def test_larger(n, k, out):
    _run(np.random.default_rng(n), n, k, out)


@pytest.mark.parametrize("xt,k", [(torch.uint8, 65793), (torch.int8, 131071), (torch.uint8, 65776), (torch.int8, 131056)])
@pytest.mark.parametrize("n", [1, 130])
def test_longest_sums(xt, k, n):
    """The largest sums that the 32-bit accumulator can be asked for, and their refusal one step beyond."""
    a = api()
    x = torch.full((n, k), 255 if xt == torch.uint8 else -128, dtype=xt, device="cuda")
    w = torch.full((3, k), -128, dtype=torch.int8, device="cuda")
    w[1] = 127
    one = torch.ones(1, device="cuda")
    y = torch.empty(n, 3, device="cuda")
    a.f8_linear_scaled(x, one, w, one, y)
    torch.cuda.synchronize()
    _check(y, x, one, w, one, None)
    limit = 65794 if xt == torch.uint8 else 131072
    with pytest.raises(a.F8Error) as e:
        a.f8_linear_scaled(torch.zeros(1, limit, dtype=xt, device="cuda"), one, torch.zeros(3, limit, dtype=torch.int8, device="cuda"), one, y[:1])
    assert e.value.status == 7


def test_what_is_not_finite_stays_in_its_row():
    a = api()
    rng = np.random.default_rng(3)
    x, w = _codes(rng, 140, 128, torch.int8).cuda(), _codes(rng, 96, 128, torch.int8).cuda()
    x[5] = 0
    xs = torch.full((140,), 0.01, device="cuda")
    xs[5], xs[77] = float("inf"), float("nan")
    ws = torch.full((96,), 0.001, device="cuda")
    y = torch.empty(140, 96, dtype=BF16, device="cuda")
    a.f8_linear_scaled(x, xs, w, ws, y)
    bad = torch.isnan(y).all(dim=1).nonzero().flatten().tolist()
    assert bad == [5, 77] and bool(torch.isfinite(y[[i for i in range(140) if i not in (5, 77)]]).all())


def test_overflow_of_the_output_type_is_infinite():
    a = api()
    x = torch.full((2, 64), 127, dtype=torch.int8, device="cuda")
    w = torch.full((1, 64), 127, dtype=torch.int8, device="cuda")
    y = torch.empty(2, 1, dtype=F16, device="cuda")
    a.f8_linear_scaled(x, torch.tensor([1.0, 0.01], device="cuda"), w, torch.ones(1, device="cuda"), y)
    assert torch.isinf(y[0, 0]) and abs(float(y[1, 0]) - 127 * 127 * 64 * 0.01) <= 8


@pytest.mark.parametrize("n", [4, 300])
def test_guard_bands(n):
    a = api()
    rng = np.random.default_rng(9)
    x, w = _codes(rng, n, 288, torch.int8).cuda(), _codes(rng, 312, 288, torch.int8).cuda()
    xs, ws = torch.full((n,), 0.01, device="cuda"), torch.full((312,), 0.001, device="cuda")
    out = Guarded((n, 312), BF16)
    a.f8_linear_scaled(x, xs, w, ws, out.t)
    torch.cuda.synchronize()
    assert out.intact()
    _check(out.t, x, xs, w, ws, None)


@pytest.mark.parametrize("n,k,out", [(1, 1024, 512), (24, 2048, 300), (300, 512, 640)])
def test_captured_replayed_and_on_other_streams(n, k, out):
    """A captured call follows what its inputs hold at the replay; two graphs and an eager call that overlap do not meet anywhere."""
    a = api()
    rng = np.random.default_rng(8)
    side = [torch.cuda.Stream() for _ in range(2)]
    sets = []
    for i in range(3):
        x, w = _codes(rng, n, k, torch.int8).cuda(), _codes(rng, out, k, torch.int8).cuda()
        xs, ws = torch.rand(n, device="cuda") * 0.01 + 0.001, torch.rand(out, device="cuda") * 0.001 + 0.0005
        sets.append((x, xs, w, ws, torch.empty(n, out, dtype=BF16, device="cuda")))
    a.f8_linear_scaled(*sets[0])
    torch.cuda.synchronize()
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            a.f8_linear_scaled(*sets[i])
        graphs.append(g)
    for x, _, _, _, y in sets:
        x.copy_(_codes(rng, n, k, torch.int8))
        y.fill_(float("nan"))
    torch.cuda.synchronize()
    for _ in range(20):
        for g, s in zip(graphs, side):
            with torch.cuda.stream(s):
                g.replay()
        a.f8_linear_scaled(*sets[2])
    torch.cuda.synchronize()
    a.f8_device_status()
    for x, xs, w, ws, y in sets:
        _check(y, x, xs, w, ws, None)


def test_same_result_every_time():
    a = api()
    rng = np.random.default_rng(2)
    for n, k, out in ((1, 4096, 4096), (37, 4096, 1000), (257, 2048, 1031)):
        x, w = _codes(rng, n, k, torch.int8).cuda(), _codes(rng, out, k, torch.int8).cuda()
        xs, ws = torch.rand(n, device="cuda"), torch.rand(out, device="cuda")
        ys = [torch.empty(n, out, device="cuda") for _ in range(5)]
        for y in ys:
            a.f8_linear_scaled(x, xs, w, ws, y)
        assert all(torch.equal(y, ys[0]) for y in ys[1:])


@pytest.mark.parametrize("n,k,out,ldw", [(2, 96, 3, 2_400_000_000), (2, 97, 3, 2_400_000_001), (300, 4096, 3, 2_400_000_000)])
def test_rows_beyond_four_gigabytes(n, k, out, ldw):
    """Rows of weights and of outputs whose distance from the first passes 32 bits."""
    a = api()
    rng = np.random.default_rng(k)
    flat = torch.zeros(2 * ldw + k + 64, dtype=torch.int8, device="cuda")
    w = torch.as_strided(flat, (out, k), (ldw, 1))
    w.copy_(_codes(rng, out, k, torch.int8))
    x = _codes(rng, n, k, torch.int8).cuda()
    xs, ws = torch.rand(n, device="cuda"), torch.rand(out, device="cuda")
    ldy = 3_000_000_000 if n == 2 else 20_000_000
    y = torch.as_strided(torch.zeros((n - 1) * ldy + out, dtype=BF16, device="cuda"), (n, out), (ldy, 1))
    a.f8_linear_scaled(x, xs, w, ws, y)
    torch.cuda.synchronize()
    a.f8_device_status()
    _check(y, x, xs, w, ws, None)


def test_many_rows_of_weights():
    """More than four gigabytes of weights, one token."""
    a = api()
    out, k = 600_000, 8192
    w = torch.zeros(out, k, dtype=torch.int8, device="cuda")
    w[-5:] = torch.randint(-127, 128, (5, k), dtype=torch.int8, device="cuda")
    x = torch.randint(-127, 128, (1, k), dtype=torch.int8, device="cuda")
    one, y = torch.full((1,), 0.01, device="cuda"), torch.full((1, out), 9.0, device="cuda")
    a.f8_linear_scaled(x, one, w, one, y)
    torch.cuda.synchronize()
    _check(y[:, -5:], x, one, w[-5:], one, None)
    assert not bool(y[:, :-5].any())


def test_a_pending_record_of_a_timeout_is_reported():
    """Every entry point looks at the record of a wait that ran out before it enqueues anything, and works again once it is cleared."""
    a = api()
    x, w, y = torch.ones(2, 64, dtype=torch.int8, device="cuda"), torch.ones(8, 64, dtype=torch.int8, device="cuda"), torch.zeros(2, 8, device="cuda")
    one, r = torch.ones(1, device="cuda"), torch.ones(2, 64, device="cuda")
    q, s, h = torch.zeros(2, 64, dtype=torch.int8, device="cuda"), torch.zeros(2, device="cuda"), torch.zeros(2, device="cuda")
    calls = [lambda: a.f8_linear_scaled(x, one, w, one, y), lambda: a.f8_quantize_rows(r, q, s), lambda: a.f8_norm_quantize(r, q, s), lambda: a.f8_token_logprobs(r, entropy=h)]
    for call in calls:
        call()
    torch.cuda.synchronize()
    y.zero_()
    a.f8_debug_wait_timeout_probe(1.0)
    torch.cuda.synchronize()
    for call in calls:
        with pytest.raises(a.F8Error) as e:
            call()
        assert e.value.status == 11
    with pytest.raises(a.F8Error):
        a.f8_device_status()
    assert not bool(y.any())
    for call in calls:
        call()
    torch.cuda.synchronize()
    a.f8_device_status()
    assert bool((y == 64).all())


def test_no_rows_is_a_noop():
    a = api()
    one = torch.ones(1, device="cuda")
    a.f8_linear_scaled(torch.zeros(0, 64, dtype=torch.int8, device="cuda"), one, torch.zeros(8, 64, dtype=torch.int8, device="cuda"), one,
                       torch.empty(0, 8, device="cuda"))


def test_sequence_of_dependent_calls():
    """Calls in a row, each reading what the one before wrote, while that may still be running."""
    a = api()
    torch.manual_seed(0)
    n, c = 48, 1024
    w = torch.randint(-127, 128, (c, c), dtype=torch.int8, device="cuda")
    ws = torch.full((c,), 1 / (73.0 * 32), device="cuda")
    x = torch.randn(n, c, device="cuda").to(BF16)
    q, s = torch.empty(n, c, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
    y = torch.empty(n, c, dtype=BF16, device="cuda")
    seen = []
    src = x
    for _ in range(30):
        a.f8_quantize_rows(src, q, s)
        a.f8_linear_scaled(q, s, w, ws, y)
        src = y
    torch.cuda.synchronize()
    last = y.clone()
    src = x
    for _ in range(30):
        a.f8_quantize_rows(src, q, s)
        torch.cuda.synchronize()
        a.f8_linear_scaled(q, s, w, ws, y)
        torch.cuda.synchronize()
        src = y
        seen.append(float(y.float().abs().max()))
    assert torch.equal(last, y) and seen[-1] > 0


@pytest.mark.parametrize("n", [4096 + 1, 4096 + 13, 4096 + 31, 4096 + 97, 4352 - 1])
@pytest.mark.parametrize("out,pady,yt", [(2304, 0, BF16), (2301, 0, BF16), (2049, 3, F32)])
def test_last_rows_that_fill_part_of_a_warp(n, out, pady, yt):
    """Many tiles for each pair of blocks, rows of the last ones that only some lanes of a warp have, stored in words and element by element."""
    _run(np.random.default_rng(n), n, 640, out, yt=yt, bt=F32, pady=pady)


@pytest.mark.parametrize("n", [5, 41, 100, 127])
@pytest.mark.parametrize("k", [512, 513])
def test_few_rows_that_fill_part_of_a_warp(n, k):
    """The same of the kernel that divides K, and of its form for rows that bulk copies cannot fetch."""
    _run(np.random.default_rng(n), n, k, 1031, yt=F16, bt=F16)
