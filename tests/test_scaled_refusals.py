"""Argument checks of the entry points on real-valued tensors: they run on the host, before anything is enqueued."""
import ctypes

import pytest
import torch

from paper_2202_05239_b200 import api

A = ctypes.c_void_p(0x1000)          # never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x1001)
NAN, INF = float("nan"), float("inf")


def _scaled(**kw):
    base = dict(n=4, k=64, out=8, x_dtype=api.F8_S8, y_dtype=api.F8_BF16, bias_dtype=api.F8_F32, x_scales=4, w_scales=8, ldx=0, ldw=0, ldy=0)
    base.update(kw)
    return api.ScaledDesc(**base)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), 2), (dict(k=0), 2), (dict(out=0), 2), (dict(x_dtype=api.F8_S32), 3), (dict(y_dtype=api.F8_S8), 3), (dict(y_dtype=7), 3),
    (dict(bias_dtype=api.F8_S32), 3), (dict(x_scales=2), 2), (dict(w_scales=4), 2), (dict(ldx=63), 2), (dict(ldw=-64), 2), (dict(ldy=7), 2),
    (dict(ldx=1 << 50), 2), (dict(k=131072), 7), (dict(k=65794, x_dtype=api.F8_U8), 7)])
def test_scaled_product_refuses(kw, status):
    d = _scaled(**kw)
    assert api._lib.f8_linear_scaled(ctypes.byref(d), A, A, A, A, A, A, None) == status, api._lib.f8_last_error()


def test_scaled_product_refuses_pointers():
    d, f = _scaled(), api._lib.f8_linear_scaled
    assert f(None, A, A, A, A, None, A, None) == 1
    for i in (0, 1, 2, 3, 5):
        p = [A, A, A, A, None, A]
        p[i] = None
        assert f(ctypes.byref(d), *p, None) == 1
    for i in (1, 3, 4, 5):
        p = [A, A, A, A, A, A]
        p[i] = ODD
        assert f(ctypes.byref(d), *p, None) == 6
    assert f(ctypes.byref(_scaled(n=0, x_scales=1)), None, None, None, None, None, None, None) == 0


def _rows(**kw):
    base = dict(n=4, c=64, dtype=api.F8_BF16, act=0, ldx=0, ldu=0, ldy=0, ldq=0)
    base.update(kw)
    return api.RowsDesc(**base)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), 2), (dict(n=1 << 31), 2), (dict(c=0), 2), (dict(dtype=api.F8_S8), 3), (dict(dtype=9), 3), (dict(act=3), 9), (dict(act=-1), 9), (dict(ldx=63), 2), (dict(ldu=1), 2),
    (dict(ldy=-1), 2), (dict(ldq=63), 2), (dict(ldx=1 << 49), 2)])
def test_rows_refuse(kw, status):
    assert api._lib.f8_quantize_rows(ctypes.byref(_rows(**kw)), A, A, A, A, A, None) == status, api._lib.f8_last_error()


def test_rows_refuse_pointers():
    d, f = ctypes.byref(_rows()), api._lib.f8_quantize_rows
    assert f(None, A, None, A, A, None, None) == 1
    assert f(d, None, None, A, A, None, None) == 1
    assert f(d, A, None, None, None, None, None) == 1       # no output
    assert f(d, A, None, A, None, None, None) == 1          # codes without scales
    assert f(d, A, None, None, A, A, None) == 1             # scales without codes
    for p in ((ODD, None, A, A, None), (A, ODD, A, A, None), (A, None, A, ODD, None), (A, None, A, A, ODD)):
        assert f(d, *p, None) == 6
    assert f(ctypes.byref(_rows(n=0)), None, None, None, None, None, None) == 0


def _norm(**kw):
    base = dict(n=4, c=64, dtype=api.F8_BF16, w_dtype=api.F8_F32, post_norm=1, pre_norm=1, gate_act=0, gate_rows=4, eps=1e-5, weight_offset=0.0, branch_scale=1.0,
                ldx=0, ldg=0, ldr=0, lds=0, ldy=0, ldq=0)
    base.update(kw)
    return api.NormDesc(**base)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), 2), (dict(c=0), 2), (dict(dtype=api.F8_S32), 3), (dict(w_dtype=api.F8_F16), 3), (dict(post_norm=3), 9), (dict(pre_norm=-1), 9), (dict(gate_act=1), 9),
    (dict(post_norm=0), 9), (dict(pre_norm=0), 9), (dict(gate_rows=2), 2), (dict(eps=-1.0), 2), (dict(eps=NAN), 2), (dict(eps=INF), 2), (dict(weight_offset=NAN), 2),
    (dict(branch_scale=INF), 2), (dict(ldx=63), 2), (dict(ldg=63), 2), (dict(ldr=63), 2), (dict(lds=63), 2), (dict(ldy=63), 2), (dict(ldq=63), 2)])
def test_norm_refuses(kw, status):
    assert api._lib.f8_norm_quantize(ctypes.byref(_norm(**kw)), *([A] * 11), None) == status, api._lib.f8_last_error()


def test_norm_refuses_pointers():
    d, f = ctypes.byref(_norm()), api._lib.f8_norm_quantize
    assert f(None, *([A] * 11), None) == 1
    for missing in ([0], [7, 8, 9, 10], [9], [8]):           # x; every output; scales; codes
        p = [None if i in missing else A for i in range(11)]
        assert f(d, *p, None) == 1
    for i in (0, 1, 2, 3, 4, 5, 6, 7, 9, 10):
        p = [ODD if j == i else A for j in range(11)]
        assert f(d, *p, None) == 6
    assert f(ctypes.byref(_norm(n=0)), *([None] * 11), None) == 0


def _lp(**kw):
    base = dict(n=4, v=100, dtype=api.F8_BF16, fl=0, tokens=2, top=5, inv_temperature=1.0, ldl=0)
    base.update(kw)
    return api.LogprobsDesc(**base)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), 2), (dict(v=0), 2), (dict(tokens=-1), 2), (dict(top=33), 2), (dict(top=-1), 2), (dict(v=4), 2), (dict(dtype=api.F8_U8), 3), (dict(dtype=api.F8_S32, fl=33), 4),
    (dict(dtype=api.F8_S32, fl=-9), 4), (dict(inv_temperature=0.0), 2), (dict(inv_temperature=-1.0), 2), (dict(inv_temperature=NAN), 2), (dict(inv_temperature=INF), 2), (dict(inv_temperature=3e38), 2),
    (dict(dtype=api.F8_S32, fl=-8, inv_temperature=3e38), 2), (dict(dtype=api.F8_S32, fl=32, inv_temperature=1e-44), 2), (dict(ldl=99), 2), (dict(ldl=1 << 49), 2)])
def test_logprobs_refuse(kw, status):
    assert api._lib.f8_token_logprobs(ctypes.byref(_lp(**kw)), A, A, A, A, A, A, None) == status, api._lib.f8_last_error()


def test_logprobs_refuse_pointers():
    d, f = ctypes.byref(_lp()), api._lib.f8_token_logprobs
    assert f(None, A, A, A, A, A, A, None) == 1
    assert f(d, None, A, A, A, A, A, None) == 1
    assert f(d, A, None, A, A, A, A, None) == 1             # log probabilities of no tokens
    assert f(d, A, A, None, None, None, None, None) == 1    # no output
    assert f(ctypes.byref(_lp(top=0)), A, A, None, None, A, A, None) == 1
    for i in range(6):
        p = [ctypes.c_void_p(0x1001 if j == i else 0x1000) for j in range(6)]
        assert f(d, *p, None) == 6
    assert f(ctypes.byref(_lp(n=0)), None, None, None, None, None, None, None) == 0


def test_binding_refuses_wrong_tensors():
    """Shapes, types, strides and places are checked before the library is called."""
    x, w, one = torch.zeros(4, 64, dtype=torch.int8), torch.zeros(8, 64, dtype=torch.int8), torch.ones(1)
    with pytest.raises(ValueError, match="x: .*CUDA device"):
        api.f8_linear_scaled(x, one, w, one, torch.zeros(4, 8))
    for bad in (None, 3, "x", [1, 2]):
        with pytest.raises(ValueError, match="x: a tensor is needed"):
            api.f8_linear_scaled(bad, one, w, one, torch.zeros(4, 8))
    with pytest.raises(ValueError):
        api.f8_quantize_rows(torch.zeros(4, 64, dtype=torch.int8))
    with pytest.raises(ValueError):
        api.f8_norm_quantize(torch.zeros(4, 64))
    with pytest.raises(ValueError):
        api.f8_token_logprobs(torch.zeros(4, 64, dtype=torch.int8))


@pytest.mark.parametrize("extent,status", [(2 ** 31 - 255, 2), (2 ** 31 - 1, 2), (2 ** 31 - 256, 6)])
def test_longest_rows(extent, status):
    """Rows that the kernels could not count through in 32 bits are refused; the longest others come as far as the check of their pointers."""
    b = ctypes.byref
    assert api._lib.f8_quantize_rows(b(_rows(c=extent, n=1)), ODD, A, A, A, A, None) == status
    assert api._lib.f8_norm_quantize(b(_norm(c=extent, n=1, gate_rows=1)), ODD, *([A] * 10), None) == status
    assert api._lib.f8_token_logprobs(b(_lp(v=extent, n=1)), ODD, A, A, A, A, A, None) == status
    assert api._lib.f8_token_logprobs(b(_lp(tokens=extent, n=1)), ODD, A, A, A, A, A, None) == status
    assert api._lib.f8_linear_scaled(b(_scaled(out=extent, w_scales=1, n=1, x_scales=1)), A, ODD, A, A, A, A, None) == status
