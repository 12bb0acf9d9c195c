"""Plain 64-bit forms of the operators on real-valued rows, and error bounds for 32-bit arithmetic (not collected by pytest)."""
import math

import torch

U = 2.0 ** -24          # half a step of a 32-bit float, relative: the most one operation rounds by


def half_step(t: torch.dtype) -> float:
    return torch.finfo(t).eps / 2


def tiny(t: torch.dtype) -> float:
    """Half the distance of the type's smallest numbers: what a rounding may add where values are subnormal."""
    return torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2


def strided(rows, cols, dtype, pad=0, offset=0, fill=None):
    """A [rows, cols] view with `pad` elements between rows, `offset` elements into its allocation; and the allocation."""
    flat = torch.zeros(offset + rows * (cols + pad) + 64, dtype=dtype, device="cuda")
    if fill is not None:
        flat.fill_(fill)
    return flat[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols], flat


def silu(v):
    return v / (1 + torch.exp(-v))


def gelu(v):
    return 0.5 * v * torch.special.erfc(-v / math.sqrt(2.0))


def check_codes(v, err, q, scale, y=None, what=""):
    """Codes and scales of rows whose exact values are v (64 bits), each computed with an error of at most `err`.

    The scale is within the error of the largest value (and one rounding) of its definition; a code stands for a value no further than half a
    step from v, but for v's error and the three roundings of scale, inverse and division (each 2^-24 of at most 127 steps).
    """
    v, err, s = v.double(), err.double(), scale.double()
    peak, at = v.abs().max(dim=1)
    peak_err = (err.max(dim=1).values + 2 * U * peak) / 127
    assert bool(((s - peak / 127).abs() <= peak_err + 1e-45).all()), f"{what}: scale"
    # the inverse the kernel used is 127 / (127 s) but for roundings: compare in steps of its own scale
    steps = torch.where(s[:, None] > 0, v / s[:, None], torch.zeros_like(v))
    slack = torch.where(s[:, None] > 0, err / s[:, None], torch.zeros_like(v)) + 127 * 4 * U
    off = (q.double() - steps).abs()
    assert bool((off <= 0.5 + slack).all()), f"{what}: a code is {off.max().item()} steps off"
    assert int(q.abs().max()) <= 127
    if y is not None:       # the values: code times scale in 32 bits, rounded once
        assert torch.equal(y, (q.float() * scale[:, None]).to(y.dtype)), f"{what}: values"


def same_codes(v32, q, scale, y=None):
    """Codes of rows known exactly in 32 bits: equal to the definition, evaluated exactly in 64 bits."""
    a = v32.abs().amax(dim=1, keepdim=True)
    zeros = a < 2.0 ** -100
    top = torch.full_like(a, 127.0)         # tensors on both sides: torch multiplies by the reciprocal of a plain number
    inverse = torch.where(zeros, torch.zeros_like(a), top / a)
    s = torch.where(zeros, torch.zeros_like(a), a / top)
    want = torch.floor(v32.double() * inverse.double() + 0.5)
    assert torch.equal(scale, s[:, 0])
    assert torch.equal(q.double(), want)
    if y is not None:
        assert torch.equal(y, (q.float() * scale[:, None]).to(y.dtype))


def norm64(z, z_err, kind, w, b, offset, eps):
    """(value, error bound) of a norm in 64 bits, for a 32-bit evaluation of inputs with errors of at most z_err.

    Sums of c terms in any order of the kernels add at most (c / 32 + 64) times (a thread's own terms, then a tree); every other step rounds once.
    """
    if kind == 0:
        return z, z_err
    c = z.shape[1]
    depth = (c / 32 + 64) * U
    size = z.abs()
    if kind == 2:
        mean = z.mean(dim=1, keepdim=True)
        mean_err = depth * size.mean(dim=1, keepdim=True) + z_err.mean(dim=1, keepdim=True) + U * mean.abs()
        z = z - mean
        z_err = z_err + mean_err + U * z.abs()
    ms = (z * z).mean(dim=1, keepdim=True)
    ms_err = (2 * z.abs() * z_err + z_err * z_err).mean(dim=1, keepdim=True) + ms * (depth + 2 * U)
    rstd = 1 / torch.sqrt(ms + eps)
    rel = 0.5 * ms_err / (ms + eps) + 6 * U
    g = torch.ones(c, dtype=torch.float64, device=z.device) if w is None else w.double() + offset
    v = z * rstd * g
    err = (z_err * rstd * g.abs()) + v.abs() * (rel * 1.5 + 5 * U)
    if b is not None:
        v = v + b.double()
        err = err + U * v.abs()
    return v, err
