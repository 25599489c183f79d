"""The operators of an encoder served in 8 bits, in 64 bits from their
definitions (CPU), with bounds on what rounding may cost a correct kernel.

u is the rounding of the features' type (half an ulp of 1); E32 that of 32-bit
steps.  A value in 8 bits is off by half a step; where 32-bit steps before the
rounding move a value over a border between two whole numbers, that is half a
step and what they moved it by.
"""

import math

import torch

from tests.encoder_reference import TINY, UNIT, check, rotary  # noqa: F401

E32 = 2.0 ** -24


def sum_error(n):
    """Relative error of a 32-bit sum of n terms of one sign in a few partial
    sums, and of some ten 32-bit steps after it."""
    return E32 * (12 + 4 * math.log2(n + 1))


def rms_norm(x, weight, eps, residual=None, grad_y=None, grad_sum=None):
    # (float16 numbers below 2^-14 are 2^-24 apart: rounding to one is off by up to 2^-25, TINY, whatever its size)
    dtype, u, tiny = x.dtype, UNIT[x.dtype], TINY[x.dtype] + 1e-30
    h = x.double()
    r, b = {}, {}
    if residual is not None:
        h = (x.float() + residual.float()).to(dtype).double()
        r["h"], b["h"] = h, torch.zeros_like(h)
    n = x.shape[1]
    rstd = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    xh = h * rstd
    w = torch.ones(n, dtype=torch.float64) if weight is None else weight.double()
    y = xh * w
    e = sum_error(n)
    r["rstd"], b["rstd"] = rstd[:, 0], e * rstd[:, 0]
    r["y"], b["y"] = y, (u + e) * y.abs() + tiny
    r["y32"], b["y32"] = y, e * y.abs() + 1e-30
    if grad_y is None:
        return r, b
    g0 = grad_y.double()
    g = g0 * w
    m = (g * xh).mean(1, keepdim=True)
    dx = rstd * (g - xh * m)
    off = rstd * e * (g.abs() + 2 * xh.abs() * (g * xh).abs().mean(1, keepdim=True))
    if grad_sum is not None:
        dx = dx + grad_sum.double()
        off = off + E32 * (grad_sum.double().abs() + dx.abs())
    r["dx"], b["dx"] = dx, u * dx.abs() + off + tiny
    # sums over the rows: blocks of rows in a row each, then joined
    many = E32 * (12 + x.shape[0] ** 0.5)
    r["dw"], b["dw"] = (g0 * xh).sum(0), (many + e) * (g0 * xh).abs().sum(0) + 1e-30
    return r, b


def check_whole(q, scale, y, y_error, name="q"):
    """Rows in 8 bits against y in 64 bits, which 32-bit steps had off by y_error."""
    q, scale = q.cpu().double(), scale.cpu().double()
    most = y.abs().amax(1)
    off = (y_error / y.abs().clamp_min(1e-300)).amax(1) + 4 * E32
    assert ((scale - most / 127).abs() <= off * most / 127 + 1e-35).all(), f"{name}: scales"
    assert (q.abs() <= 127).all()
    err = (q * scale[:, None] - y).abs()
    # half a step; the 32-bit quotient before the rounding is off by some steps of 32 bits
    bound = scale[:, None] * (0.5 + 127 * (off[:, None] + 4 * E32)) + y_error
    assert (err <= bound).all(), f"{name}: off by up to {(err / scale[:, None].clamp_min(1e-300)).max():.4f} of a step"
