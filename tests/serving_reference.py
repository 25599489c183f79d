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


# --- tracks ---

PAGE = 64


def place(t):
    return 16 * (t % 16 // 4) + 4 * (t // 16) + t % 4


PLACES = [place(t) for t in range(PAGE)]


def in_order(v):
    """Values of pages [..., dim, 64 places] as [..., 64 tokens, dim]."""
    return v[..., PLACES].transpose(-1, -2)


def check_append(before, after, new_k, new_v, offsets, table, lengths, k_error):
    """The cache after append_tracks against what it was before and the new rows in 64
    bits (keys turned, off by up to k_error where they were turned).  before and after:
    (k, v, k_scale, v_scale) on the CPU."""
    pages, heads = before[2].shape
    touched = torch.zeros(pages, PAGE, dtype=torch.bool)   # places that may change
    began = torch.zeros(pages, dtype=torch.bool)           # pages whose scale may change
    for t in range(len(lengths)):
        rows = offsets[t + 1] - offsets[t]
        length = lengths[t]
        if rows < 0 or offsets[t] < 0 or offsets[t + 1] > len(new_k) or not rows <= length <= PAGE * table.shape[1]:
            continue
        start = length - rows
        for p in range(start // PAGE, (length + PAGE - 1) // PAGE):
            page = int(table[t, p])
            s0, s1 = max(start - p * PAGE, 0), min(length - p * PAGE, PAGE)
            if not 0 <= page < pages or s1 <= s0:
                continue
            row = offsets[t] + p * PAGE + s0 - start
            began[page] = True
            touched[page, :s1] = True
            for name, new, error in (("k", new_k, k_error), ("v", new_v, torch.zeros_like(new_v))):
                i = 0 if name == "k" else 1
                old, got = ((c[i][page] if name == "k" else in_order(c[i][page])).double() for c in (before, after))
                old_scale, scale = before[2 + i][page].double(), after[2 + i][page].double()
                y, e = new[row:row + s1 - s0].transpose(0, 1), error[row:row + s1 - s0].transpose(0, 1)
                most = y.abs().amax((1, 2)) / 127
                if s0:
                    most = torch.maximum(most, old_scale)
                off = 4 * E32 * most + e.amax((1, 2)) / 127
                assert ((scale - most).abs() <= off).all(), f"{name}_scale of track {t}, page {p}: {scale} for {most}"
                # half a step, and what 32-bit steps before the rounding moved
                err = (got[:, s0:s1] - y / scale[:, None, None]).abs()
                assert (err <= 0.5 + 127 * 4 * E32 + e / scale[:, None, None]).all(), f"{name} of track {t}, page {p}: {err.max()}"
                held = old[:, :s0] * (old_scale / scale)[:, None, None]
                err = (got[:, :s0] - held).abs()
                assert (err <= 0.5 + 127 * 4 * E32).all(), f"held {name} of track {t}, page {p}"
                for h in range(heads):
                    if old_scale[h] == scale[h]:
                        assert torch.equal(got[h, :s0], old[h, :s0]), f"held {name} of track {t}, page {p} changed"
    # nothing else is written
    for i in (0, 1):
        old, got = ((c[i] if i == 0 else in_order(c[i])).transpose(1, 2) for c in (before, after))
        assert torch.equal(old[~touched], got[~touched]), "places beyond the tracks' tokens were written"
        assert torch.equal(before[2 + i][~began], after[2 + i][~began])


def attention_tracks(q, cache, offsets, table, lengths, scale, cap=0.0, window=0):
    """Outputs and bounds; cache: (k, v, k_scale, v_scale), all on the CPU."""
    k8, v8, k_scale, v_scale = cache
    u = UNIT[q.dtype]
    Hq, D = q.shape[1:]
    G = Hq // k_scale.shape[1]
    out = torch.zeros(q.shape, dtype=torch.float64)
    bound = torch.zeros(q.shape, dtype=torch.float64)
    for t in range(len(lengths)):
        n, length = offsets[t + 1] - offsets[t], lengths[t]
        if n <= 0:
            continue
        ids = table[t, :(length + PAGE - 1) // PAGE].long()
        good = (ids >= 0) & (ids < len(k8))
        ids = ids.clamp(0, max(len(k8) - 1, 0))
        seen0 = good.repeat_interleave(PAGE)[:length]
        j = torch.arange(length)[None]
        i = torch.arange(length - n, length)[:, None]
        seen = (j <= i) & seen0[None]
        if window:
            seen &= j > i - window
        for h in range(Hq):
            K = (k8[ids, h // G].double() * k_scale[ids, h // G].double()[:, None, None]).reshape(-1, D)[:length]
            V = (in_order(v8[ids, h // G]).double() * v_scale[ids, h // G].double()[:, None, None]).reshape(-1, D)[:length]
            K[~seen0], V[~seen0] = 0, 0
            Q = q[offsets[t]:offsets[t + 1], h].double()
            s = scale * (Q @ K.T)
            # A query's dimension is a whole number of 1 / 32512 of its row's largest: off by half of that (2^-16 / 1.98),
            # a score by the sum of those times the keys.  Then steps in 32 bits.
            ds = scale * (E32 * (8 + D ** 0.5) * (Q.abs() @ K.abs().T) + Q.abs().amax(1, keepdim=True) / 65024 * K.abs().sum(1))
            if cap:
                s = cap * torch.tanh(s / cap)
                ds = ds + 4e-7 * (s.abs() if cap > 64 else torch.full_like(s, cap))
            ds = ds + 4 * E32 * s.abs()     # in units of log 2, and the shift's difference
            s = torch.where(seen, s, -math.inf)
            some = seen.any(1, keepdim=True) if length else torch.zeros(n, 1, dtype=torch.bool)
            if not length:
                continue
            m = torch.where(some, s.amax(1, keepdim=True), 0.0)
            p = torch.exp(s - m)
            total = torch.where(some, p.sum(1, keepdim=True), 1.0)
            o = (p @ V) / total
            shift = torch.where(seen, ds, 0.0).amax(1, keepdim=True)
            size = (p @ V.abs()) / total
            # weights: their scores, 32-bit steps, 2^-11 in float16 and below its normal range 2^-25 of the largest value
            b = (2.0 ** -11 + 2 * shift + 64 * E32) * size + 2.0 ** -25 * 2 * seen.sum(1, keepdim=True) / total * V.abs().amax()
            rows = slice(offsets[t], offsets[t + 1])
            out[rows, h] = o
            bound[rows, h] = u * (o.abs() + b) + b + TINY[q.dtype] + 1e-30
    return out, bound
