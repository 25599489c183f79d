"""The per-bird encoder's operators in 64 bits, straight from their
definitions (CPU), with bounds on what rounding may cost a correct kernel.

u is the rounding of the features' type (half an ulp of 1: 2^-8 bfloat16, 2^-11
float16, 2^-24 float32).  Where a kernel rounds a factor of a
product to the features' type, each of its terms may be off by u of itself;
float16 factors below the normal range by 2^-25.  32-bit steps in between are
allowed SLACK of the terms they produce.
"""

import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}
SLACK = 1e-4    # weights: scores of up to some hundred in 32 bits


def attention(q, k, v, q_off, k_off, scale, cap=0.0, q_xy=None, k_xy=None, slopes=None, keep=None, causal=False,
              prefix=None, grad=None):
    """Outputs and bounds; tensors on the CPU, offsets as lists."""
    dtype = q.dtype
    u, tiny = UNIT[dtype], TINY[dtype]
    Hq, Hk, D = q.shape[1], k.shape[1], q.shape[2]
    G = Hq // Hk
    names = ["out", "lse"] + (["dq", "dk", "dv", "ds"] if grad is not None else [])
    shapes = {"out": q.shape, "lse": (q.shape[0], Hq), "dq": q.shape, "dk": k.shape, "dv": v.shape, "ds": (Hq,)}
    r = {n: torch.zeros(shapes[n], dtype=torch.float64) for n in names}
    b = {n: torch.zeros(shapes[n], dtype=torch.float64) for n in names}
    r["lse"].fill_(-math.inf)
    for f in range(len(q_off) - 1):
        qs, ks = slice(q_off[f], q_off[f + 1]), slice(k_off[f], k_off[f + 1])
        nq, nk = qs.stop - qs.start, ks.stop - ks.start
        seen = torch.ones(nq, nk, dtype=torch.bool)
        if keep is not None:
            seen &= (keep[ks] != 0)[None, :]
        if causal:
            i, j = torch.arange(nq)[:, None], torch.arange(nk)[None, :]
            order = j <= i + nk - nq
            if prefix is not None:
                order = order | (j < prefix[f])
            seen &= order
        for h in range(Hq):
            Q, K, V = q[qs, h].double(), k[ks, h // G].double(), v[ks, h // G].double()
            # hidden keys are not read
            gone = ~seen.any(0)
            K = torch.where(gone[:, None], 0.0, K)
            V = torch.where(gone[:, None], 0.0, V)
            t = scale * (Q @ K.T)
            th = torch.zeros_like(t)
            if cap:
                th = torch.tanh(t / cap)
                t = cap * th
            s = t
            d2 = torch.zeros_like(t)
            if slopes is not None:
                d = (q_xy[qs].double()[:, None] - k_xy[ks].double()[None]) / 16
                d2 = (d * d).sum(-1)
                s = t - slopes[h].double() * d2
            s = torch.where(seen, s, -math.inf)
            lse = torch.logsumexp(s, 1) if nk else torch.full((nq,), -math.inf, dtype=torch.float64)
            P = torch.where(seen, torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[:, None]), 0.0)
            o = P @ V
            r["out"][qs, h] = o
            r["lse"][qs, h] = lse
            # a weight's rounding is relative to its size before the division by the sum, at most 1
            b["out"][qs, h] = (u + SLACK) * (P @ V.abs()) + tiny * V.abs().sum(0) + u * o.abs() + 1e-7
            b["lse"][qs, h] = 2e-5 * (1 + torch.where(lse == -math.inf, 0.0, lse).abs())
            if grad is None:
                continue
            g = grad[qs, h].double()
            dP = g @ V.T
            delta = (g * o).sum(1, keepdim=True)
            dS = P * (dP - delta)
            r["dv"][ks, h // G] += P.T @ g
            b["dv"][ks, h // G] += (u + SLACK) * (P.T @ g.abs()) + tiny * g.abs().sum(0) + 1e-7
            r["ds"][h] -= (dS * d2).sum()
            b["ds"][h] += SLACK * ((P * dP.abs() * d2).sum() + (delta[:, 0].abs() * (P * d2).sum(1)).sum()) + 1e-6
            dT = dS * (1 - th * th) if cap else dS
            # delta comes from the rounded output
            off = (u + SLACK) * dT.abs() + (u + SLACK) * P * (g.abs() * (P @ V.abs() + o.abs())).sum(1, keepdim=True) + tiny
            off = torch.where(seen, off, 0.0)
            off += SLACK * P * dP.abs()
            r["dq"][qs, h] = scale * (dT @ K)
            b["dq"][qs, h] = scale * (off @ K.abs()) + 1e-7
            r["dk"][ks, h // G] += scale * (dT.T @ Q)
            b["dk"][ks, h // G] += scale * (off.T @ Q.abs()) + 1e-7
    for n in ("dq", "dk", "dv"):
        if n in b:
            b[n] += u * r[n].abs()
    return r, b


def layer_norm(x, weight, bias, eps, residual=None, grad_y=None, grad_sum=None):
    dtype = x.dtype
    u = UNIT[dtype]
    h = x.double()
    r, b = {}, {}
    if residual is not None:
        h = (x.float() + residual.float()).to(dtype).double()
        r["h"], b["h"] = h, torch.zeros_like(h)
    n = x.shape[1]
    mean = h.mean(1, keepdim=True)
    c = h - mean
    rstd = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + eps)
    xh = c * rstd
    w = torch.ones(n, dtype=torch.float64) if weight is None else weight.double()
    y = xh * w + (0.0 if bias is None else bias.double())
    # 32-bit sums of a row: the mean is off by 2^-24 log2(n) of the mean size
    e32 = 2.0 ** -24 * (8 + math.log2(n + 1) * 4)
    row = h.abs().mean(1, keepdim=True) * rstd
    r["mean"], b["mean"] = mean[:, 0], e32 * (h.abs().mean(1) + 1e-30)
    r["rstd"], b["rstd"] = rstd[:, 0], e32 * rstd[:, 0] * (1 + (row * row)[:, 0] * 2.0 ** -20)
    xoff = e32 * (xh.abs() + row + h.abs() * rstd)
    r["y"], b["y"] = y, u * y.abs() + xoff * w.abs() + e32 * y.abs() + 1e-30
    if grad_y is None:
        return r, b
    g0 = grad_y.double()
    g = g0 * w
    m1, m2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    dx = rstd * (g - m1 - xh * m2)
    off = e32 * (g.abs() + g.abs().mean(1, keepdim=True) + xh.abs() * (g * xh).abs().mean(1, keepdim=True)) \
        + xoff * (g.abs() * xh.abs()).mean(1, keepdim=True) + xh.abs() * (g.abs() * xoff).mean(1, keepdim=True)
    off = off * rstd
    if grad_sum is not None:
        dx = dx + grad_sum.double()
        off = off + e32 * grad_sum.double().abs()
    r["dx"], b["dx"] = dx, u * dx.abs() + off + 1e-30
    many = 2.0 ** -24 * (8 + x.shape[0] ** 0.5)
    r["dw"], b["dw"] = (g0 * xh).sum(0), (many * (g0 * xh).abs() + g0.abs() * xoff).sum(0) + 1e-30
    r["db"], b["db"] = g0.sum(0), many * g0.abs().sum(0) + 1e-30
    return r, b


def rotary(z, xy, time, freq, counts, interleaved, inverse):
    nt, ny, nx = counts
    P = nt + ny + nx
    w = z.double().clone()
    big = torch.zeros_like(w)
    for p in range(P):
        pos = time.double() if p < nt else (xy[:, 1] if p < nt + ny else xy[:, 0]).double() / 16
        ang = (pos * freq[p] * (-1 if inverse else 1))[:, None]
        i, j = (2 * p, 2 * p + 1) if interleaved else (p, p + P)
        a, b = z[:, :, i].double(), z[:, :, j].double()
        w[:, :, i] = a * torch.cos(ang) - b * torch.sin(ang)
        w[:, :, j] = a * torch.sin(ang) + b * torch.cos(ang)
        big[:, :, i] = big[:, :, j] = a.abs() + b.abs()
    # the reference's own angle is rounded to 2^-53 of itself, the kernel's sine is off by 2^-23
    return w, UNIT[z.dtype] * w.abs() + 4 * 2.0 ** -23 * big + 1e-30


def check(got, want, bound, name):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (name, got.shape, want.shape)
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), f"{name}: infinities differ"
    err = (got - want)[~inf].abs()
    assert torch.isfinite(err).all(), f"{name}: not finite"
    over = err - bound.expand(want.shape)[~inf]
    assert err.numel() == 0 or over.max() <= 0, \
        f"{name}: off by up to {err.max():.3e}, {(over > 0).sum()} of {err.numel()} values above their bound"
