"""A per-bird encoder on ragged frames, trained with torch's autograd.

The library's layer norm, rotary positions and attention as differentiable
functions, and a block that puts them together:

    block = EncoderBlock(width=256, q_heads=4, axes=RotaryAxes(y=..., x=...)).to("cuda")
    h = block(features, offsets, xy)         # [T, width] bfloat16, a row per bird

Linear layers are plain matrix products of torch.  The functions have first
derivatives only: differentiating their gradients raises.
"""

from __future__ import annotations

import functools

import torch

from .binding import (RotaryAxes, attention_frames, attention_frames_backward, layer_norm_rows,
                      layer_norm_rows_backward, rotary_frames)


class _Final(torch.autograd.Function):
    """Gradients as they are, whose own gradients raise."""

    @staticmethod
    def forward(ctx, *values):
        return values

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("the encoder's operators have no second derivatives")


def _once(backward):
    """A backward pass by kernels that autograd does not see: under create_graph
    its results must not pass for constants."""
    @functools.wraps(backward)
    def run(ctx, *grads):
        with torch.no_grad():
            result = backward(ctx, *grads)
        if not torch.is_grad_enabled():
            return result
        return _Final.apply(*(r.detach().requires_grad_() if torch.is_tensor(r) else r for r in result))
    return run


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, bias, eps):
        y, h, mean, rstd = layer_norm_rows(x, weight, bias, eps, residual=residual)
        ctx.save_for_backward(h, weight, mean, rstd)
        ctx.summed = residual is not None
        return (y, h) if ctx.summed else y

    @staticmethod
    @_once
    def backward(ctx, grad_y, grad_h=None):
        h, weight, mean, rstd = ctx.saved_tensors
        dx, dw, db = layer_norm_rows_backward(grad_y.contiguous(), h, weight, mean, rstd,
                                              grad_sum=grad_h.contiguous() if grad_h is not None else None)
        needs = ctx.needs_input_grad
        return dx, dx if ctx.summed else None, dw if needs[2] else None, db if needs[3] else None, None


def layer_norm(x, weight, bias, eps=1e-5, residual=None):
    """Layer norm of the rows of x, or of x + residual: y, or (y, the sum).
    weight and bias may be None (1 and 0)."""
    return _LayerNorm.apply(x, residual, weight, bias, eps)


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, xy, time, axes):
        # (saved as tensors: autograd then refuses a backward pass on places that were overwritten)
        ctx.save_for_backward(xy, time)
        ctx.axes = axes
        return rotary_frames(q, k, xy, axes, time=time)

    @staticmethod
    @_once
    def backward(ctx, grad_q, grad_k):
        xy, time = ctx.saved_tensors
        grads = (g.contiguous() if g is not None else None for g in (grad_q, grad_k))
        return *rotary_frames(*grads, xy, ctx.axes, time=time, inverse=True), None, None, None


def rotary(q, k, xy, axes: RotaryAxes, time=None):
    """Queries and keys (either may be None) turned by their birds' time, y and x."""
    return _Rotary.apply(q, k, xy, time, axes)


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, slopes, offsets, more):
        out, lse = attention_frames(q, k, v, offsets, slopes=slopes, return_lse=True, **more)
        # places and masks too are saved as tensors, so that one that was overwritten is refused
        ctx.names = [name for name, value in more.items() if torch.is_tensor(value)]
        ctx.more = {name: value for name, value in more.items() if name not in ctx.names}
        ctx.save_for_backward(q, k, v, slopes, offsets, out, lse, *(more[name] for name in ctx.names))
        return out

    @staticmethod
    @_once
    def backward(ctx, grad_out):
        q, k, v, slopes, offsets, out, lse, *saved = ctx.saved_tensors
        grad_out = grad_out.contiguous()
        if grad_out.data_ptr() % 16:  # a part of another gradient
            grad_out = grad_out.clone()
        dq, dk, dv, ds = attention_frames_backward(grad_out, q, k, v, out, lse, offsets, slopes=slopes,
                                                   **ctx.more, **dict(zip(ctx.names, saved)))
        return dq, dk, dv, ds, None, None


def attention(q, k, v, offsets, slopes=None, **more):
    """attention_frames with gradients of q, k, v and slopes; `more` holds its
    other arguments (k_offsets, q_xy, k_xy, scale, cap, keep, causal, prefix)."""
    return _Attention.apply(q, k, v, slopes, offsets, more)


class EncoderBlock(torch.nn.Module):
    """Attention among the birds of a frame, then a layer per bird, each on the
    layer norm of what came before and added to it."""

    def __init__(self, width: int, q_heads: int, axes: RotaryAxes, kv_heads: int | None = None,
                 head_dim: int = 64, sigma_px=(30.0, 960.0), cap: float = 0.0, hidden: int | None = None,
                 dtype=torch.bfloat16):
        super().__init__()
        if dtype not in (torch.float16, torch.bfloat16):
            raise ValueError(f"features of {dtype}: attention takes float16 or bfloat16")
        kv_heads = q_heads if kv_heads is None else kv_heads
        hidden = 4 * width if hidden is None else hidden
        self.heads = (q_heads, kv_heads, head_dim)
        self.axes, self.cap = axes, cap

        def linear(rows, columns):
            return torch.nn.Parameter((torch.randn(rows, columns) * columns ** -0.5).to(dtype))

        self.qkv = linear((q_heads + 2 * kv_heads) * head_dim, width)
        self.out = linear(width, q_heads * head_dim)
        self.up, self.down = linear(hidden, width), linear(width, hidden)
        self.norm_weight = torch.nn.Parameter(torch.ones(2, width))
        self.norm_bias = torch.nn.Parameter(torch.zeros(2, width))
        # heads that look from sigma_px[0] to sigma_px[1] around a bird, learned from there
        low, high = sigma_px
        sigma = low * (high / low) ** (torch.arange(q_heads) / max(q_heads - 1, 1))
        self.log_slopes = torch.nn.Parameter(torch.log(0.5 / sigma ** 2))

    def forward(self, x, offsets, xy, time=None, keep=None):
        hq, hk, dim = self.heads
        # the norms and the slopes are in 32 bits, whatever type the block was moved to
        weight, bias, slopes = self.norm_weight.float(), self.norm_bias.float(), self.log_slopes.float().exp()
        y = layer_norm(x, weight[0], bias[0])
        qkv = (y @ self.qkv.t()).view(-1, hq + 2 * hk, dim)
        q, k = rotary(qkv[:, :hq], qkv[:, hq:hq + hk], xy, self.axes, time)
        a = attention(q, k, qkv[:, hq + hk:], offsets, slopes, q_xy=xy, cap=self.cap, keep=keep)
        y, x = layer_norm(a.flatten(1) @ self.out.t(), weight[1], bias[1], residual=x)
        return x + torch.nn.functional.gelu(y @ self.up.t()) @ self.down.t()
