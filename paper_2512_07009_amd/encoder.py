"""A per-bird encoder on ragged frames, trained with torch's autograd.

The library's layer norm, rotary positions and attention as differentiable
functions, and a block that puts them together:

    block = EncoderBlock(width=256, q_heads=4, axes=RotaryAxes(y=..., x=...)).to("cuda")
    h = block(features, offsets, xy)         # [T, width] bfloat16, a row per bird

Linear layers are plain matrix products of torch.  The functions have first
derivatives only: differentiating their gradients raises.

A block that was trained on tracks (norm="rms", sigma_px=None, causal) is served on the
live stream in 8 bits, its keys and values kept in pages of a cache:

    served = ServedBlock(block)
    cache = served.cache(pages=4096)
    h = served(features, cache, offsets, table, lengths, xy, time)
"""

from __future__ import annotations

import functools

import torch

from .binding import (RotaryAxes, TrackCache, append_tracks, attention_frames, attention_frames_backward,
                      attention_tracks, layer_norm_rows, layer_norm_rows_backward, linear_rows_i8, quantize_rows,
                      rms_norm_rows, rms_norm_rows_backward, rms_norm_rows_i8, rotary_frames)


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


class _RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, eps):
        y, h, rstd = rms_norm_rows(x, weight, eps, residual=residual)
        ctx.save_for_backward(h, weight, rstd)
        ctx.summed = residual is not None
        return (y, h) if ctx.summed else y

    @staticmethod
    @_once
    def backward(ctx, grad_y, grad_h=None):
        h, weight, rstd = ctx.saved_tensors
        dx, dw = rms_norm_rows_backward(grad_y.contiguous(), h, weight, rstd,
                                        grad_sum=grad_h.contiguous() if grad_h is not None else None)
        return dx, dx if ctx.summed else None, dw if ctx.needs_input_grad[2] else None, None


def rms_norm(x, weight, eps=1e-6, residual=None):
    """Root-mean-square norm of the rows of x, or of x + residual: y, or (y, the
    sum).  weight may be None (1)."""
    return _RmsNorm.apply(x, residual, weight, eps)


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
    """Attention among the birds of a frame (or the detections of a track), then a
    layer per bird, each on the norm of what came before and added to it.

    norm: "layer" or "rms".  sigma_px: the heads' first Gaussian weights of distances
    (None: distances take no part)."""

    def __init__(self, width: int, q_heads: int, axes: RotaryAxes, kv_heads: int | None = None,
                 head_dim: int = 64, sigma_px=(30.0, 960.0), cap: float = 0.0, hidden: int | None = None,
                 dtype=torch.bfloat16, norm: str = "layer"):
        super().__init__()
        if dtype not in (torch.float16, torch.bfloat16):
            raise ValueError(f"features of {dtype}: attention takes float16 or bfloat16")
        if norm not in ("layer", "rms"):
            raise ValueError(f"norm {norm!r}: expected 'layer' or 'rms'")
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
        self.norm_bias = torch.nn.Parameter(torch.zeros(2, width)) if norm == "layer" else None
        if sigma_px is None:
            self.log_slopes = None
            return
        # heads that look from sigma_px[0] to sigma_px[1] around a bird, learned from there
        low, high = sigma_px
        sigma = low * (high / low) ** (torch.arange(q_heads) / max(q_heads - 1, 1))
        self.log_slopes = torch.nn.Parameter(torch.log(0.5 / sigma ** 2))

    def _norm(self, i, x, residual=None):
        # the norms are in 32 bits, whatever type the block was moved to
        weight = self.norm_weight.float()[i]
        if self.norm_bias is None:
            return rms_norm(x, weight, residual=residual)
        return layer_norm(x, weight, self.norm_bias.float()[i], residual=residual)

    def forward(self, x, offsets, xy, time=None, keep=None, causal=False):
        hq, hk, dim = self.heads
        slopes = self.log_slopes.float().exp() if self.log_slopes is not None else None
        y = self._norm(0, x)
        qkv = (y @ self.qkv.t()).view(-1, hq + 2 * hk, dim)
        q, k = rotary(qkv[:, :hq], qkv[:, hq:hq + hk], xy, self.axes, time)
        a = attention(q, k, qkv[:, hq + hk:], offsets, slopes, q_xy=xy if slopes is not None else None, cap=self.cap,
                      keep=keep, causal=causal)
        y, x = self._norm(1, a.flatten(1) @ self.out.t(), residual=x)
        return x + torch.nn.functional.gelu(y @ self.up.t()) @ self.down.t()


class ServedBlock:
    """A trained EncoderBlock (norm="rms", sigma_px=None) on tracks as they go on: its
    products in 8 bits, a scale for each row and each output, and the keys and values of
    every detection in a cache in 8 bits.

    A call takes the newest detections of each track and returns what the block gives for
    them (causal, over the whole track), to what 8 bits hold.  Weights are laid out when
    the ServedBlock is made: make another after more training."""

    def __init__(self, block: EncoderBlock):
        if block.norm_bias is not None:
            raise ValueError("a block with layer norm: expected norm='rms'")
        if block.log_slopes is not None:
            raise ValueError("a block with distances: expected sigma_px=None")
        if not block.qkv.is_cuda or block.qkv.dtype not in (torch.float16, torch.bfloat16):
            raise ValueError("expected a block on the GPU in float16 or bfloat16")
        if block.heads[2] % 16:
            raise ValueError(f"heads of {block.heads[2]}: a cache takes multiples of 16")
        self.heads, self.axes, self.cap, self.dtype = block.heads, block.axes, block.cap, block.qkv.dtype
        with torch.no_grad():
            self.norms = block.norm_weight.float().clone().unbind()
            self.qkv, self.out, self.up, self.down = (quantize_rows(w.detach()) for w in (block.qkv, block.out, block.up,
                                                                                         block.down))

    def cache(self, pages: int) -> TrackCache:
        """A pool of pages for this block's keys and values."""
        return TrackCache.empty(pages, self.heads[1], self.heads[2], self.qkv[0].device)

    @torch.no_grad()
    def __call__(self, x, cache: TrackCache, offsets, table, lengths, xy, time=None, window: int = 0):
        """x [T, width], the rows of each track by offsets (int32 [tracks + 1]), which
        become its last tokens; table and lengths as for append_tracks.  Rows that belong
        to no track, or to one that is passed over, are of no meaning in what is returned."""
        hq, hk, dim = self.heads
        if x.dtype != self.dtype:
            raise ValueError(f"features of {x.dtype}: the block is in {self.dtype}")
        y, scale, _ = rms_norm_rows_i8(x, self.norms[0])
        qkv = linear_rows_i8(y, scale, *self.qkv, dtype=x.dtype).view(-1, hq + 2 * hk, dim)
        q, _ = rotary_frames(qkv[:, :hq], None, xy, self.axes, time=time)
        append_tracks(cache, qkv[:, hq:hq + hk], qkv[:, hq + hk:], offsets, table, lengths, axes=self.axes, xy=xy, time=time)
        a = attention_tracks(q, cache, offsets, table, lengths, cap=self.cap, window=window)
        a = linear_rows_i8(*quantize_rows(a.flatten(1)), *self.out, dtype=x.dtype)
        y, scale, x = rms_norm_rows_i8(a, self.norms[1], residual=x)
        y = linear_rows_i8(y, scale, *self.up, gelu=True, dtype=x.dtype)
        return x + linear_rows_i8(*quantize_rows(y), *self.down, dtype=x.dtype)
