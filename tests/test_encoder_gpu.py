"""The per-bird encoder's differentiable functions and its example."""

import os
import sys

import pytest
import torch

import paper_2512_07009_amd as flock
from paper_2512_07009_amd import RotaryAxes, encoder

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_block_gradients_follow_the_loss():
    """A small step against the gradient lowers the loss by the gradient's
    square, to first order (bfloat16 features: within a quarter)."""
    torch.manual_seed(1)
    n = 300
    off = torch.tensor([0, 100, 100, 180, 300], dtype=torch.int32, device="cuda")
    xy = torch.randint(0, 16 * 300, (n, 2), dtype=torch.int32, device="cuda")
    block = encoder.EncoderBlock(64, q_heads=4, kv_heads=2, head_dim=32, axes=RotaryAxes(y=[0.1] * 8, x=[0.05] * 8),
                                 cap=20.0).cuda()
    x = torch.randn(n, 64, device="cuda").to(torch.bfloat16)
    goal = torch.randn(n, 64, device="cuda")

    def loss():
        return ((block(x, off, xy).float() - goal) ** 2).mean()

    first = loss()
    first.backward()
    moved = [block.norm_weight, block.norm_bias, block.log_slopes]
    square = sum((p.grad ** 2).sum() for p in moved)
    assert square > 0 and all(torch.isfinite(p.grad).all() for p in block.parameters())
    step = 0.02 * first.item() / square.item()
    with torch.no_grad():
        for p in moved:
            p -= step * p.grad
    drop = (first - loss()).item()
    assert 0.75 * step * square.item() <= drop <= 1.25 * step * square.item()


def test_frames_do_not_see_each_other():
    torch.manual_seed(2)
    off = torch.tensor([0, 70, 200], dtype=torch.int32, device="cuda")
    xy = torch.randint(0, 16 * 300, (200, 2), dtype=torch.int32, device="cuda")
    block = encoder.EncoderBlock(64, q_heads=2, head_dim=32, axes=RotaryAxes(y=[0.1] * 8, x=[0.05] * 8)).cuda()
    x = torch.randn(200, 64, device="cuda").to(torch.bfloat16)
    with torch.no_grad():
        a = block(x, off, xy)
        x[70:] = 0
        xy[70:] = 0
        b = block(x, off, xy)
    assert torch.equal(a[:70], b[:70])


@pytest.mark.parametrize("weight,bias", [(False, False), (True, False), (False, True)])
def test_layer_norm_without_weight_or_bias(weight, bias):
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(20, 48, generator=gen).cuda().requires_grad_()
    w = torch.rand(48, generator=gen).cuda().requires_grad_() if weight else None
    b = torch.rand(48, generator=gen).cuda().requires_grad_() if bias else None
    g = torch.randn(20, 48, generator=gen).cuda()
    encoder.layer_norm(x, w, b).backward(g)
    leaves = [t for t in (x, w, b) if t is not None]
    same = [t.detach().cpu().double().requires_grad_() for t in leaves]
    rest = same[1:]
    x64, w64, b64 = same[0], rest.pop(0) if weight else torch.ones(48).double(), rest.pop(0) if bias else 0.0
    centred = x64 - x64.mean(1, keepdim=True)
    y = centred / (centred.pow(2).mean(1, keepdim=True) + 1e-5).sqrt() * w64 + b64
    y.backward(g.cpu().double())
    for got, want in zip(leaves, same):
        # 32-bit arithmetic over sums of 48 and 20: well below 2^-17 of the norm
        assert (got.grad.cpu().double() - want.grad).norm() <= 2 ** -17 * want.grad.norm()


@pytest.mark.parametrize("which", [0, 1])
def test_rotary_of_queries_or_keys_alone(which):
    x = torch.randn(9, 2, 8, device="cuda", requires_grad=True)
    xy = torch.randint(0, 4000, (9, 2), dtype=torch.int32, device="cuda")
    pair = [None, None]
    pair[which] = x
    turned = encoder.rotary(*pair, xy, RotaryAxes(y=[0.1, 0.2], x=[0.3, 0.4]))
    assert turned[1 - which] is None
    g = torch.randn(9, 2, 8, device="cuda")
    turned[which].backward(g)
    # a turn keeps products (32 bits): <turn x, g> = <x, turned back g>
    assert torch.allclose((turned[which].double() * g).sum((1, 2)), (x.double() * x.grad).sum((1, 2)), rtol=0, atol=1e-4)


@pytest.mark.parametrize("off", [[0], [0, 0, 0]])
def test_block_without_birds(off):
    block = encoder.EncoderBlock(64, q_heads=2, head_dim=32, axes=RotaryAxes(y=[0.1] * 8, x=[0.05] * 8)).cuda()
    x = torch.zeros(0, 64, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    y = block(x, torch.tensor(off, dtype=torch.int32, device="cuda"), torch.zeros(0, 2, dtype=torch.int32, device="cuda"))
    y.sum().backward()
    assert y.shape == (0, 64)
    assert all((p.grad == 0).all() for p in block.parameters())


def test_example_learns():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import bird_encoder
    losses, right = bird_encoder.main(steps=40, frames=4, height=240, width=320, n_birds=150, quiet=True)
    assert torch.isfinite(losses).all()
    assert losses[-5:].mean() < 0.7 * losses[:5].mean()


@pytest.mark.parametrize("name", ["q_xy", "k_xy", "k_offsets", "keep", "prefix", "offsets", "slopes", "v"])
def test_overwritten_inputs_of_attention_are_refused(name):
    """Gradients of other places or masks than the forward pass had are wrong."""
    n = 40
    q = torch.randn(n, 2, 32, device="cuda").to(torch.bfloat16).requires_grad_()
    v = torch.randn(n, 2, 32, device="cuda").to(torch.bfloat16)
    offsets = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    slopes = torch.ones(2, device="cuda")
    more = dict(q_xy=torch.zeros(n, 2, dtype=torch.int32, device="cuda"),
                k_xy=torch.zeros(n, 2, dtype=torch.int32, device="cuda"), k_offsets=offsets.clone(),
                keep=torch.ones(n, dtype=torch.uint8, device="cuda"),
                prefix=torch.zeros(1, dtype=torch.int32, device="cuda"), causal=True)
    out = encoder.attention(q, q, v, offsets, slopes, **more)
    dict(more, offsets=offsets, slopes=slopes, v=v)[name].add_(0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()


@pytest.mark.parametrize("name", ["xy", "time"])
def test_overwritten_places_of_rotary_are_refused(name):
    q = torch.randn(9, 2, 8, device="cuda", requires_grad=True)
    places = dict(xy=torch.zeros(9, 2, dtype=torch.int32, device="cuda"),
                  time=torch.zeros(9, dtype=torch.int32, device="cuda"))
    turned, _ = encoder.rotary(q, None, places["xy"], RotaryAxes(time=[0.1], y=[0.1]), time=places["time"])
    places[name].add_(0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        turned.sum().backward()


@pytest.mark.parametrize("steady", [False, True])
@pytest.mark.parametrize("name", ["norm", "norm of a sum", "rotary", "attention"])
def test_second_derivatives_are_refused(name, steady):
    """Also where the first derivative's own input (steady) needs no gradient,
    and where another path leads to the loss."""
    x = torch.randn(24, 2, 32, device="cuda").to(torch.bfloat16).requires_grad_()
    xy = torch.randint(0, 4000, (24, 2), dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 24], dtype=torch.int32, device="cuda")

    def apply():
        if name == "norm":
            return encoder.layer_norm(x.flatten(1), None, None)
        if name == "norm of a sum":
            return encoder.layer_norm(x.flatten(1), None, None, residual=x.flatten(1))[0]
        if name == "rotary":
            return encoder.rotary(x, x, xy, RotaryAxes(x=[0.1]))[1]
        return encoder.attention(x, x, x, off)

    y = apply().float()
    first, = torch.autograd.grad((y if steady else y * y).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="no second derivatives"):
        (first.float().pow(2).sum() + x.float().pow(2).sum()).backward()
    # create_graph alone changes no first derivative
    y = apply().float()
    plain, = torch.autograd.grad((y if steady else y * y).sum(), x)
    assert torch.equal(plain, first)


def test_gradient_that_is_a_part_of_another():
    """The output's gradient may begin at any element of a larger one."""
    x = torch.randn(10, 2, 32, device="cuda").to(torch.bfloat16)
    off = torch.tensor([0, 10], dtype=torch.int32, device="cuda")
    weights = torch.randn(641, device="cuda").to(torch.bfloat16)
    grads = []
    for first in (torch.zeros(1, device="cuda").to(torch.bfloat16), None):
        q = x.clone().requires_grad_()
        out = encoder.attention(q, q, q, off).flatten()
        (torch.cat([first, out]) @ weights if first is not None else out @ weights[1:]).backward()
        grads.append(q.grad)
    assert torch.equal(*grads)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_block_moved_to_a_16_bit_type(dtype):
    """Its norms and slopes are used in 32 bits, and are trained as they are held."""
    torch.manual_seed(4)
    block = encoder.EncoderBlock(64, q_heads=2, head_dim=32, axes=RotaryAxes(y=[0.1] * 8, x=[0.05] * 8)).cuda().to(dtype)
    x = torch.randn(50, 64, device="cuda").to(dtype)
    xy = torch.randint(0, 16 * 300, (50, 2), dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 50], dtype=torch.int32, device="cuda")
    y = block(x, off, xy)
    y.float().pow(2).sum().backward()
    assert y.dtype == dtype and torch.isfinite(y).all()
    assert all(p.grad.dtype == dtype and torch.isfinite(p.grad).all() for p in block.parameters())
    # the same values held in 32 bits give the same block
    for p in (block.norm_weight, block.norm_bias, block.log_slopes):
        p.data = p.data.float()
    assert torch.equal(block(x, off, xy), y)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float64])
def test_block_refuses_types_that_attention_does_not_take(dtype):
    with pytest.raises(ValueError, match="float16 or bfloat16"):
        encoder.EncoderBlock(64, q_heads=2, axes=RotaryAxes(x=[0.1]), dtype=dtype)


@pytest.mark.parametrize("name", ["norm", "norm backward", "rotary", "attention", "attention backward", "density"])
def test_outputs_on_another_stream_are_not_memory_in_use(name):
    """A call on a stream of its own must not write into what the current stream
    freed and is still working on."""
    n = 300
    off = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    xy = torch.randint(0, 16 * 1000, (n, 2), dtype=torch.int32, device="cuda")
    x = torch.randn(n, 8, 64, device="cuda").to(torch.bfloat16)
    _, h, mean, rstd = flock.layer_norm_rows(x.flatten(1))
    out, lse = flock.attention_frames(x, x, x, off, return_lse=True)
    call = {"norm": lambda s: flock.layer_norm_rows(x.flatten(1), stream=s)[0],
            "norm backward": lambda s: flock.layer_norm_rows_backward(x.flatten(1), h, None, mean, rstd, stream=s)[0],
            "rotary": lambda s: flock.rotary_frames(x, None, xy, RotaryAxes(x=[0.1]), stream=s)[0],
            "attention": lambda s: flock.attention_frames(x, x, x, off, stream=s),
            "attention backward": lambda s: flock.attention_frames_backward(x, x, x, x, out, lse, off, stream=s)[0],
            "density": lambda s: flock.density_frames(xy, off, 1920, 1080, 128, 72, 40.0, stream=s)}[name]
    want = call(None)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    freed = [torch.empty_like(want) for _ in range(4)]
    torch.cuda._sleep(100_000_000)  # some 50 ms
    for t in freed:
        t.fill_(7)
    del freed, t
    got = call(stream)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
