"""layer_norm_rows, its backward pass and rotary_frames against the 64-bit
reference: widths around the kernels' shapes, odd and wide rows, strides,
residuals, constant rows, large means; far positions; in place."""

import math

import pytest
import torch

import paper_2512_07009_amd as flock
from tests import encoder_reference as ref

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.float16, torch.bfloat16]


def norm_case(seed, rows, width, dtype, residual=False, train=True, affine=True, shift=0.5):
    gen = torch.Generator().manual_seed(seed)
    rnd = lambda: torch.randn(rows, width, generator=gen).to(dtype)  # noqa: E731
    c = dict(x=rnd() + shift, weight=None, bias=None, residual=None, grad_y=None, grad_sum=None)
    if affine:
        c["weight"], c["bias"] = 1 + 0.3 * torch.randn(width, generator=gen), torch.randn(width, generator=gen)
    if residual:
        c["residual"] = rnd()
    if train:
        c["grad_y"] = rnd()
        if residual:
            c["grad_sum"] = rnd()
    return c


def norm_compare(c, eps=1e-5):
    d = {n: (t.cuda() if t is not None else None) for n, t in c.items()}
    y, h, mean, rstd = flock.layer_norm_rows(d["x"], d["weight"], d["bias"], eps, residual=d["residual"])
    got = {"y": y, "mean": mean, "rstd": rstd}
    if c["residual"] is not None:
        got["h"] = h
    if c["grad_y"] is not None:
        got["dx"], got["dw"], got["db"] = flock.layer_norm_rows_backward(d["grad_y"], h, d["weight"], mean, rstd,
                                                                         grad_sum=d["grad_sum"])
    torch.cuda.synchronize()
    want, bound = ref.layer_norm(c["x"], c["weight"], c["bias"], eps, c["residual"], c["grad_y"], c["grad_sum"])
    for n in want:
        ref.check(got[n], want[n], bound[n], n)
    return got


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("width", [1, 2, 7, 8, 16, 31, 64, 65, 128, 200, 256, 333, 512, 768, 1000, 1024, 2048, 2500])
def test_norm_widths(width, dtype):
    norm_compare(norm_case(width, 13, width, dtype, residual=width % 2 == 0))


@pytest.mark.parametrize("width", [4096, 4104, 5001, 8192, 8200, 20000])
def test_norm_wide_rows(width):
    norm_compare(norm_case(width, 5, width, torch.bfloat16, residual=True))
    norm_compare(norm_case(width, 70, width, torch.float32))


@pytest.mark.parametrize("rows", [1, 2, 3, 5, 127, 4099])
@pytest.mark.parametrize("width", [24, 64, 520])
def test_norm_rows(rows, width):
    norm_compare(norm_case(rows, rows, width, torch.bfloat16))


def test_norm_without_weights():
    norm_compare(norm_case(1, 40, 96, torch.float16, affine=False))


def test_norm_rows_of_one_value_and_a_large_mean():
    c = norm_case(2, 6, 512, torch.float32, train=False)
    c["x"][2] = 3.0
    c["x"][3] = 0.0
    c["x"] = c["x"] + 0.0
    got = norm_compare(c)
    assert torch.isfinite(got["y"]).all()
    c = norm_case(3, 6, 512, torch.float32, train=True, shift=1000.0)
    norm_compare(c)


def test_norm_strides():
    c = norm_case(4, 50, 64, torch.bfloat16)
    for width in (64, 61):
        wide = torch.zeros(50, 200, dtype=torch.bfloat16, device="cuda")
        x = wide[:, 3:3 + width] if width == 61 else wide[:, 8:8 + width]
        x.copy_(c["x"][:, :width])
        w, b = c["weight"][:width].cuda(), c["bias"][:width].cuda()
        a = flock.layer_norm_rows(x, w, b)
        e = flock.layer_norm_rows(x.contiguous(), w, b)
        want, bound = ref.layer_norm(x.cpu(), w.cpu(), b.cpu(), 1e-5)
        ref.check(a[0], want["y"], bound["y"], "y")
        ref.check(e[0], want["y"], bound["y"], "y")
    # one row for all (stride 0)
    y = flock.layer_norm_rows(c["x"][:1].cuda().expand(9, 64))[0]
    assert (y == y[:1]).all()


def test_norm_in_place_and_out():
    c = norm_case(5, 33, 512, torch.bfloat16, residual=True, train=False)
    x, r, w, b = (c[n].cuda() for n in ("x", "residual", "weight", "bias"))
    y, h, mean, rstd = flock.layer_norm_rows(x, w, b, residual=r)
    x2, r2 = x.clone(), r.clone()
    flock.layer_norm_rows(x2, w, b, residual=r2, out=(x2, r2, torch.empty_like(mean), torch.empty_like(rstd)))
    assert torch.equal(x2, y) and torch.equal(r2, h)


def test_norm_repeats_bit_for_bit():
    c = norm_case(6, 5000, 320, torch.bfloat16, residual=True)
    a, b = norm_compare(c), norm_compare(c)
    for n in a:
        assert torch.equal(a[n], b[n]), n


def test_norm_gradients_against_differences():
    c = norm_case(7, 7, 40, torch.float32, residual=True)
    got = norm_compare(c)
    gen = torch.Generator().manual_seed(3)
    gy, gs = c["grad_y"].double(), c["grad_sum"].double()
    eps = 1e-5

    def loss(h, w, b):
        mean = h.mean(1, keepdim=True)
        z = (h - mean) / torch.sqrt(((h - mean) ** 2).mean(1, keepdim=True) + 1e-5) * w + b
        return (z * gy).sum() + (h * gs).sum()

    h0 = (c["x"] + c["residual"]).double()
    args = [h0, c["weight"].double(), c["bias"].double()]
    for i, name in enumerate(("dx", "dw", "db")):
        step = torch.randn(args[i].shape, generator=gen, dtype=torch.float64)
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + eps * step, args[i] - eps * step
        diff = (loss(*up) - loss(*down)) / (2 * eps)
        mine = (got[name].cpu().double() * step).sum()
        assert (mine - diff).abs() <= 1e-4 * (1 + diff.abs()), name


def test_norm_empty_and_refusals():
    x = torch.empty(0, 16, device="cuda")
    y, h, mean, rstd = flock.layer_norm_rows(x)
    dx, dw, db = flock.layer_norm_rows_backward(y, x, None, mean, rstd)
    assert y.shape == (0, 16) and (dw == 0).all() and (db == 0).all()
    x = torch.zeros(4, 16, device="cuda")
    with pytest.raises(ValueError, match="contiguous rows"):
        flock.layer_norm_rows(x.t())
    with pytest.raises(ValueError, match="eps"):
        flock.layer_norm_rows(x, eps=-1.0)
    with pytest.raises(ValueError, match="weight"):
        flock.layer_norm_rows(x, weight=torch.ones(15, device="cuda"))
    with pytest.raises(ValueError, match="residual"):
        flock.layer_norm_rows(x, residual=x.half())
    with pytest.raises(ValueError, match="float64"):
        flock.layer_norm_rows(x.double())


# --- rotary ---

def turn(seed, n, Hq, Hk, D, counts, dtype, interleaved=False, inverse=False, fused=False, far=0, in_place=False):
    gen = torch.Generator().manual_seed(seed)
    nt, ny, nx = counts
    z = torch.randn(n, Hq + 2 * Hk, D, generator=gen).to(dtype)
    xy = (torch.rand(n, 2, generator=gen) * 16 * 1000).int() + far
    time = torch.randint(-1000, 100000, (n,), generator=gen).int()
    freq = [2 * math.pi / w for w in torch.logspace(0.6, 4, max(nt + ny + nx, 1)).tolist()][:nt + ny + nx]
    if nx:
        freq[-1] = -freq[-1]
    axes = flock.RotaryAxes(freq[:nt], freq[nt:nt + ny], freq[nt + ny:])
    dz = z.cuda()
    q, k = dz[:, :Hq], dz[:, Hq:Hq + Hk]
    if not fused:
        q, k = q.contiguous(), k.contiguous()
    want_q = ref.rotary(z[:, :Hq], xy, time, freq, counts, interleaved, inverse)
    want_k = ref.rotary(z[:, Hq:Hq + Hk], xy, time, freq, counts, interleaved, inverse)
    gq, gk = flock.rotary_frames(q if Hq else None, k if Hk else None, xy.cuda(), axes, time=time.cuda(),
                                 interleaved=interleaved, inverse=inverse, out=(q, k) if in_place else None)
    torch.cuda.synchronize()
    if Hq:
        ref.check(gq, *want_q, "q")
    if Hk:
        ref.check(gk, *want_k, "k")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("counts", [(8, 12, 12), (0, 16, 16), (32, 0, 0), (0, 0, 5), (3, 4, 6), (4, 8, 4)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_axes(counts, dtype, interleaved):
    turn(1, 37, 3, 1, 64, counts, dtype, interleaved=interleaved)


@pytest.mark.parametrize("dim,counts", [(2, (0, 0, 1)), (3, (0, 1, 0)), (7, (1, 1, 1)), (40, (4, 8, 8)), (96, (16, 16, 16)),
                                        (128, (0, 32, 32)), (256, (40, 40, 48)), (256, (0, 1, 0))])
def test_rotary_widths(dim, counts):
    turn(dim, 50, 2, 2, dim, counts, torch.bfloat16)
    turn(dim, 3, 5, 0, dim, counts, torch.float32, inverse=True)
    turn(dim, 3, 0, 7, dim, counts, torch.float16, interleaved=True)


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 1000])
def test_rotary_birds(n):
    turn(n, n, 8, 8, 64, (8, 12, 12), torch.bfloat16, fused=True)
    turn(n, n, 1, 1, 32, (0, 8, 8), torch.float16)


def test_rotary_far_positions():
    """Phases of positions up to 2^24 (and late times) have no rounding error."""
    turn(2, 200, 2, 2, 64, (8, 12, 12), torch.float32, far=(1 << 24) - 16 * 1000 - 1)


def test_rotary_in_place():
    turn(3, 100, 4, 2, 64, (0, 12, 12), torch.bfloat16, in_place=True)
    turn(3, 100, 4, 2, 64, (0, 12, 12), torch.bfloat16, in_place=True, fused=True)


def test_rotary_many_heads():
    turn(4, 5, 256, 256, 16, (0, 4, 4), torch.bfloat16)


def test_rotary_back_is_the_gradient():
    """<turn(q), g> = <q, turn_back(g)>, and turning back undoes the turn."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    q = torch.randn(64, 2, 64, generator=gen, device="cuda")
    g = torch.randn(64, 2, 64, generator=gen, device="cuda")
    xy = torch.randint(0, 30000, (64, 2), generator=gen, device="cuda", dtype=torch.int32)
    axes = flock.RotaryAxes(y=[0.2] * 10, x=[0.01] * 10)
    t, _ = flock.rotary_frames(q, None, xy, axes)
    back, _ = flock.rotary_frames(g, None, xy, axes, inverse=True)
    a, b = (t.double() * g.double()).sum(), (q.double() * back.double()).sum()
    assert abs(a - b) <= 1e-5 * (q.double().abs() * g.double().abs()).sum()
    assert (flock.rotary_frames(t, None, xy, axes, inverse=True)[0] - q).abs().max() <= 4e-6


def test_rotary_refusals():
    q = torch.zeros(4, 2, 8, device="cuda")
    xy = torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="fit head_dim"):
        flock.rotary_frames(q, None, xy, flock.RotaryAxes(x=[1.0] * 5))
    with pytest.raises(ValueError, match="time"):
        flock.rotary_frames(q, None, xy, flock.RotaryAxes(time=[1.0]))
    with pytest.raises(ValueError, match="xy"):
        flock.rotary_frames(q, None, xy[:3], flock.RotaryAxes(x=[1.0]))
    with pytest.raises(ValueError, match="finite"):
        flock.rotary_frames(q, None, xy, flock.RotaryAxes(x=[math.inf]))
    with pytest.raises(ValueError, match="q or k"):
        flock.rotary_frames(None, None, xy, flock.RotaryAxes(x=[1.0]))
    assert flock.rotary_frames(q[:0], None, xy[:0], flock.RotaryAxes(x=[1.0]))[0].shape == (0, 2, 8)


def ends(n, at):
    """Rows at the beginning, the end, and round a place between."""
    return [slice(0, 100), slice(at - 100, at + 100), slice(n - 100, n)]


def test_norm_of_more_rows_than_a_launch_holds():
    """2^24 - 1 workgroups, of 32 narrow rows each."""
    most = ((1 << 24) - 1) * 32
    n = most + 1000
    x = torch.empty(n, 4, dtype=torch.bfloat16, device="cuda")
    for i in range(0, n, 1 << 26):
        x[i:i + (1 << 26)].normal_()
    w = torch.rand(4, device="cuda")
    y, _, mean, rstd = flock.layer_norm_rows(x, w)
    for rows in ends(n, most):
        want = flock.layer_norm_rows(x[rows], w)
        assert torch.equal(y[rows], want[0]) and torch.equal(mean[rows], want[2]) and torch.equal(rstd[rows], want[3])


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_of_more_birds_than_a_launch_holds(interleaved):
    """2^24 - 1 workgroups, of 64 birds each."""
    most = ((1 << 24) - 1) * 64
    n = most + 1000
    q = torch.empty(n, 1, 2, dtype=torch.bfloat16, device="cuda")
    for i in range(0, n, 1 << 26):
        q[i:i + (1 << 26)].normal_()
    time = torch.arange(n, dtype=torch.int32, device="cuda")
    axes = flock.RotaryAxes(time=[0.1])
    want = [flock.rotary_frames(q[r], None, None, axes, time=time[r], interleaved=interleaved)[0] for r in ends(n, most)]
    flock.rotary_frames(q, None, None, axes, time=time, interleaved=interleaved, out=(q, None))
    for r, w in zip(ends(n, most), want):
        assert torch.equal(q[r], w)


def test_sizes_beyond_32_bits_are_refused():
    """Not cut to what is left modulo 2^32."""
    wide = torch.zeros(1, 8, dtype=torch.bfloat16, device="cuda").expand(2 ** 31 + 5, 8)
    with pytest.raises(ValueError, match="2\\^31"):
        flock.layer_norm_rows(wide)
    birds = wide[:, None]
    one = torch.zeros(1, dtype=torch.int32, device="cuda").expand(2 ** 31 + 5)
    with pytest.raises(ValueError, match="2\\^31"):
        flock.rotary_frames(birds, None, None, flock.RotaryAxes(time=[1.0]), time=one)
    off = torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="2\\^31"):
        flock.attention_frames(birds, birds, birds, off)
