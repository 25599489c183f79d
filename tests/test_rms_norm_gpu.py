"""rms_norm_rows, its backward pass, its output in 8 bits and quantize_rows
against 64 bits: widths around the kernels' shapes, odd and wide rows, strides,
residuals, rows of zeros, tiny and huge rows, values that are not finite."""

import pytest
import torch

import paper_2512_07009_amd as flock
from tests import serving_reference as ref

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.float16, torch.bfloat16]
WIDTHS = [1, 2, 7, 8, 16, 31, 64, 65, 128, 200, 256, 333, 512, 768, 1000, 1024, 2048, 2500]


def case(seed, rows, width, dtype, residual=False, train=True, affine=True):
    gen = torch.Generator().manual_seed(seed)
    rnd = lambda: torch.randn(rows, width, generator=gen).to(dtype)  # noqa: E731
    c = dict(x=rnd() + 0.25, weight=None, residual=None, grad_y=None, grad_sum=None)
    if affine:
        c["weight"] = 1 + 0.3 * torch.randn(width, generator=gen)
    if residual:
        c["residual"] = rnd()
    if train:
        c["grad_y"] = rnd()
        if residual:
            c["grad_sum"] = rnd()
    return c


def compare(c, eps=1e-6):
    d = {n: (t.cuda() if t is not None else None) for n, t in c.items()}
    y, h, rstd = flock.rms_norm_rows(d["x"], d["weight"], eps, residual=d["residual"])
    got = {"y": y, "rstd": rstd}
    if c["residual"] is not None:
        got["h"] = h
    if c["grad_y"] is not None:
        got["dx"], got["dw"] = flock.rms_norm_rows_backward(d["grad_y"], h, d["weight"], rstd, grad_sum=d["grad_sum"])
    q, scale, h8 = flock.rms_norm_rows_i8(d["x"], d["weight"], eps, residual=d["residual"])
    torch.cuda.synchronize()
    want, bound = ref.rms_norm(c["x"], c["weight"], eps, c["residual"], c["grad_y"], c["grad_sum"])
    for n in want:
        if n != "y32":
            ref.check(got[n], want[n], bound[n], n)
    assert torch.equal(h8, h)
    ref.check_whole(q, scale, want["y32"], bound["y32"])
    return dict(got, q=q, scale=scale)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("width", WIDTHS)
def test_widths(width, dtype):
    compare(case(width, 13, width, dtype, residual=width % 2 == 0))


@pytest.mark.parametrize("width", [4096, 4104, 5001, 8192, 8200, 20000])
def test_wide_rows(width):
    compare(case(width, 5, width, torch.bfloat16, residual=True))
    compare(case(width, 70, width, torch.float32))


@pytest.mark.parametrize("rows", [1, 2, 3, 5, 127, 4099])
@pytest.mark.parametrize("width", [24, 64, 520])
def test_rows(rows, width):
    compare(case(rows, rows, width, torch.bfloat16))


def test_without_weight():
    compare(case(1, 40, 96, torch.float16, affine=False, residual=True))


def test_strides_in_place_and_out():
    c = case(4, 50, 61, torch.bfloat16, train=False)
    wide = torch.zeros(50, 200, dtype=torch.bfloat16, device="cuda")
    x = wide[:, 3:64]
    x.copy_(c["x"])
    w = c["weight"].cuda()
    want, bound = ref.rms_norm(c["x"], c["weight"], 1e-6)
    ref.check(flock.rms_norm_rows(x, w)[0], want["y"], bound["y"], "y")
    room = torch.full((50, 70), 99, dtype=torch.int8, device="cuda")
    scale = torch.empty(50, device="cuda")
    flock.rms_norm_rows_i8(x, w, out=(room[:, 5:66], scale, None))
    ref.check_whole(room[:, 5:66], scale, want["y32"], bound["y32"])
    assert (room[:, :5] == 99).all() and (room[:, 66:] == 99).all()
    # one row for all
    y = flock.rms_norm_rows(c["x"][:1].cuda().expand(9, 61))[0]
    assert (y == y[:1]).all()
    # in place
    c = case(5, 33, 512, torch.bfloat16, residual=True, train=False)
    x, r, w = (c[n].cuda() for n in ("x", "residual", "weight"))
    y, h, rstd = flock.rms_norm_rows(x, w, residual=r)
    flock.rms_norm_rows(x, w, residual=r, out=(x, r, torch.empty_like(rstd)))
    assert torch.equal(x, y) and torch.equal(r, h)


def test_repeats_bit_for_bit():
    c = case(6, 5000, 320, torch.bfloat16, residual=True)
    a, b = compare(c), compare(c)
    for n in a:
        assert torch.equal(a[n], b[n]), n


def test_gradients_against_differences():
    c = case(7, 7, 40, torch.float32, residual=True)
    got = compare(c)
    gen = torch.Generator().manual_seed(3)
    gy, gs = c["grad_y"].double(), c["grad_sum"].double()

    def loss(h, w):
        return (h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6) * w * gy).sum() + (h * gs).sum()

    args = [(c["x"] + c["residual"]).double(), c["weight"].double()]
    eps = 1e-5
    for i, name in enumerate(("dx", "dw")):
        step = torch.randn(args[i].shape, generator=gen, dtype=torch.float64)
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + eps * step, args[i] - eps * step
        diff = (loss(*up) - loss(*down)) / (2 * eps)
        mine = (got[name].cpu().double() * step).sum()
        assert (mine - diff).abs() <= 1e-4 * (1 + diff.abs()), name


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("width", [1, 16, 37, 512, 1000, 9000])
def test_quantize_rows(width, dtype):
    gen = torch.Generator().manual_seed(width)
    x = torch.randn(21, width, generator=gen).to(dtype)
    q, scale = flock.quantize_rows(x.cuda())
    y = x.double()
    ref.check_whole(q, scale, y, torch.zeros_like(y))


@pytest.mark.parametrize("width", [24, 600, 9000])
def test_quantize_rows_that_have_no_scale(width):
    x = torch.randn(8, width, generator=torch.Generator().manual_seed(1)).cuda()
    x[0] = 0
    x[1] = 1e-33
    x[2, width // 2] = float("nan")
    x[3, width - 1] = float("inf")
    x[4, 0] = -float("inf")
    x[5] = 3.0e38
    x[6] = -127.0
    q, scale = flock.quantize_rows(x)
    assert (q[:5] == 0).all() and (scale[:2] == 0).all() and torch.isnan(scale[2:5]).all()
    assert (q[5] == 127).all() and (q[6] == -127).all() and scale[6] == 1.0
    assert torch.isfinite(scale[5:]).all()
    # ties go to even whole numbers
    x = torch.zeros(1, width, device="cuda")
    x[0, :8] = torch.tensor([127.0, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 126.5])
    q, scale = flock.quantize_rows(x)
    assert q[0, :8].tolist() == [127, 0, 2, 2, 0, -2, -2, 126] and (q[0, 8:] == 0).all()


def test_rows_of_zeros():
    x = torch.zeros(5, 200, dtype=torch.bfloat16, device="cuda")
    y, h, rstd = flock.rms_norm_rows(x, eps=1e-6)
    q, scale, _ = flock.rms_norm_rows_i8(x, eps=1e-6)
    assert (y == 0).all() and (q == 0).all() and (scale == 0).all()
    dx, dw = flock.rms_norm_rows_backward(torch.ones_like(x), h, None, rstd)
    assert torch.isfinite(dx).all() and (dw == 0).all()


def test_another_stream():
    c = case(9, 3000, 512, torch.bfloat16, residual=True, train=False)
    x, r, w = (c[n].cuda() for n in ("x", "residual", "weight"))
    here = flock.rms_norm_rows_i8(x, w, residual=r)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    there = flock.rms_norm_rows_i8(x, w, residual=r, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(here, there):
        assert torch.equal(a, b)


def test_empty_and_refusals():
    x = torch.empty(0, 16, device="cuda")
    y, h, rstd = flock.rms_norm_rows(x)
    dx, dw = flock.rms_norm_rows_backward(y, x, None, rstd)
    assert y.shape == (0, 16) and (dw == 0).all()
    q, scale = flock.quantize_rows(x)
    assert q.shape == (0, 16) and scale.shape == (0,)
    x = torch.zeros(4, 16, device="cuda")
    for fn in (flock.rms_norm_rows, flock.rms_norm_rows_i8, flock.quantize_rows):
        with pytest.raises(ValueError, match="contiguous rows"):
            fn(x.t())
        with pytest.raises(ValueError, match="float64"):
            fn(x.double())
    for fn in (flock.rms_norm_rows, flock.rms_norm_rows_i8):
        with pytest.raises(ValueError, match="eps"):
            fn(x, eps=-1.0)
        with pytest.raises(ValueError, match="weight"):
            fn(x, weight=torch.ones(15, device="cuda"))
        with pytest.raises(ValueError, match="residual"):
            fn(x, residual=x.half())
    with pytest.raises(ValueError, match="int8"):
        flock.quantize_rows(x, out=(torch.empty(4, 16, dtype=torch.uint8, device="cuda"), torch.empty(4, device="cuda")))
    with pytest.raises(ValueError, match="scale"):
        flock.quantize_rows(x, out=(torch.empty(4, 16, dtype=torch.int8, device="cuda"), torch.empty(5, device="cuda")))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("width", [8, 100, 512, 2500, 9000])
def test_whole_numbers_are_the_rounded_quotients(width, dtype):
    """To the bit what a division in 32 bits rounds to, numbers at half a step among them (half a row's largest is 63.5)."""
    gen = torch.Generator().manual_seed(width)
    x = torch.randn(400, width, generator=gen).to(dtype)
    most = x.abs().amax(1)
    x[:, 0], x[:, 1], x[:, 2] = most, most / 2, -most / 2
    q, scale = flock.quantize_rows(x.cuda())
    q, scale = q.cpu(), scale.cpu()
    assert torch.equal(scale, most.float() / 127)
    assert torch.equal(q.float(), torch.round(x.float() / scale[:, None]))
