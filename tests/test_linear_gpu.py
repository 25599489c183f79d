"""linear_rows_i8 against whole numbers in 64 bits: sizes around the kernels'
tiles, odd widths, rows that begin anywhere, sums near the end of 32 bits,
scales that are not finite, and the range of gelu."""

import math

import pytest
import torch

import paper_2512_07009_amd as flock
from tests.encoder_reference import TINY, UNIT

pytestmark = pytest.mark.gpu

E32 = 2.0 ** -24


def case(seed, rows, width, outputs, bias=True, full=False):
    gen = torch.Generator().manual_seed(seed)

    def whole(n):
        if full:
            return torch.randint(-128, 128, (n, width), generator=gen, dtype=torch.int8)
        return (40 * torch.randn(n, width, generator=gen)).round().clamp(-127, 127).to(torch.int8)

    return dict(x=whole(rows), w=whole(outputs), xs=0.01 + 0.02 * torch.rand(rows, generator=gen),
                ws=(0.5 + torch.rand(outputs, generator=gen)) / (40 * width ** 0.5),
                bias=torch.randn(outputs, generator=gen) if bias else None)


def padded(t, pitch):
    """t on the device, its rows `pitch` bytes apart, with other values between them."""
    room = torch.full((t.shape[0], pitch), 77, dtype=torch.int8, device="cuda")
    room[:, :t.shape[1]] = t.cuda()
    return room[:, :t.shape[1]]


def compare(c, dtype, gelu=False, x=None, w=None):
    d = {n: (t.cuda() if t is not None else None) for n, t in c.items()}
    got = flock.linear_rows_i8(d["x"] if x is None else x, d["xs"], d["w"] if w is None else w, d["ws"], d["bias"],
                               gelu=gelu, dtype=dtype)
    torch.cuda.synchronize()
    s = d["x"].double() @ d["w"].double().t()          # exact: below 2^53
    y = s * d["xs"].double()[:, None] * d["ws"].double()
    size = y.abs()
    if d["bias"] is not None:
        y = y + d["bias"].double()
        size = size + y.abs()
    # the sum's rounding to 32 bits, two products and a sum
    bound = 4 * E32 * size
    if gelu:
        # 1.13: the largest derivative of t Phi(t).  Its fit is off by 6.5e-6 in 32 bits; in 16 by 3.2e-5 (five terms), and
        # by the 14 steps of 32 bits around it, of which the tail takes that of t^2 / 2 up to 40 times: 3.7e-5, below 4e-5
        value = y * 0.5 * torch.special.erfc(-y / math.sqrt(2))
        y, bound = value, 1.13 * bound + (1e-5 if dtype == torch.float32 else 4e-5) * value.abs()
    bound = bound + (UNIT[dtype] * (1 + 2 * E32)) * (y.abs() + bound) + TINY[dtype] + 1e-30
    err = (got.double() - y).abs()
    assert got.shape == y.shape and got.dtype == dtype
    assert (err <= bound).all(), f"off by up to {err.max():.3e}, {(err > bound).sum()} of {err.numel()} above their bound"
    return got


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 32, 33, 63, 64, 65, 127, 129, 500])
@pytest.mark.parametrize("outputs", [1, 16, 63, 64, 130, 501])
def test_rows_and_outputs(rows, outputs):
    compare(case(rows * outputs, rows, 96, outputs), torch.bfloat16)


@pytest.mark.parametrize("rows", [5, 40, 200])
@pytest.mark.parametrize("width", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 100, 127, 128, 129, 144, 255, 256, 257, 272, 512,
                                   1000, 2047, 2048, 2049])
def test_widths(width, rows):
    compare(case(width, rows, width, 70), torch.float16)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,outputs", [(9, 48), (100, 100), (9000, 600), (4097, 1030)])
def test_types(rows, outputs, dtype):
    compare(case(3, rows, 160, outputs, bias=False), dtype)
    compare(case(4, rows, 160, outputs), dtype, gelu=True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("width", [40, 128, 130, 256, 384, 500, 1000])
def test_tiles_of_128_by_workgroups_that_stay(width, dtype):
    """785 tiles, the last of each side cut, over 512 workgroups: steps of one to eight a tile."""
    c = case(width, 20001, width, 601)
    pitch = (width + 15) // 16 * 16
    compare(c, dtype, x=padded(c["x"], pitch), w=padded(c["w"], pitch))
    if width in (40, 500):
        compare(c, dtype, gelu=True, x=padded(c["x"], pitch + 16), w=padded(c["w"], pitch))


def test_whole_tiles_of_128():
    compare(case(1, 128 * 160, 256, 128 * 8), torch.bfloat16)


@pytest.mark.parametrize("rows", [3, 50, 8500])
@pytest.mark.parametrize("pitch_x,pitch_w", [(208, 208), (201, 208), (208, 217), (203, 203), (600, 224)])
def test_rows_that_begin_anywhere(rows, pitch_x, pitch_w):
    c = case(5, rows, 200, 520)
    whole = compare(c, torch.bfloat16)
    assert torch.equal(whole, compare(c, torch.bfloat16, x=padded(c["x"], pitch_x), w=padded(c["w"], pitch_w)))
    x = padded(torch.nn.functional.pad(c["x"], (3, 0)), pitch_x + 5)[:, 3:]
    assert torch.equal(whole, compare(c, torch.bfloat16, x=x))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,width,outputs", [(33, 129, 64), (70, 1, 130), (1000, 127, 513), (4001, 2047, 200)])
def test_rows_side_by_side_of_odd_widths(rows, width, outputs, dtype):
    """Contiguous rows that begin anywhere: within their bounds, and the same to the bit every time."""
    c = case(21, rows, width, outputs)
    for gelu in (False, True):
        first = compare(c, dtype, gelu=gelu)
        for _ in range(10):
            assert torch.equal(first, compare(c, dtype, gelu=gelu))


def test_one_row_for_all():
    c = case(6, 70, 128, 66)
    c["x"] = c["x"][:1].expand(70, 128)
    compare(c, torch.float32, x=c["x"][:1].cuda().expand(70, 128))


def test_out_with_rows_apart():
    c = case(7, 300, 128, 90)
    want = compare(c, torch.bfloat16)
    room = torch.full((300, 101), 7.0, dtype=torch.bfloat16, device="cuda")
    d = {n: t.cuda() for n, t in c.items()}
    flock.linear_rows_i8(d["x"], d["xs"], d["w"], d["ws"], d["bias"], out=room[:, 3:93])
    assert torch.equal(room[:, 3:93], want) and (room[:, :3] == 7).all() and (room[:, 93:] == 7).all()


@pytest.mark.parametrize("rows", [4, 40])
def test_sums_near_the_end_of_32_bits(rows):
    width = 2 ** 17 - 1
    c = case(8, rows, width, 20, bias=False)
    c["x"][0], c["w"][0], c["w"][1] = -128, -128, 127
    c["x"][1] = 127
    compare(c, torch.float32)
    compare(case(9, rows, 5000, 40, full=True), torch.float32)


def test_scales_that_are_not_finite():
    c = case(10, 40, 64, 40, bias=False)
    c["xs"][3], c["ws"][5] = math.nan, math.inf
    d = {n: t.cuda() if t is not None else None for n, t in c.items()}
    y = flock.linear_rows_i8(d["x"], d["xs"], d["w"], d["ws"])
    assert torch.isnan(y[3]).all() and not torch.isfinite(y[:, 5]).any()
    rest = torch.ones(40, 40, dtype=torch.bool)
    rest[3], rest[:, 5] = False, False
    assert torch.isfinite(y.cpu()[rest]).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_gelu_over_its_range_in_16_bits(dtype):
    """The same values of t to types of 16 bits, by the kernel for few rows and by the one for many."""
    x = torch.arange(-127, 128, dtype=torch.int8)[:, None].cuda()
    w = torch.ones(40, 1, dtype=torch.int8, device="cuda")
    ws = torch.linspace(0.0005, 0.1, 40, device="cuda")
    t = x.double() * ws.double()
    want = t * 0.5 * torch.special.erfc(-t / math.sqrt(2))
    bound = want.abs() * (4e-5 + E32 * (2 + t * t))
    bound = bound + UNIT[dtype] * (want.abs() + bound) + TINY[dtype] + 1e-37
    for rows in (x, *x.split(16)):
        y = flock.linear_rows_i8(rows, torch.ones(len(rows), device="cuda"), w, ws, gelu=True, dtype=dtype)
        at = slice(None) if len(rows) == 255 else slice(int(rows[0]) + 127, int(rows[-1]) + 128)
        assert ((y.double() - want[at]).abs() <= bound[at]).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows", [2, 20, 200])
def test_gelu_of_what_is_not_finite(rows, dtype):
    """Sums that leave the range of 32 bits: infinity stays, its negative is nothing, NaN stays."""
    x = torch.full((rows, 32), 100, dtype=torch.int8, device="cuda")
    w = torch.full((3, 32), 100, dtype=torch.int8, device="cuda")
    w[1] = -100
    ws = torch.tensor([3e38, 3e38, math.nan], device="cuda")
    y = flock.linear_rows_i8(x, torch.ones(rows, device="cuda"), w, ws, gelu=True, dtype=dtype)
    assert (y[:, 0] == math.inf).all() and (y[:, 1] == 0).all() and y[:, 2].isnan().all()


@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("rows,width,outputs,dtype", [
    (7936, 768, 2048, torch.bfloat16),   # whole tiles, one each
    (7901, 300, 2016, torch.float16),    # rows, outputs and a width that end inside a tile, a step and a chunk
    (16301, 256, 2016, torch.bfloat16),  # two tiles each, of two steps
    (24000, 1001, 2048, torch.float16),  # three, of eight
    (29001, 577, 480, torch.bfloat16),
    (30001, 1100, 501, torch.float16),   # outputs that begin anywhere
    (16000, 1025, 1999, torch.bfloat16),
])
def test_tiles_of_256(rows, width, outputs, dtype, gelu):
    c = case(19, rows, width, outputs)
    compare(c, dtype, gelu=gelu, x=padded(c["x"], (width + 15) // 16 * 16), w=padded(c["w"], (width + 15) // 16 * 16))


@pytest.mark.parametrize("before,after", [(32, 64), (33, 64), (32, 1)])
def test_tiles_of_256_leave_what_is_beside_them(before, after):
    """Outputs in rows of a wider tensor, and the tensor's other elements as they were."""
    c = case(20, 7700, 1040, 1952)
    wide = torch.full((7702, before + 1952 + after), 7.0, dtype=torch.bfloat16, device="cuda")
    out = wide[1:-1, before:-after]
    d = {n: (t.cuda() if t is not None else None) for n, t in c.items()}
    flock.linear_rows_i8(d["x"], d["xs"], d["w"], d["ws"], d["bias"], out=out)
    want = flock.linear_rows_i8(d["x"], d["xs"], d["w"], d["ws"], d["bias"], dtype=torch.float32).bfloat16()
    assert torch.equal(out, want)
    out.fill_(7.0)
    assert (wide == 7.0).all()


@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("rows,width,outputs,dtype", [
    (6144, 512, 8192, torch.bfloat16),       # whole turns of whole tiles
    (6400 + 31, 272, 7520, torch.float16),   # outputs and rows that end inside a tile, a width inside a chunk pair
    (12400, 509, 3584 + 512, torch.bfloat16),
    (49152 + 1, 257, 992, torch.bfloat16),
])
def test_weights_that_stay(rows, width, outputs, dtype, gelu):
    c = case(17, rows, width, outputs)
    compare(c, dtype, gelu=gelu, x=padded(c["x"], (width + 15) // 16 * 16), w=padded(c["w"], (width + 15) // 16 * 16))


def test_weights_that_stay_leave_what_is_beside_them():
    """Outputs in rows of a wider tensor, and the tensor's other elements as they were."""
    c = case(18, 6200, 320, 7552)
    wide = torch.full((6202, 7552 + 96), 7.0, dtype=torch.bfloat16, device="cuda")
    out = wide[1:-1, 32:-64]
    d = {n: (t.cuda() if t is not None else None) for n, t in c.items()}
    flock.linear_rows_i8(d["x"], d["xs"], d["w"], d["ws"], d["bias"], out=out)
    want = flock.linear_rows_i8(d["x"], d["xs"], d["w"], d["ws"], d["bias"], dtype=torch.float32).bfloat16()
    assert torch.equal(out, want)
    wide[1:-1, 32:-64] = 7.0
    assert (wide == 7.0).all()


def test_gelu_over_its_range():
    """One product of width 1 for each of 8-bit values: t from -13 to 13."""
    x = torch.arange(-127, 128, dtype=torch.int8)[:, None].cuda()
    w = torch.ones(40, 1, dtype=torch.int8, device="cuda")
    ws = torch.linspace(0.0005, 0.1, 40, device="cuda")
    y = flock.linear_rows_i8(x, torch.ones(255, device="cuda"), w, ws, gelu=True, dtype=torch.float32)
    t = x.double() * ws.double()
    want = t * 0.5 * torch.special.erfc(-t / math.sqrt(2))
    # 32-bit steps before it: t is off by 2^-24 of itself, which the tail's e^(-t^2 / 2) takes t^2 times
    bound = want.abs() * (1e-5 + E32 * (2 + t * t)) + 1e-37
    assert ((y.double() - want).abs() <= bound).all()


def test_empty_and_refusals():
    c = case(11, 4, 32, 8)
    d = {n: t.cuda() for n, t in c.items()}
    x, xs, w, ws = d["x"], d["xs"], d["w"], d["ws"]
    assert flock.linear_rows_i8(x[:0], xs[:0], w, ws).shape == (0, 8)
    with pytest.raises(ValueError, match="int8"):
        flock.linear_rows_i8(x.float(), xs, w, ws)
    with pytest.raises(ValueError, match="weight"):
        flock.linear_rows_i8(x, xs, w[:, :16], ws)
    with pytest.raises(ValueError, match="x_scale"):
        flock.linear_rows_i8(x, xs[:3], w, ws)
    with pytest.raises(ValueError, match="weight_scale"):
        flock.linear_rows_i8(x, xs, w, ws.double())
    with pytest.raises(ValueError, match="bias"):
        flock.linear_rows_i8(x, xs, w, ws, torch.zeros(9, device="cuda"))
    with pytest.raises(ValueError, match="outputs of"):
        flock.linear_rows_i8(x, xs, w, ws, dtype=torch.float64)
    with pytest.raises(ValueError, match="out must"):
        flock.linear_rows_i8(x, xs, w, ws, out=torch.empty(4, 9, device="cuda"))
    with pytest.raises(ValueError, match="contiguous rows"):
        flock.linear_rows_i8(x.t(), xs, w, ws)
