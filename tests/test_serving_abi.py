"""The served encoder's entry points reject bad arguments on the host before
touching any device, and empty calls are no-ops (no GPU needed)."""

import ctypes
import math

import pytest

from paper_2512_07009_amd import binding

FAKE = ctypes.c_void_p(0x100000)       # never dereferenced on these paths
FAKE2 = ctypes.c_void_p(0x100002)
FAKE4 = ctypes.c_void_p(0x100004)
FAKE8 = ctypes.c_void_p(0x100008)
F32, F16, BF16 = 0, 1, 2


def refused(status, needle, want=binding.FLOCK_EINVAL):
    assert status == want
    assert needle in binding.lib().flock_last_error().decode()


def norm(dtype=BF16, x=FAKE, xs=64, r=None, rs=0, rows=4, width=64, w=FAKE, eps=1e-5, y=FAKE, ys=64, s=None, ss=0, rstd=FAKE):
    return binding.lib().rms_norm_rows(dtype, x, xs, r, rs, rows, width, w, eps, y, ys, s, ss, rstd, None)


def norm_i8(dtype=BF16, x=FAKE, xs=64, r=None, rs=0, rows=4, width=64, w=FAKE, eps=1e-5, y=FAKE, ys=64, scale=FAKE, s=None,
            ss=0):
    return binding.lib().rms_norm_rows_i8(dtype, x, xs, r, rs, rows, width, w, eps, y, ys, scale, s, ss, None)


NORM = [
    (dict(dtype=3), "dtype"), (dict(rows=-1), "rows"), (dict(width=0), "width"), (dict(width=(1 << 20) + 1), "width"),
    (dict(eps=-1.0), "eps"), (dict(eps=math.nan), "eps"), (dict(xs=-1), "strides"), (dict(ys=63), "hold a row"),
    (dict(x=None), "non-NULL"), (dict(y=None), "non-NULL"), (dict(r=FAKE, rs=64, ss=64), "sum"),
    (dict(r=FAKE, rs=64, s=FAKE, ss=1), "hold a row"), (dict(r=FAKE, rs=-1, s=FAKE, ss=64), "strides"),
    (dict(dtype=F32, x=FAKE2), "aligned"), (dict(w=FAKE2), "aligned"),
]


@pytest.mark.parametrize("kwargs,needle", NORM + [(dict(rstd=FAKE2), "aligned"), (dict(dtype=F32, y=FAKE2), "aligned")])
def test_rms_norm_rejects(kwargs, needle):
    refused(norm(**kwargs), needle)


@pytest.mark.parametrize("kwargs,needle", NORM + [(dict(scale=None), "scale"), (dict(scale=FAKE2), "aligned")])
def test_rms_norm_i8_rejects(kwargs, needle):
    refused(norm_i8(**kwargs), needle)


def norm_back(dtype=BF16, gy=FAKE, gys=64, gs=None, gss=0, x=FAKE, xs=64, rows=4, width=64, w=FAKE, rstd=FAKE, dx=FAKE,
              dxs=64, dw=FAKE, ws=None, n=0):
    return binding.lib().rms_norm_rows_backward(dtype, gy, gys, gs, gss, x, xs, rows, width, w, rstd, dx, dxs, dw, ws, n, None)


@pytest.mark.parametrize("kwargs,needle", [
    (dict(dtype=9), "dtype"), (dict(rows=-2), "rows"), (dict(width=-1), "width"), (dict(gys=-1), "strides"),
    (dict(gs=FAKE, gss=-8), "strides"), (dict(dxs=8), "hold a row"), (dict(gy=None), "non-NULL"),
    (dict(rstd=None), "non-NULL"), (dict(dx=None), "non-NULL"), (dict(dw=FAKE2), "aligned"), (dict(dtype=F32, x=FAKE2), "aligned"),
])
def test_rms_norm_backward_rejects(kwargs, needle):
    refused(norm_back(**kwargs), needle)


def quantize(dtype=BF16, x=FAKE, xs=64, rows=4, width=64, q=FAKE, qs=64, scale=FAKE):
    return binding.lib().quantize_rows(dtype, x, xs, rows, width, q, qs, scale, None)


@pytest.mark.parametrize("kwargs,needle", [
    (dict(dtype=-1), "dtype"), (dict(rows=-1), "rows"), (dict(width=0), "width"), (dict(xs=-1), "strides"),
    (dict(qs=63), "hold a row"), (dict(x=None), "non-NULL"), (dict(q=None), "non-NULL"), (dict(scale=None), "scale"),
    (dict(dtype=F16, x=ctypes.c_void_p(0x100001)), "aligned"),
])
def test_quantize_rejects(kwargs, needle):
    refused(quantize(**kwargs), needle)


def linear(dtype=BF16, x=FAKE, xs=64, xscale=FAKE, w=FAKE, ws=64, wscale=FAKE, rows=4, width=64, outputs=32, bias=None, gelu=0,
           y=FAKE, ys=32):
    return binding.lib().linear_rows_i8(dtype, x, xs, xscale, w, ws, wscale, rows, width, outputs, bias, gelu, y, ys, None)


@pytest.mark.parametrize("kwargs,needle", [
    (dict(dtype=3), "dtype"), (dict(rows=-1), "rows"), (dict(width=0), "width"), (dict(width=2 ** 17), "width"),
    (dict(outputs=0), "outputs"), (dict(outputs=2 ** 20 + 1), "outputs"), (dict(gelu=2), "gelu"), (dict(xs=-1), "strides"),
    (dict(ws=2 ** 24), "strides"), (dict(ys=31), "hold a row"), (dict(x=None), "non-NULL"), (dict(xscale=None), "non-NULL"),
    (dict(w=None), "non-NULL"), (dict(wscale=None), "non-NULL"), (dict(y=None), "non-NULL"), (dict(dtype=F32, y=FAKE2), "aligned"),
    (dict(xscale=FAKE2), "aligned"), (dict(bias=FAKE2), "aligned"),
])
def test_linear_rejects(kwargs, needle):
    refused(linear(**kwargs), needle)


FREQ = (ctypes.c_double * 3)(1.0, 2.0, 3.0)
NAN = (ctypes.c_double * 3)(1.0, math.nan, 3.0)


def append(dtype=BF16, nk=FAKE, nks=128, nv=FAKE, nvs=128, off=FAKE, tracks=2, total=4, table=FAKE, tstride=3, columns=3,
           lengths=FAKE, xy=FAKE, time=FAKE, freq=FREQ, nt=1, ny=1, nx=1, il=0, k=FAKE, v=FAKE, ks=FAKE, vs=FAKE, pages=8, hk=2,
           dim=64):
    return binding.lib().append_tracks(dtype, nk, nks, nv, nvs, off, tracks, total, table, tstride, columns, lengths, xy, time,
                                       freq, nt, ny, nx, il, k, v, ks, vs, pages, hk, dim, None)


def attend(dtype=BF16, q=FAKE, qs=256, off=FAKE, tracks=2, total=4, table=FAKE, tstride=3, columns=3, lengths=FAKE, k=FAKE,
           v=FAKE, ks=FAKE, vs=FAKE, pages=8, hq=4, hk=2, dim=64, window=0, scale=0.125, cap=0.0, out=FAKE, os=256, ws=None, n=0):
    return binding.lib().attention_tracks(dtype, q, qs, off, tracks, total, table, tstride, columns, lengths, k, v, ks, vs, pages,
                                          hq, hk, dim, window, scale, cap, out, os, ws, n, None)


SHARED = [
    (dict(dtype=5), "dtype"), (dict(tracks=-1), "n_tracks"), (dict(total=-1), "total"), (dict(pages=-1), "pages"),
    (dict(columns=-1), "max_pages"), (dict(columns=2 ** 24 + 1), "max_pages"), (dict(tstride=-1), "table_stride"),
    (dict(hk=0), "kv_heads"), (dict(hk=257), "kv_heads"), (dict(dim=0), "head_dim"), (dict(dim=72), "head_dim"),
    (dict(dim=144), "head_dim"), (dict(off=None), "offsets"), (dict(lengths=None), "lengths"), (dict(table=None), "table"),
    (dict(k=None), "non-NULL"), (dict(vs=None), "non-NULL"), (dict(k=FAKE8), "16-byte"), (dict(v=FAKE4), "16-byte"),
    (dict(lengths=FAKE2), "4-byte"), (dict(ks=FAKE2), "4-byte"),
]


@pytest.mark.parametrize("kwargs,needle", SHARED + [
    (dict(nks=-1), "strides"), (dict(nt=-1), "pairs"), (dict(nx=31), "pairs"), (dict(freq=None), "freq"),
    (dict(freq=NAN), "finite"), (dict(nk=None), "non-NULL"), (dict(nv=None), "non-NULL"), (dict(dtype=F32, nk=FAKE2), "aligned"),
    (dict(xy=None), "xy"), (dict(time=None), "time"), (dict(xy=FAKE4), "aligned"),
])
def test_append_rejects(kwargs, needle):
    refused(append(**kwargs), needle)


@pytest.mark.parametrize("kwargs,needle", SHARED + [
    (dict(dtype=F32), "dtype"), (dict(hq=0), "multiple"), (dict(hq=3), "multiple"), (dict(hq=258), "multiple"),
    (dict(window=-1), "window"), (dict(scale=0.0), "scale"), (dict(scale=math.nan), "scale"), (dict(cap=-1.0), "cap"),
    (dict(cap=math.inf), "cap"), (dict(qs=-1), "stride"), (dict(os=255), "hold a row"), (dict(q=None), "non-NULL"),
    (dict(out=None), "non-NULL"), (dict(q=ctypes.c_void_p(0x100001)), "aligned"),
])
def test_attention_tracks_rejects(kwargs, needle):
    refused(attend(**kwargs), needle)


def test_batches_beyond_a_launch_are_refused():
    refused(append(tracks=2 ** 22, total=4), "workgroups", binding.FLOCK_EUNSUPPORTED)
    refused(append(tracks=2, total=2 ** 30), "workgroups", binding.FLOCK_EUNSUPPORTED)
    refused(attend(tracks=2 ** 23, total=4), "workgroups", binding.FLOCK_EUNSUPPORTED)
    refused(attend(total=2 ** 31 - 1), "rows", binding.FLOCK_EUNSUPPORTED)


def test_empty_calls_without_a_device():
    lib = binding.lib()
    assert norm(rows=0, x=None, y=None, w=None, rstd=None) == 0
    assert norm_i8(rows=0, x=None, y=None, w=None, scale=None) == 0
    assert norm_back(rows=0, gy=None, x=None, rstd=None, dx=None, dw=None) == 0
    assert quantize(rows=0, x=None, q=None, scale=None) == 0
    assert linear(rows=0, x=None, xscale=None, w=None, wscale=None, y=None) == 0
    assert append(tracks=0, total=0, off=None, lengths=None, table=None) == 0
    assert append(total=0) == 0
    assert append(pages=0, k=None, v=None, ks=None, vs=None) == 0
    assert attend(tracks=0, total=0, off=None) == 0
    assert attend(total=0, q=None, out=None) == 0
    assert lib.flock_last_error().decode() == ""


def test_workspace_queries():
    lib = binding.lib()
    assert lib.rms_norm_rows_backward_workspace(0, 512) == 0
    assert lib.rms_norm_rows_backward_workspace(500, 512) >= 125 * 512 * 4
    assert lib.attention_tracks_workspace(0, 0, 3, 8, 2, 64) == 0
    assert lib.attention_tracks_workspace(1, 1, 1, 8, 2, 64) == 0
    assert lib.attention_tracks_workspace(1, 1, 200, 8, 2, 64) > 0
    assert lib.attention_tracks_workspace(2, 2, 200, 8, 3, 64) == 0    # no such heads: refused by the call
